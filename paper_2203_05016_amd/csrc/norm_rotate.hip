// Norms of queries and keys per head and the rotation by position, in one pass over both.
//
//     y = x / sqrt(mean(x^2) + eps) * weight;   (a, b) -> (a cos t - b sin t, a sin t + b cos t),  t = position * frequency
//
// A lane has a part of the pairs of one token's head (few tokens), or of 8 neighbouring tokens' (many), and neighbouring lanes neighbouring tokens, so that
// the norm is a sum over a few lanes and loads are contiguous along the tokens.  All heads of a token turn by the
// same angles: a workgroup works them out once, into the LDS, and takes several heads.  The angle is a product in 64 bits, taken to
// one turn there (a position of 2^20 times a frequency, in 32 bits, leaves 0.03 radians), its sine and cosine in 32.
//
// Everything between the loads and the one rounding at the store is in 32 bits.  Squares of bfloat16 may be more than 32 bits hold, or, with an
// eps that is as small, less: such columns' sums are done again in 64, and the factor is applied in two steps.
//
// Bound by memory: 4 bytes for each value.  72 heads of 128 (bf16) by 8192 tokens, 302 MB, 56 us, 5.4 TB/s (of inputs that no cache holds 72,
// 4.2 TB/s), where a large copy moves 5.2; by 8191, whose rows are in no alignment, 76 and 87 (lines are written in parts: 175 MB each way); by 64, 5.6, a launch and one chain of latencies.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "shflbw.h"
#include "shflbw_internal.h"

namespace shflbw {
namespace {

struct RotateArgs {
    const uint16_t* in[2];     // queries, keys
    uint16_t* out[2];
    int64_t ld_in[2], ld_out[2];
    const uint16_t* weight[2];
    const int32_t* positions;
    const double* frequencies;
    const int32_t* axes;
    int64_t ldp, tokens;
    unsigned eighth, head_step;            // blocks of tokens to an XCD; heads from one of a wavefront's to its next
    int q_heads, all_heads, pairs, interleaved, norm, position_rows;
    double eps;
};

template <bool BF>
__device__ __forceinline__ float rot_widen(unsigned v)
{
    if constexpr (BF) return __builtin_bit_cast(float, v << 16);
    else return (float)__builtin_bit_cast(_Float16, (uint16_t)v);
}
template <bool BF>
__device__ __forceinline__ uint16_t rot_narrow(float f)
{
    if constexpr (BF) return __builtin_bit_cast(uint16_t, (__bf16)f);
    else return __builtin_bit_cast(uint16_t, (_Float16)f);
}
// two values to 16 bits, to nearest even
typedef float rot_float2 __attribute__((ext_vector_type(2)));
typedef _Float16 rot_half2 __attribute__((ext_vector_type(2)));
typedef __bf16 rot_bf2 __attribute__((ext_vector_type(2)));
template <bool BF>
__device__ __forceinline__ unsigned rot_pack(float a, float b)
{
    if constexpr (BF) return __builtin_bit_cast(unsigned, __builtin_convertvector((rot_float2{a, b}), rot_bf2));
    else return __builtin_bit_cast(unsigned, __builtin_convertvector((rot_float2{a, b}), rot_half2));
}
// the features of pair n: those past 2 * pairs are pairs of neighbours that are not turned
struct RotPair {
    int a, b;
};
__device__ __forceinline__ RotPair rot_features(int n, int pairs, int interleaved)
{
    if (interleaved || n >= pairs) return RotPair{2 * n, 2 * n + 1};
    return RotPair{n, n + pairs};
}
// cosine and sine of `half` half turns, |half| <= 1: Taylor's series about the nearest quarter turn, at most 1/4 away, where the first
// terms left out are below 2e-9.  Nothing branches, so that several angles are worked out side by side.
__device__ __forceinline__ float2 rot_turn(float half)
{
    const float quarter = __builtin_rintf(2 * half), r = __builtin_fmaf(-0.5f, quarter, half), z = r * r;
    // pi^n / n!
    float s = __builtin_fmaf(z, 0.0821458866f, -0.599264529f);
    s = __builtin_fmaf(z, s, 2.55016404f);
    s = __builtin_fmaf(z, s, -5.16771278f);
    s = r * __builtin_fmaf(z, s, 3.14159265f);
    float c = __builtin_fmaf(z, -0.0258068913f, 0.235330630f);
    c = __builtin_fmaf(z, c, -1.33526277f);
    c = __builtin_fmaf(z, c, 4.05871213f);
    c = __builtin_fmaf(z, c, -4.93480220f);
    c = __builtin_fmaf(z, c, 1.0f);
    const int q = (int)quarter;
    const float cosine = q & 1 ? s : c, sine = q & 1 ? c : s;
    return float2{(q + 1) & 2 ? -cosine : cosine, q & 2 ? -sine : sine};
}
// turns (u, v) by the angle of cosine c.x and sine c.y; the same roundings wherever it is called
__device__ __forceinline__ void rot_pair(float& u, float& v, float2 c)
{
    const float turned = __builtin_fmaf(u, c.x, -(v * c.y));
    v = __builtin_fmaf(u, c.y, v * c.x);
    u = turned;
}
// cosine and sine of pair n at a token's position
__device__ __forceinline__ float2 rot_angle(const RotateArgs& a, int n, int64_t token)
{
    const int row = a.axes ? a.axes[n] : 0;
    const bool known = (unsigned)row < (unsigned)a.position_rows;
    const double half = (double)a.positions[(known ? row : 0) * a.ldp + token] * a.frequencies[n] * 0.31830988618379067154;
    const float2 r = rot_turn((float)(half - 2 * __builtin_rint(half * 0.5)));
    return known ? r : float2{__builtin_nanf(""), __builtin_nanf("")};
}
// 1 / sqrt(mean + eps) as first * second, of which neither leaves 32 bits where the result is no more than they hold
struct RotFactor {
    float first, second;
};
__device__ __forceinline__ RotFactor rot_factor(double sum, int D, double eps)
{
    const double r = 1 / __builtin_sqrt(sum / D + eps);
    const float first = r < 0x1p-60 ? 0x1p-64f : r > 0x1p60 ? 0x1p64f : 1;
    return RotFactor{first, (float)(r / first)};
}

// The token of column c of a workgroup's T: runs of RUN tokens, the last of which end with the last token
template <int RUN>
__device__ __forceinline__ int64_t rot_token(const RotateArgs& a, int64_t token0, int c)
{
    const int64_t from = token0 + c / RUN * RUN;
    return (from + RUN <= a.tokens ? from : a.tokens - RUN) + c % RUN;
}
// What the two kernels share: cosines and sines of T tokens, and the weights pair by pair
template <bool BF, int D, int T, int RUN>
__device__ __forceinline__ void rot_tables(const RotateArgs& a, int64_t token0, float2 (*angle)[T], float2 (*weight)[D / 2])
{
    // (four at a time, side by side)
    const int all = a.pairs * T;
    for (int e0 = threadIdx.x; e0 < all; e0 += 1024) {
        float2 r[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int e = e0 + 256 * i < all ? e0 + 256 * i : all - 1;
            r[i] = rot_angle(a, e / T, rot_token<RUN>(a, token0, e % T));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int e = e0 + 256 * i;
            if (e < all) angle[e / T][e % T] = r[i];
        }
    }
    if (threadIdx.x < D) {
        const int kind = threadIdx.x / (D / 2), n = threadIdx.x % (D / 2);
        const RotPair f = rot_features(n, a.pairs, a.interleaved);
        weight[kind][n] = a.weight[kind] ? float2{rot_widen<BF>(a.weight[kind][f.a]), rot_widen<BF>(a.weight[kind][f.b])} : float2{1, 1};
    }
    __syncthreads();
}
// Whether a sum of squares in 32 bits can be relied on, whatever eps is.  A column of zeros is not ordinary by this, and in the kernel for many tokens the 32 or 64
// tokens of its wavefront go token by token: 72 heads of 128 by 8192 56 us, 209 if the last 5 columns are zeros, 706 if one in 32 is; by 64 tokens 5.8 whatever there is.
__device__ __forceinline__ bool rot_ordinary(float sum) { return sum > 0x1p-60f && sum < 0x1p120f; }
template <int D>
__device__ __forceinline__ float rot_root(float sum, float eps) { return __builtin_amdgcn_rsqf(sum * (1.0f / D) + eps); }

// Which tokens and heads a workgroup has.  Neighbouring tokens' rows share lines of memory where T tokens are not whole lines, so that an eighth of the
// tokens is one XCD's (the GPU deals workgroups to its eight XCDs in turn): a line is written by one L2.
struct RotPlace {
    int64_t token0;
    int heads;                 // the first of the four that a workgroup takes at a time
};
template <int T>
__device__ __forceinline__ RotPlace rot_place(const RotateArgs& a)
{
    const unsigned on = blockIdx.x % 8, i = blockIdx.x / 8;
    return RotPlace{((int64_t)on * a.eighth + i % a.eighth) * T, (int)(i / a.eighth) * 4};
}

// ---- few tokens, or rows that are far apart: T tokens and 64 / T parts of a head's pairs to a wavefront
template <bool BF, int D, int T>
__global__ __launch_bounds__(256) void norm_rotate_few_kernel(RotateArgs a)
{
    constexpr int F = 64 / T, P = D / 2 / F;
    __shared__ float2 angle[D / 2][T], weight[2][D / 2];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), t = lane % T, part = lane / T;
    const RotPlace place = rot_place<T>(a);
    const int64_t token0 = place.token0;
    if (token0 >= a.tokens) return;
    const int64_t token = rot_token<1>(a, token0, t);
    const int h0 = place.heads + wave;
    unsigned x[P];
    const auto load = [&](int h) __attribute__((always_inline)) {
        const int kind = h >= a.q_heads, head = kind ? h - a.q_heads : h;
        const uint16_t* src = a.in[kind] + (int64_t)head * D * a.ld_in[kind] + token;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const RotPair f = rot_features(part * P + i, a.pairs, a.interleaved);
            x[i] = src[f.a * a.ld_in[kind]] | (unsigned)src[f.b * a.ld_in[kind]] << 16;
        }
    };
    if (h0 < a.all_heads) load(h0);                        // on its way while the angles are worked out
    rot_tables<BF, D, T, 1>(a, token0, angle, weight);
    for (int h = h0; h < a.all_heads; h += a.head_step) {
        const int kind = h >= a.q_heads, head = kind ? h - a.q_heads : h;
        uint16_t* dst = a.out[kind] + (int64_t)head * D * a.ld_out[kind] + token;
        if (h != h0) load(h);
        RotFactor by = {1, 1};
        if (a.norm) {
            float sum = 0;
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const float u = rot_widen<BF>(x[i] & 0xffffu), v = rot_widen<BF>(x[i] >> 16);
                sum = __builtin_fmaf(u, u, __builtin_fmaf(v, v, sum));
            }
#pragma unroll
            for (int step = T; step < 64; step *= 2) sum += __shfl_xor(sum, step);
            by.second = rot_root<D>(sum, (float)a.eps);
            if (!rot_ordinary(sum)) {                      // (the lanes of a token have the same sum and go the same way)
                double wide = 0;
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const double u = rot_widen<BF>(x[i] & 0xffffu), v = rot_widen<BF>(x[i] >> 16);
                    wide += u * u + v * v;
                }
#pragma unroll
                for (int step = T; step < 64; step *= 2) wide += __shfl_xor(wide, step);
                by = rot_factor(wide, D, a.eps);
            }
        }
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int n = part * P + i;
            const RotPair f = rot_features(n, a.pairs, a.interleaved);
            const float2 w = weight[kind][n];
            float u = rot_widen<BF>(x[i] & 0xffffu) * by.first * by.second * w.x, v = rot_widen<BF>(x[i] >> 16) * by.first * by.second * w.y;
            if (n < a.pairs) {
                rot_pair(u, v, angle[n][t]);
            }
            if (token0 + t < a.tokens) {
                dst[f.a * a.ld_out[kind]] = rot_narrow<BF>(u);
                dst[f.b * a.ld_out[kind]] = rot_narrow<BF>(v);
            }
        }
    }
}

// ---- many tokens: a lane has 8 neighbouring tokens of every PARTS-th part of a head's pairs, and moves 16 bytes at a time
//
// Whatever the rows' alignment.  The last tokens are taken with those before them, whose results are dropped: tokens do not
// depend on each other, so it does not matter that another workgroup may have stored them by then.
typedef unsigned rot4 __attribute__((ext_vector_type(4)));
template <int CTRL>
__device__ __forceinline__ float rot_ror(float x)            // lanes of 16 in a circle
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
template <int RUNS>
__device__ __forceinline__ float rot_across(float x)         // the sum over lanes that are RUNS (4 or 8) apart
{
    if constexpr (RUNS == 4) x += rot_ror<0x124>(x);         // by 4
    x += rot_ror<0x128>(x);                                  // by 8
    unsigned u = __builtin_bit_cast(unsigned, x);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    x = __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
    u = __builtin_bit_cast(unsigned, x);
    const auto s = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __builtin_bit_cast(float, (unsigned)s[0]) + __builtin_bit_cast(float, (unsigned)s[1]);
}
typedef rot4 rot4_anywhere __attribute__((aligned(2)));
template <bool STREAM>
__device__ __forceinline__ void rot_store(uint16_t* p, rot4 x)
{
    if constexpr (STREAM) __builtin_nontemporal_store(x, reinterpret_cast<rot4_anywhere*>(p));
    else *reinterpret_cast<rot4_anywhere*>(p) = x;
}
template <bool BF>
__device__ __forceinline__ float rot_value(const rot4& x, int e) { return rot_widen<BF>(x[e / 2] >> 16 * (e % 2) & 0xffffu); }
template <bool BF, int D, int T, bool STREAM>
__global__ __launch_bounds__(256) void norm_rotate_kernel(RotateArgs a)
{
    constexpr int RUNS = T / 8, PARTS = 64 / RUNS, P = D / 2 / PARTS;
    __shared__ __attribute__((aligned(16))) float2 angle[D / 2][T], weight[2][D / 2];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), part = lane / RUNS, run = lane % RUNS;
    const RotPlace place = rot_place<T>(a);
    const int64_t token0 = place.token0;
    if (token0 >= a.tokens) return;
    // the first of the tokens that are loaded, and how many of them are not this lane's
    const unsigned from = (unsigned)rot_token<8>(a, token0, 8 * run);
    const int64_t before = token0 + 8 * run - from;
    const int skip = before < 8 ? (int)before : 8;
    const int h0 = place.heads + wave;
    rot4 x[P][2];
    const auto load = [&](int h) __attribute__((always_inline)) {
        const int kind = h >= a.q_heads, head = kind ? h - a.q_heads : h;
        const unsigned ld_in = (unsigned)a.ld_in[kind];
        const uint16_t* src = a.in[kind] + (int64_t)head * D * ld_in;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const RotPair f = rot_features(i * PARTS + part, a.pairs, a.interleaved);
            __builtin_memcpy(&x[i][0], src + (f.a * ld_in + from), 16);
            __builtin_memcpy(&x[i][1], src + (f.b * ld_in + from), 16);
        }
    };
    if (h0 < a.all_heads) load(h0);                        // on its way while the angles are worked out
    rot_tables<BF, D, T, 8>(a, token0, angle, weight);
    for (int h = h0; h < a.all_heads; h += a.head_step) {
        const int kind = h >= a.q_heads, head = kind ? h - a.q_heads : h;
        const unsigned ld_in = (unsigned)a.ld_in[kind], ld_out = (unsigned)a.ld_out[kind];
        const uint16_t* src = a.in[kind] + (int64_t)head * D * ld_in;
        uint16_t* dst = a.out[kind] + (int64_t)head * D * ld_out;
        if (h != h0) load(h);
        float by[8];
        bool ordinary = true;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            by[e] = 1;
            if (!a.norm) continue;
            float sum = 0;
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const float u = rot_value<BF>(x[i][0], e), v = rot_value<BF>(x[i][1], e);
                sum = __builtin_fmaf(u, u, __builtin_fmaf(v, v, sum));
            }
            sum = rot_across<RUNS>(sum);
            ordinary &= rot_ordinary(sum);
            by[e] = rot_root<D>(sum, (float)a.eps);
        }
        if (__all(ordinary)) {
            // (what was widened for the sums is widened again, not kept: bfloat16 heads of 128 took 254 registers)
#pragma unroll
            for (int i = 0; i < P; ++i) asm volatile("" : "+v"(x[i][0]), "+v"(x[i][1]));
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const int n = i * PARTS + part;
                const RotPair f = rot_features(n, a.pairs, a.interleaved);
                const float2 w = weight[kind][n];
                float u[8], v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    u[e] = rot_value<BF>(x[i][0], e) * by[e] * w.x;
                    v[e] = rot_value<BF>(x[i][1], e) * by[e] * w.y;
                }
                if (n < a.pairs) {
                    const float4* c = reinterpret_cast<const float4*>(&angle[n][8 * run]);
#pragma unroll
                    for (int e = 0; e < 8; e += 2) {
                        const float4 t = c[e / 2];
                        rot_pair(u[e], v[e], float2{t.x, t.y});
                        rot_pair(u[e + 1], v[e + 1], float2{t.z, t.w});
                    }
                }
                uint16_t* p = dst + (f.a * ld_out + from);
                uint16_t* q = dst + (f.b * ld_out + from);
                rot4 y, z;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    y[e] = rot_pack<BF>(u[2 * e], u[2 * e + 1]);
                    z[e] = rot_pack<BF>(v[2 * e], v[2 * e + 1]);
                }
                if (skip == 0) {
                    rot_store<STREAM>(p, y);
                    rot_store<STREAM>(q, z);
                } else {

#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (e >= skip) {
                            p[e] = (uint16_t)(y[e / 2] >> 16 * (e % 2));
                            q[e] = (uint16_t)(z[e / 2] >> 16 * (e % 2));
                        }
                }
                __builtin_amdgcn_sched_barrier(0);         // (pairs one after the other: registers for three workgroups on a CU)
            }
            continue;
        }
        // a token whose squares 32 bits do not hold is among them: token by token, from memory again
#pragma unroll 1
        for (int e = 0; e < 8; ++e) {
            float sum = 0;
            double wide = 0;
#pragma unroll 1
            for (int i = 0; i < P; ++i) {
                const RotPair f = rot_features(i * PARTS + part, a.pairs, a.interleaved);
                const float u = rot_widen<BF>(src[f.a * ld_in + from + e]), v = rot_widen<BF>(src[f.b * ld_in + from + e]);
                sum = __builtin_fmaf(u, u, __builtin_fmaf(v, v, sum));   // (as above, bit for bit)
                wide += (double)u * u + (double)v * v;
            }
            sum = rot_across<RUNS>(sum);
#pragma unroll
            for (int step = RUNS; step < 64; step *= 2) wide += __shfl_xor(wide, step);
            const RotFactor factor = rot_ordinary(sum) ? RotFactor{1, rot_root<D>(sum, (float)a.eps)} : rot_factor(wide, D, a.eps);
#pragma unroll 1
            for (int i = 0; i < P; ++i) {
                const int n = i * PARTS + part;
                const RotPair f = rot_features(n, a.pairs, a.interleaved);
                const float2 w = weight[kind][n];
                float u = rot_widen<BF>(src[f.a * ld_in + from + e]) * factor.first * factor.second * w.x;
                float v = rot_widen<BF>(src[f.b * ld_in + from + e]) * factor.first * factor.second * w.y;
                if (n < a.pairs) rot_pair(u, v, angle[n][8 * run + e]);
                if (e >= skip) {
                    dst[f.a * ld_out + from + e] = rot_narrow<BF>(u);
                    dst[f.b * ld_out + from + e] = rot_narrow<BF>(v);
                }
            }
        }
    }
}

template <bool BF, int D>
int launch(RotateArgs a, hipStream_t stream)
{
    bool near = true, whole = true;                        // offsets inside a head are 32 bits of 2 bytes; runs of 32 tokens are 64 whole bytes of memory
    for (int i = 0; i < 2; ++i) {
        near &= a.ld_in[i] < 1 << 23 && a.ld_out[i] < 1 << 23;
        whole &= a.ld_out[i] % 32 == 0 && reinterpret_cast<uintptr_t>(a.out[i]) % 64 == 0;
    }
    // In heads of 128, us: 72 heads by 64, 128 and 256 tokens, 4 tokens to a wavefront 5.6, 6.5 and 9.5, 8 tokens 6.0, 6.2 and 7.4, 32 in runs of 8
    // 7.5, 7.4 and 7.6; 5 heads by 64, 512 and 4096 4.2, 4.4 and 9.5, 5.0, 5.1 and 7.8, 6.5, 6.7 and 7.7: a wavefront's instructions, fetched once,
    // are most of what few tokens take.
    const int64_t work = a.tokens * a.all_heads;
    const bool many = near && a.tokens >= 8 && work > 18000;
    // Results of 16 MB and more leave past the L2s, if in whole 64 bytes: 72 by 8192 56 us, through them 76, by 1024 10.4 and 12.8, by 8191, in parts of lines, 136
    // and 91.  Such rows take 64 tokens to a wavefront where there are many, 76, of 32 82 (by 2048 28 and 21).
    const bool stream_out = whole && work * D * 2 >= 16 << 20, wide = !whole && work >= 300000;
    const int T = many ? (wide ? 64 : 32) : work <= 6000 ? 4 : 8;
    const int64_t eighth = (a.tokens + 8 * T - 1) / (8 * T);
    // heads to a workgroup: as many as leave 4096 workgroups, the same number to each.  72 heads of 128 by 8191, 8192 and 4099 tokens that no cache holds:
    // 87, 72 and 50 us, with 1024 workgroups 95, 84 and 55, with 512 99, 84 and 58; with four heads to each 88, 74 and 50.
    const int64_t steps = ((int64_t)a.all_heads + 3) / 4, wanted = (4096 + 8 * eighth - 1) / (8 * eighth), each = (steps + wanted - 1) / wanted;
    const int64_t parts = (steps + each - 1) / each, blocks = 8 * eighth * parts;
    if (blocks > 0x7fffffffLL) return fail(SHFLBW_ERR_BAD_SHAPE, "grid too large");
    a.eighth = (unsigned)eighth;
    a.head_step = (unsigned)(4 * parts);
    const dim3 grid((unsigned)blocks);
    if (many && wide) hipLaunchKernelGGL((norm_rotate_kernel<BF, D, 64, false>), grid, dim3(256), 0, stream, a);
    else if (many && stream_out) hipLaunchKernelGGL((norm_rotate_kernel<BF, D, 32, true>), grid, dim3(256), 0, stream, a);
    else if (many) hipLaunchKernelGGL((norm_rotate_kernel<BF, D, 32, false>), grid, dim3(256), 0, stream, a);
    else if (T == 4) hipLaunchKernelGGL((norm_rotate_few_kernel<BF, D, 4>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((norm_rotate_few_kernel<BF, D, 8>), grid, dim3(256), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(SHFLBW_ERR_HIP, "kernel launch: %s", hipGetErrorString(e));
    return SHFLBW_OK;
}

// Rows of `columns` values of 2 bytes: whether two such matrices share any
struct Rows {
    const void* base;
    int64_t rows, columns, ld;
};
bool overlap(const Rows& x, const Rows& y)
{
    const uintptr_t a = reinterpret_cast<uintptr_t>(x.base), b = reinterpret_cast<uintptr_t>(y.base);
    const uintptr_t a_end = a + 2 * ((x.rows - 1) * x.ld + x.columns), b_end = b + 2 * ((y.rows - 1) * y.ld + y.columns);
    if (x.rows == 0 || y.rows == 0 || a_end <= b || b_end <= a) return false;
    if (x.ld != y.ld) return true;
    // side by side in the same rows
    const int64_t pitch = 2 * x.ld, d = ((int64_t)(b - a) % pitch + pitch) % pitch;
    return d < 2 * x.columns || pitch - d < 2 * y.columns;
}

}  // namespace
}  // namespace shflbw

extern "C" int shflbw_norm_rotate(const shflbw_rotation* r, const int32_t* positions, int64_t ldp, const void* q, int64_t ldq, int q_heads,
                                  const void* k, int64_t ldk, int heads, void* q_out, int64_t ldqo, void* k_out, int64_t ldko, int64_t tokens,
                                  void* stream)
{
    using namespace shflbw;
    if (!r) return fail(SHFLBW_ERR_NULL_ARG, "rotation is NULL");
    if (r->dtype != SHFLBW_F16 && r->dtype != SHFLBW_BF16) return fail(SHFLBW_ERR_BAD_DTYPE, "dtype must be SHFLBW_F16 or SHFLBW_BF16");
    const int D = r->head_dim;
    if (D != 64 && D != 96 && D != 128) return fail(SHFLBW_ERR_BAD_SHAPE, "head_dim must be 64, 96 or 128");
    if (r->pairs < 0 || r->pairs > D / 2) return fail(SHFLBW_ERR_BAD_SHAPE, "pairs must be 0 to head_dim / 2");
    if (q_heads < 0 || heads < 0 || q_heads > 65535 || heads > 65535) return fail(SHFLBW_ERR_BAD_SHAPE, "heads must be 0 to 65535");
    if (tokens < 0) return fail(SHFLBW_ERR_BAD_SHAPE, "tokens < 0");
    if (r->norm && !(r->eps >= 0 && r->eps < __builtin_inf())) return fail(SHFLBW_ERR_BAD_SHAPE, "eps must be finite and not negative");
    if (tokens == 0 || q_heads + heads == 0) return SHFLBW_OK;
    if ((q_heads && (!q || !q_out)) || (heads && (!k || !k_out))) return fail(SHFLBW_ERR_NULL_ARG, "q, k and their results must not be NULL");
    if ((q_heads && (ldq < tokens || ldqo < tokens)) || (heads && (ldk < tokens || ldko < tokens)))
        return fail(SHFLBW_ERR_BAD_SHAPE, "leading dimension too small");
    if (r->pairs && (!positions || !r->frequencies)) return fail(SHFLBW_ERR_NULL_ARG, "positions and frequencies must not be NULL");
    if (r->pairs && (r->position_rows < 1 || ldp < tokens)) return fail(SHFLBW_ERR_BAD_SHAPE, "position_rows < 1 or ldp < tokens");
    const Rows in[2] = {{q, (int64_t)q_heads * D, tokens, ldq}, {k, (int64_t)heads * D, tokens, ldk}};
    const Rows out[2] = {{q_out, (int64_t)q_heads * D, tokens, ldqo}, {k_out, (int64_t)heads * D, tokens, ldko}};
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2; ++j)
            if (overlap(out[i], in[j]) && !(i == j && out[i].base == in[i].base && out[i].ld == in[i].ld))
                return fail(SHFLBW_ERR_BAD_SHAPE, "results overlap q or k other than in place");
    if (overlap(out[0], out[1])) return fail(SHFLBW_ERR_BAD_SHAPE, "q_out and k_out overlap");
    RotateArgs a = {};
    a.in[0] = static_cast<const uint16_t*>(q);
    a.in[1] = static_cast<const uint16_t*>(k);
    a.out[0] = static_cast<uint16_t*>(q_out);
    a.out[1] = static_cast<uint16_t*>(k_out);
    a.ld_in[0] = ldq; a.ld_in[1] = ldk;
    a.ld_out[0] = ldqo; a.ld_out[1] = ldko;
    if (r->norm) {
        a.weight[0] = static_cast<const uint16_t*>(r->q_weight);
        a.weight[1] = static_cast<const uint16_t*>(r->k_weight);
    }
    a.positions = positions;
    a.frequencies = r->frequencies;
    a.axes = r->axes;
    a.ldp = ldp;
    a.tokens = tokens;
    a.q_heads = q_heads;
    a.all_heads = q_heads + heads;
    a.pairs = r->pairs;
    a.interleaved = r->interleaved != 0;
    a.norm = r->norm != 0;
    a.position_rows = r->position_rows;
    a.eps = r->eps;
    typedef int (*launcher)(RotateArgs, hipStream_t);
    static const launcher table[2][3] = {{&launch<false, 64>, &launch<false, 96>, &launch<false, 128>},
                                         {&launch<true, 64>, &launch<true, 96>, &launch<true, 128>}};
    return table[r->dtype == SHFLBW_BF16][D / 32 - 2](a, static_cast<hipStream_t>(stream));
}
