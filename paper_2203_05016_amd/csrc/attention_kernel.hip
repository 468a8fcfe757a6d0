// Attention kernels: few queries over the 4-bit cache, tiles of queries over the cache or over a prompt's own keys and
// values, and the join of parts.  Weights are softmax(q.k / sqrt(D)) over the keys a query sees.
//
// All compute transposed products, so that activations stay features x tokens: the scores of a tile are K Q (rows keys,
// columns queries), the result is V^T P.  The running maximum and sum of a query's softmax are then one lane's, and a
// score's place among the lanes of the accumulators is, up to the order of the keys, its place among the lanes of the
// operand P of the second product: nothing is exchanged between lanes but the maximum.  The reduction over keys
// takes any order, as long as both operands have the same.
//
// Sums, maxima and accumulators are in 32 bits.  The weights are rounded to the operands' 16 bits for the second
// product, which has no wider operands at its rate (half a step: relative 2^-11 or 2^-8 of each, beside the same rounding of the result; in binary16 at
// most 2^-31 of the largest where they are subnormal).  Keys read from the cache are
// exact in 16 bits but for binary16 blocks below 2^-21, whose values are rounded to multiples of 2^-24.
//
// A query whose mask leaves nothing gets zeros.  Infinities and NaN in keys or values that a query does not see leave
// it alone; those it sees reach its result.
#pragma once
#include <hip/hip_runtime.h>

#include <cfloat>
#include <cstdint>
#include <type_traits>

#include "attention.h"

namespace shflbw {

typedef unsigned short ushort8v __attribute__((ext_vector_type(8)));
typedef unsigned uint4v __attribute__((ext_vector_type(4)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 b16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 b16x2 __attribute__((ext_vector_type(2)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef short short4w __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char* attn_lds;
typedef __attribute__((address_space(3))) short4w* attn_lds4;

template <bool BF>
__device__ __forceinline__ float4v attn_mma16(uint4v a, uint4v b, float4v c)
{
    if constexpr (BF) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b16x8, a), __builtin_bit_cast(b16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
template <bool BF>
__device__ __forceinline__ float16v attn_mma32(uint4v a, uint4v b, float16v c)
{
    if constexpr (BF) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b16x8, a), __builtin_bit_cast(b16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
// two values to 16 bits, to nearest even
template <bool BF>
__device__ __forceinline__ unsigned attn_pack(float a, float b)
{
    if constexpr (BF) return __builtin_bit_cast(unsigned, __builtin_convertvector((float2v{a, b}), b16x2));
    else return __builtin_bit_cast(unsigned, __builtin_convertvector((float2v{a, b}), f16x2));
}
template <bool BF>
__device__ __forceinline__ uint16_t attn_narrow(float f)
{
    if constexpr (BF) return __builtin_bit_cast(uint16_t, (__bf16)f);
    else return __builtin_bit_cast(uint16_t, (_Float16)f);
}
template <bool BF>
__device__ __forceinline__ float attn_widen(uint16_t v)
{
    if constexpr (BF) return __builtin_bit_cast(float, (unsigned)v << 16);
    else return (float)__builtin_bit_cast(_Float16, v);
}
// A word of 8 codes under the scale whose byte is `code`, as 8 values of 16 bits.  The conversion takes the scale's
// exponent field and gives NaN for 255.
template <bool BF>
__device__ __forceinline__ uint4v attn_unpack(unsigned word, unsigned code)
{
    const float scale = __builtin_bit_cast(float, code << 23);
    uint4v r;
    if constexpr (BF) {
        r[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 0));
        r[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 1));
        r[2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 2));
        r[3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 3));
    } else {
        r[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(word, scale, 0));
        r[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(word, scale, 1));
        r[2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(word, scale, 2));
        r[3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(word, scale, 3));
    }
    return r;
}
// a lane's value and that of the lane 32 (16) away
__device__ __forceinline__ float2v attn_pair32(float x)
{
    const unsigned u = __builtin_bit_cast(unsigned, x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return float2v{__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1])};
}
__device__ __forceinline__ float2v attn_pair16(float x)
{
    const unsigned u = __builtin_bit_cast(unsigned, x);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return float2v{__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1])};
}
__device__ __forceinline__ float attn_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// Four keys (rows) x 16 features of a 16-lane block, transposed: lane i gets the block's four rows of feature i
__device__ __forceinline__ uint2 attn_transposed(attn_lds p)
{
    return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((attn_lds4)p));
}

// Tables that nothing writes while a kernel runs, read at addresses that a wavefront's lanes share: through the scalar cache, so that
// the wait for an entry is not one for the vector loads in flight
typedef const __attribute__((address_space(4))) int32_t* attn_table;
__device__ __forceinline__ attn_table attn_scalar(const int32_t* p) { return (attn_table)(uintptr_t)p; }

// One sequence of a call
struct AttnSeq {
    int64_t t0;    // its first column of q
    int nq, len;   // queries, and keys up to the last query's own
    bool bad;      // longer than its pages can be
};
template <bool CACHE>
__device__ __forceinline__ AttnSeq attn_sequence(const AttnArgs& a, int b)
{
    AttnSeq s;
    int64_t t0 = CACHE ? b : 0, t1 = CACHE ? b + 1 : a.tokens;
    if (a.starts) {
        t0 = attn_scalar(a.starts)[b];
        t1 = attn_scalar(a.starts)[b + 1];
    }
    t0 = t0 < 0 ? 0 : t0;
    t1 = t1 > a.tokens ? a.tokens : t1;
    s.t0 = t0;
    s.nq = t1 > t0 ? (int)(t1 - t0) : 0;
    s.bad = false;
    if constexpr (CACHE) {
        const int64_t most = (int64_t)a.table_width << a.page_shift;
        const int len = attn_scalar(a.lengths)[b];
        s.bad = len > most;
        s.len = s.bad ? (int)most : len < 0 ? 0 : len;
    } else {
        s.len = s.nq;
    }
    return s;
}

// The tiles of keys (shifted by `shift`: tile t holds keys tile * t - shift and up) that queries at positions first..last need: those of
// the sinks, then those of the window
struct AttnTiles {
    int sinks;     // tiles before the window's that sinks lie in
    int window;    // the window's first tile
    int count;
    __device__ __forceinline__ int real(int v) const { return v < sinks ? v : v - sinks + window; }
};
__device__ __forceinline__ AttnTiles attn_tiles(int first, int last, int window, int sinks, int shift, int tile)
{
    AttnTiles t = {0, 0, 0};
    if (last < 0) return t;
    const int64_t low = (int64_t)first - window + 1;
    const int lo = low > 0 ? (int)low : 0;
    t.window = (int)(((int64_t)lo + shift) / tile);
    const int64_t sink_end = lo < sinks ? lo : sinks;
    const int n = (int)((sink_end + (sink_end > 0 ? shift : 0) + tile - 1) / tile);
    t.sinks = n < t.window ? n : t.window;
    t.count = t.sinks + (int)(((int64_t)last + shift) / tile) + 1 - t.window;
    return t;
}
// whether a query at position p, whose window begins at key lo (or before the first), sees key j
__device__ __forceinline__ bool attn_sees(int j, int p, int lo, int sinks) { return (unsigned)j <= (unsigned)p && p >= 0 && (j >= lo || j < sinks); }
__device__ __forceinline__ int attn_window_start(int p, int window) { return p < window ? 0 : p - window + 1; }

// The maximum that scores are taken off follows the true one only when that has grown by this many powers of two: rescaling the
// accumulators is rare then, and weights stay below 2^ATTN_SLACK.
constexpr float ATTN_SLACK = 8;
// In binary16 that maximum is taken 2^6 lower, so that all weights are 2^6 times as large: there are none below 2^-24, and a key of weight 1 beside
// 40000 of 2^-26 lost all of these.  Now what is lost of a weight is at most 2^-31 of the largest.  The largest may be 2^(6 + ATTN_SLACK), a fourth of
// what binary16 holds: room for the rounding of the maximum itself (half a step of it is below 2 while scores times log2(e) stay below 2^25).
template <bool BF>
constexpr float ATTN_LIFT = BF ? 0 : 6;
// (not in assembly: matrix results need wait states before a vector instruction reads them, which the compiler puts in)
__device__ __forceinline__ float attn_max3(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }

// ---- few queries over the cache
//
// A workgroup takes one sequence, key head and part of the keys, and up to 16 NT columns: a column is one query head of the
// key head's group, of one query.  Its wavefronts take tiles of 32 keys in turn, each with its own maximum, sum
// and accumulators, and join through the LDS at the end.  Bound by the cache's bytes: a value is read once, as four bits.
// The keys' words unpack in the registers of the lane that hands them to the matrix instruction; the
// values' words belong to one key each (they share its scale) where the second product wants eight keys of one
// feature per lane, so they go through a tile of LDS that only this wavefront uses and come back by transposing reads.
// Loads are two tiles ahead, page numbers three: no wait but for the tile at hand.
//
// Measured: 64 sequences of 819 to 4096 keys, 64 query heads over 8 of 128 (bf16), 189 MB: 40 us, 4.7 TB/s, where a large copy moves 5.1;
// 2 of 131071 keys (f16, 277 MB) 48 us, 5.8 TB/s (part of it lies in the memory-side cache), and 4.2 for the join; 128 under a window of
// 1024 with 4 sinks, 16 heads of 64, 144 MB: 30 us, 4.7 TB/s.  Vector instructions are issued in 32 % of the cycles, the matrix units busy in 10.
// With 5 queries each (48 columns; 24 sequences of up to 3001 keys, 56 MB) 34 us: a CU has 8 wavefronts, half of the CUs none.
template <bool BF, int D, int NT, int W>
__global__ __launch_bounds__(64 * W, decode_residency(NT, D)) void attention_decode_kernel(AttnArgs a)
{
    constexpr int S = D / 32, DT = D / 16, C = 16 * NT;
    constexpr int VP = 2 * D + 32;                        // LDS pitch of a key's values: 8 rows x 32 bytes in 64 banks
    constexpr int OP = D + 4;                             // pitch of a column's sums, in floats
    constexpr int QP = 2 * D + 16;                        // pitch of a column's query: 16 rows in different banks
    constexpr int SB = scale_bytes(D);
    constexpr int V_BYTES = W * 32 * VP, O_BYTES = W * 16 * OP * 4, Q_BYTES = C * QP;
    constexpr int BYTES = V_BYTES > O_BYTES ? (V_BYTES > Q_BYTES ? V_BYTES : Q_BYTES) : (O_BYTES > Q_BYTES ? O_BYTES : Q_BYTES);
    __shared__ __attribute__((aligned(16))) char smem[BYTES];
    __shared__ float stat[W][C][2];
    __shared__ int64_t where[C];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int quarter = lane >> 4, r = lane & 15;
    const int split = blockIdx.x % a.splits, rest = blockIdx.x / a.splits, block = rest % a.col_blocks, pair = rest / a.col_blocks;
    const int b = pair / a.heads, h = pair % a.heads;

    // a block of columns is a whole number of queries
    AttnSeq seq = attn_sequence<true>(a, b);
    const int skipped = block * (C / a.group), left = seq.nq - skipped;
    if (left <= 0) return;
    const int cols = (left < C / a.group ? left : C / a.group) * a.group;
    seq.t0 += skipped;
    const int p_first = seq.len - left, p_last = p_first + (cols - 1) / a.group;
    const AttnTiles tiles = attn_tiles(p_first, p_last, a.window, a.sinks, 0, ATTN_DECODE_KEYS);
    const int v_begin = split * a.split_tiles;
    // the last part takes what is left, also of a sequence longer than the plan was told
    const int v_end = split + 1 == a.splits || tiles.count - v_begin < a.split_tiles ? tiles.count : v_begin + a.split_tiles;

    const int page = 1 << a.page_shift;
    const int64_t chunk = page_head_bytes(page, D), page_bytes = chunk * a.heads;
    const char* pages = a.cache + h * chunk;
    const attn_table table = attn_scalar(a.table + (int64_t)b * a.table_ld);
    const int v_row = ((lane >> 4) & 1) * 8 + ((lane >> 1) & 7), v_part = (lane & 1) + 2 * (lane >> 5);   // of the values' words (value_lane)

    struct Raw {
        unsigned k[2][S], v[2][S], ks[2], vs[2];
        bool known;                                       // there is such a page
    };
    // page of tile v; tiles past the end read what the last one does
    const auto page_of = [&](int v) __attribute__((always_inline)) {
        return table[tiles.real(v < v_end ? v : v_end - 1) * ATTN_DECODE_KEYS >> a.page_shift];
    };
    const auto load = [&](Raw& x, int v, int id) __attribute__((always_inline)) {
        const bool known = (unsigned)id < (unsigned)a.pages;
        const int at = tiles.real(v < v_end ? v : v_end - 1) * ATTN_DECODE_KEYS & (page - 1);
        const char* base = pages + (known ? id : 0) * page_bytes;
        const char* codes = base + code_offset(D, at, 0);
        const unsigned code_lane = D == 64 ? lane * 16 : lane * (D / 8);
#pragma unroll
        for (int kind = 0; kind < 2; ++kind, codes += page * (D / 2)) {
            unsigned(&w)[2][S] = kind ? x.v : x.k;
            if constexpr (D == 64) {
                const uint4v t = *reinterpret_cast<const uint4v*>(codes + code_lane);
                w[0][0] = t[0]; w[0][1] = t[1]; w[1][0] = t[2]; w[1][1] = t[3];
            } else {
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int s = 0; s < S; ++s) w[u][s] = reinterpret_cast<const unsigned*>(codes + code_lane + u * D * 8)[s];
            }
        }
        const char* ks = base + page * D + at * SB;
        const char* vs = ks + page * SB;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const unsigned k_lane = (16 * u + r) * SB, v_lane = (16 * u + v_row) * SB;
            x.ks[u] = SB == 2 ? *reinterpret_cast<const uint16_t*>(ks + k_lane) : *reinterpret_cast<const unsigned*>(ks + k_lane);
            x.vs[u] = SB == 2 ? *reinterpret_cast<const uint16_t*>(vs + v_lane) : *reinterpret_cast<const unsigned*>(vs + v_lane);
        }
        x.known = known;
    };

    // the first two tiles travel while the queries are fetched
    Raw even = {}, odd = {};
    int id = 0;
    if (v_begin < v_end) {
        const int id0 = page_of(v_begin + wave), id1 = page_of(v_begin + wave + W);
        load(even, v_begin + wave, id0);
        load(odd, v_begin + wave + W, id1);
        id = page_of(v_begin + wave + 2 * W);
    }

    // queries: through the LDS once, columns x features, then as operands in registers.  A lane fetches one column's; neighbouring
    // lanes take neighbouring queries of a head, which share lines of memory.
    uint4v q[NT][S];
    int p[NT], lo[NT];
    {
        constexpr int CP = C == 48 ? 64 : C, FS = 64 / CP;    // lanes per feature, features at a time
        const int n = lane & (CP - 1), f0 = wave * FS + lane / CP, queries = cols / a.group;   // (a whole number: up to C columns in all)
        const bool real = n < cols;
        const int g = real ? n / queries : 0, i = real ? n % queries : 0, c = real ? i * a.group + g : n;
        const uint16_t* src = a.q + ((int64_t)(h * a.group + g) * D + f0) * a.ldq + seq.t0 + i;
        uint16_t x[D / (W * FS)];
#pragma unroll
        for (int k = 0; k < D / (W * FS); ++k) x[k] = src[(int64_t)(k * W * FS) * a.ldq];
        if (c < C)
#pragma unroll
            for (int k = 0; k < D / (W * FS); ++k) *reinterpret_cast<uint16_t*>(smem + c * QP + (f0 + k * W * FS) * 2) = real ? x[k] : 0;
        // where a column's results go: head and token
        if (wave == 0 && n < C) where[c] = a.splits == 1 ? (int64_t)(h * a.group + g) * D * a.ldo + seq.t0 + i
                                                         : ((int64_t)split * a.heads * a.group + h * a.group + g) * a.tokens + seq.t0 + i;
        __syncthreads();
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int s = 0; s < S; ++s) q[n][s] = *reinterpret_cast<const uint4v*>(smem + (16 * n + r) * QP + (32 * s + 8 * quarter) * 2);
        __syncthreads();
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int col = 16 * n + r;
            p[n] = col < cols ? p_first + col / a.group : -1;
            lo[n] = attn_window_start(p[n], a.window);
        }
    }

    float4v o[NT][DT] = {};
    float m[NT], l[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) { m[n] = -FLT_MAX; l[n] = 0; }

    char* vt = smem + wave * 32 * VP;
    char* vw = vt + v_row * VP + v_part * 16;
    const attn_lds vr = (attn_lds)vt + (4 * quarter + (r >> 2)) * VP + (r & 3) * 8;
    const int window_last = attn_window_start(p_last, a.window);

    bool special = false;
    // whether not all columns see all 32 keys from j on
    const auto is_masked = [&](int j) __attribute__((always_inline)) { return j + 31 > p_first || (j < window_last && j + 31 >= a.sinks); };
    const auto work = [&](Raw& raw, int v) __attribute__((always_inline)) {
        const int j0 = tiles.real(v) * ATTN_DECODE_KEYS;
        if (!raw.known)                                   // a page that is not there reads as NaN
#pragma unroll
            for (int u = 0; u < 2; ++u) raw.ks[u] = raw.vs[u] = 0xffffffffu;
        const bool masked = is_masked(j0);
        // values of keys that only some columns see must not reach the others as 0 * NaN: such blocks are zeros here,
        // and become NaN at the end where they are seen
        if (masked)
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int s = 0; s < S; ++s)
                    if ((raw.vs[u] >> 8 * s & 255) > most_scale(BF)) {
                        special = true;
                        raw.vs[u] &= ~(255u << 8 * s);
                        raw.v[u][s] = 0;
                    }

#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int s = 0; s < S; ++s) *reinterpret_cast<uint4v*>(vw + 16 * u * VP + s * 64) = attn_unpack<BF>(raw.v[u][s], raw.vs[u] >> 8 * s & 255);
        float4v sc[NT][2] = {};
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int s = 0; s < S; ++s) {
                const uint4v k = attn_unpack<BF>(raw.k[u][s], raw.ks[u] >> 8 * s & 255);
#pragma unroll
                for (int n = 0; n < NT; ++n) sc[n][u] = attn_mma16<BF>(k, q[n][s], sc[n][u]);
            }
        load(raw, v + 2 * W, id);
        id = page_of(v + 3 * W);

        uint4v w[NT];
        if (masked)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (!attn_sees(j0 + (i >> 2) * 16 + quarter * 4 + (i & 3), p[n], lo[n], a.sinks)) sc[n][i >> 2][i & 3] = -INFINITY;
        float top[NT];
        bool grown = false;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const float4v x = sc[n][0], y = sc[n][1];
            top[n] = attn_max3(attn_max3(x[0], x[1], x[2]), attn_max3(x[3], y[0], y[1]), attn_max3(y[2], y[3], y[3])) * a.scale;
            grown |= top[n] > m[n] + (ATTN_SLACK + ATTN_LIFT<BF>);
        }
        if (__any(grown))
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float2v t = attn_pair16(top[n]);
                t = attn_pair32(attn_max3(t[0], t[1], t[1]));
                const float now = fmaxf(fmaxf(t[0], t[1]) - ATTN_LIFT<BF>, m[n]), shrink = attn_exp2(m[n] - now);
                m[n] = now;
                l[n] *= shrink;
#pragma unroll
                for (int d = 0; d < DT; ++d) o[n][d] *= shrink;
            }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = attn_exp2(__builtin_fmaf(sc[n][i >> 2][i & 3], a.scale, -m[n]));
            l[n] += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
#pragma unroll
            for (int i = 0; i < 4; ++i) w[n][i] = attn_pack<BF>(x[2 * i], x[2 * i + 1]);
        }

        asm volatile("" ::: "memory");
#pragma unroll
        for (int t = 0; t < DT; ++t) {
            const uint2 one = attn_transposed(vr + t * 32), two = attn_transposed(vr + 16 * VP + t * 32);
            const uint4v x = {one.x, one.y, two.x, two.y};
#pragma unroll
            for (int n = 0; n < NT; ++n) o[n][t] = attn_mma16<BF>(x, w[n], o[n][t]);
        }
        asm volatile("" ::: "memory");
    };
    for (int v = v_begin + wave; v < v_end; v += W) {
        work(even, v);
        v += W;
        if (v >= v_end) break;
        work(odd, v);
    }

    if (__any(special))
        for (int v = v_begin + wave; v < v_end; v += W) {
            const int j0 = tiles.real(v) * ATTN_DECODE_KEYS;
            if (!is_masked(j0)) continue;
            for (int j = j0; j < j0 + ATTN_DECODE_KEYS && j <= p_last; ++j) {
                const int page_j = table[j >> a.page_shift];
                const bool there = (unsigned)page_j < (unsigned)a.pages;
                const char* scales = pages + (there ? page_j : 0) * page_bytes + (int64_t)page * D + (int64_t)(page + (j & (page - 1))) * SB;
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    if (attn_sees(j, p[n], lo[n], a.sinks))
#pragma unroll
                        for (int t = 0; t < DT; ++t)
                            if (!there || (unsigned char)scales[t / 2] > most_scale(BF)) o[n][t] += __builtin_nanf("");
            }
        }

    // join the wavefronts: every lane knows its column's maximum and sum over all of them
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        float2v t = attn_pair16(l[n]);
        t = attn_pair32(t[0] + t[1]);
        l[n] = t[0] + t[1];
        if (quarter == 0) {
            stat[wave][16 * n + r][0] = m[n];
            stat[wave][16 * n + r][1] = l[n];
        }
    }
    __syncthreads();
    float* sums = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int col = 16 * n + r;
        if (16 * n >= cols) break;
        float top = -FLT_MAX, total = 0;
#pragma unroll
        for (int i = 0; i < W; ++i) top = fmaxf(top, stat[i][col][0]);
#pragma unroll
        for (int i = 0; i < W; ++i) total += stat[i][col][1] * attn_exp2(stat[i][col][0] - top);
        if (seq.bad) total = __builtin_nanf("");
        float f = attn_exp2(m[n] - top);
        if (a.splits == 1) f = p[n] < 0 ? 0 : f / total;
        else if (seq.bad) f = total;
        if (a.splits > 1 && wave == 0 && quarter == 0 && col < cols) {
            const int64_t row = where[col];
            a.part_ml[2 * row] = p[n] < 0 ? -INFINITY : top;
            a.part_ml[2 * row + 1] = total;
        }
#pragma unroll
        for (int t = 0; t < DT; ++t) *reinterpret_cast<float4v*>(sums + (wave * 16 + r) * OP + 16 * t + 4 * quarter) = o[n][t] * f;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 16 * D / (64 * W); ++k) {
            const int e = threadIdx.x + k * 64 * W, c = e / D, d = e % D, at = 16 * n + c;
            if (at >= cols) break;
            float x = 0;
#pragma unroll
            for (int i = 0; i < W; ++i) x += sums[(i * 16 + c) * OP + d];
            if (a.splits == 1) a.out[where[at] + d * a.ldo] = attn_narrow<BF>(x);
            else a.part_o[where[at] * D + d] = x;
        }
        __syncthreads();
    }
}

// ---- tiles of queries
//
// A workgroup of W wavefronts takes one sequence and key head and W items, one per wavefront: 32 neighbouring queries of one of
// the group's heads; heads vary fastest, so that grouped heads share the tiles of keys and values.
//
// Tiles of 64 keys are brought to one of three LDS buffers by all wavefronts, two tiles ahead in registers, one in the
// LDS: from the cache unpacked, [key][feature]; from a prompt as they lie, [feature][key].  What lies the wrong way for its product is
// turned by transposing reads.  One barrier per tile.
//
// A wavefront works on 32 keys at a time, three of them at once: the scores of the next, the softmax of this one, the second product
// of the one before.  Matrix and vector instructions of such a step do not depend on each other, so that one wavefront issues
// the latter while the former run.  32 queries a wavefront: with 64 the accumulators and two sets of scores and weights are 400 registers, moved
// and spilled, and the rate is 215 to 690 TFLOP/s.
//
// Measured: 4 sequences of 5400 to 9000 keys, 1024 queries each of 64 heads over 8 of 128 (bf16) 893 us, 1.15 PFLOP/s of the 1.26 of a large
// matrix product; 4 prompts of up to 4096 tokens such 1023 us, 898 TFLOP/s; 2 of 16384 under a window of 1024, 16 heads of 64 (f16) 252 us, 530.  Matrix
// units are busy in 52, 44 and 30 % of the cycles, vector instructions issued in 53, 48 and 65 %; the clock is at 2.1 GHz (1.8 in the first dozen
// launches after a pause, which take up to 18 % longer).  Prompts are further from their floor than chunks: half as many tiles a workgroup, so that first loads and
// last stores weigh more, and heads of 128 in workgroups of 8 spill 74 registers (300 bytes a lane), which chunks do not.
//
// Infinities and NaN among the values of a tile that not all of the workgroup's queries see whole are zeros in the LDS, so that
// they do not reach a query that does not see them as 0 * NaN; if there were any, they are added where they are seen at the end.  In tiles that all
// see whole an infinity becomes NaN where its weight was rounded to zero, or the sum scaled down by zero: sums of prompts that are not finite at the end are
// worked out again (attn_infinite_sums).
constexpr int ATTN_AHEAD = 2;              // an operand is read this many steps of the reduction before its product

template <bool BF, int D, bool CACHE>
struct AttnStage {
    // LDS pitches in bytes.  Cache: an odd number of 16-byte units for the keys (16 lanes read 16 rows), 64 bytes past a
    // multiple of 256 for the values (32 lanes read four rows x 64 bytes).  Prompt: rows of 64 tokens, units exchanged by attn_unit.
    static constexpr int KP = CACHE ? 2 * D + 16 : 128;
    static constexpr int VP = CACHE ? (D == 96 ? 192 : 2 * D + 64) : 128;
    static constexpr int K_BYTES = CACHE ? 64 * KP : D * KP;
    static constexpr int V_BYTES = CACHE ? 64 * VP : D * VP;
    static constexpr int BYTES = K_BYTES + V_BYTES;
};
// 16-byte unit u of a row of 64 tokens lies at unit u ^ attn_unit(row): the rows of 16 lanes' reads, and the 64-byte
// pieces of four neighbouring rows, fall into different banks
__device__ __forceinline__ int attn_unit(int row) { return ((row >> 1 & 1) << 2) | (row >> 2 & 1) << 1 | (row >> 3 & 1); }
// Calls hide(i) for those of N scores, of keys from + key(i), that a query at position p does not see, or that lie below `least`.  Away from the
// sinks one comparison tells: key(i) - (begin - from) as an unsigned number is at most p - begin.
template <int N, class Key, class Hide>
__device__ __forceinline__ void attn_hide(int from, int p, int lo, int least, int sinks, bool near_sinks, Key&& key, Hide&& hide)
{
    if (near_sinks) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (!attn_sees(from + key(i), p, lo, sinks) || from + key(i) < least) hide(i);
        return;
    }
    const int begin = lo > least ? lo : least;
    const bool none = p < begin;
    const int offset = none ? 1 << 30 : begin - from;
    const unsigned span = none ? 0 : p - begin;
#pragma unroll
    for (int i = 0; i < N; ++i)
        if ((unsigned)(key(i) - offset) > span) hide(i);
}

// Sums of features whose values are not finite in the tiles that all of the workgroup's queries see whole: those values' sum in place of what their
// products with weights came to.  A lane takes 8 of a tile's 64 keys in every eighth row; its bit i of a mask is row 8 i + lane / 8.
template <bool BF, int D, class FirstKey, class Partial>
__device__ __forceinline__ void attn_infinite_sums(float16v (&o)[D / 32], const uint16_t* values, int64_t ld, int v_begin, int v_end, FirstKey&& first_key, Partial&& partial)
{
    constexpr unsigned SIZE = 0x7fffu, INF = BF ? 0x7f80u : 0x7c00u;
    const int lane = threadIdx.x & 63;
    unsigned up = 0, down = 0, none = 0;                   // rows with +infinity, -infinity, NaN
    for (int v = v_begin; v < v_end; ++v) {
        const int j = first_key(v);
        if (partial(j)) continue;
        const uint16_t* src = values + (lane >> 3) * ld + j + (lane & 7) * 8;
#pragma unroll 4
        for (int i = 0; i < D / 8; ++i) {
            uint4v x;
            __builtin_memcpy(&x, src + i * 8 * ld, 16);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const unsigned one = x[k / 2] >> 16 * (k % 2) & 0xffffu, size = one & SIZE;
                up |= (one == INF ? 1u : 0u) << i;
                down |= (one == (INF | 0x8000u) ? 1u : 0u) << i;
                none |= (size > INF ? 1u : 0u) << i;
            }
        }
    }
#pragma unroll
    for (int by = 1; by < 8; by *= 2) {
        up |= __shfl_xor(up, by);
        down |= __shfl_xor(down, by);
        none |= __shfl_xor(none, by);
    }
    // this lane's features are 32 t + 8 (e / 4) + 4 (lane / 32) + e % 4
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int from = 8 * (4 * (lane >> 5) + r);
        const unsigned row_up = __shfl(up, from), row_down = __shfl(down, from), row_none = __shfl(none, from);
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
            const int e = 4 * (i % 4) + r;
            if (row_up >> i & 1) o[i / 4][e] = INFINITY;
            if (row_down >> i & 1) o[i / 4][e] = -INFINITY;
            if ((row_none | (row_up & row_down)) >> i & 1) o[i / 4][e] = __builtin_nanf("");
        }
    }
}

// TINY: a prompt of fewer than 64 columns in all.
template <bool BF, int D, bool CACHE, int W, bool TINY = false>
__global__ __launch_bounds__(64 * W, tile_residency(D, CACHE, W)) void attention_tile_kernel(AttnArgs a)
{
    using Stage = AttnStage<BF, D, CACHE>;
    constexpr int S = D / 16, DT = D / 32, KP = Stage::KP, VP = Stage::VP;
    constexpr int SB = scale_bytes(D);
    constexpr int KINDS = W == 8 ? 1 : 2;                  // four wavefronts bring keys and values, of eight each four one of them
    constexpr int UNITS = D / 32;                          // 16-byte units of a tile (cache: words) per thread and kind
    constexpr int PARTS = KINDS * UNITS;
    __shared__ __attribute__((aligned(16))) char smem[3 * Stage::BYTES];
    __shared__ int special;                                // whether values were replaced by zeros

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int half = lane >> 5, c = lane & 31, r = lane & 15;
    const AttnPlace at = attn_place((int)blockIdx.x, a.batch * a.heads, a.heads, a.col_blocks * a.splits);
    const int pair = at.pair, inner = at.inner;      // blocks with most keys first
    const int blk = a.col_blocks - 1 - inner / a.splits, split = inner % a.splits;
    const int b = pair / a.heads, h = pair % a.heads;

    const AttnSeq seq = attn_sequence<CACHE>(a, b);
    const int blocks = (seq.nq + ATTN_TILE_QUERIES - 1) / ATTN_TILE_QUERIES;
    const int64_t items = (int64_t)blocks * a.group, item0 = (int64_t)blk * W;
    if (item0 >= items) return;
    const int64_t item_last = items < item0 + W ? items - 1 : item0 + W - 1;
    const int shift = CACHE ? 0 : (int)(seq.t0 & 7);       // tiles of a prompt begin at multiples of 8 columns
    const int p0 = seq.len - seq.nq;
    const auto position = [&](int64_t query) { return p0 + (int)(query < seq.nq ? query : seq.nq - 1); };
    const int wg_first = position(item0 / a.group * ATTN_TILE_QUERIES);
    const int wg_last = position(item_last / a.group * ATTN_TILE_QUERIES + ATTN_TILE_QUERIES - 1);
    const AttnTiles tiles = attn_tiles(wg_first, wg_last, a.window, a.sinks, shift, ATTN_TILE_KEYS);
    const int v_begin = split * (a.splits > 1 ? a.split_tiles : 0);
    const int v_end = split + 1 == a.splits || tiles.count - v_begin < a.split_tiles ? tiles.count : v_begin + a.split_tiles;   // (as in the other kernel)

    // the wavefront's item; one that is not there repeats the last one, needs no keys, and its result is dropped
    const bool works = item0 + wave <= item_last;
    const int64_t item = works ? item0 + wave : item_last;
    const int head = h * a.group + (int)(item % a.group), q0 = (int)(item / a.group) * ATTN_TILE_QUERIES, query = q0 + c;
    const int p = position(query), lo = attn_window_start(p, a.window);
    const int first = works ? position(q0) : INT32_MAX, last = works ? position(q0 + ATTN_TILE_QUERIES - 1) : -1;
    const int window_first = attn_window_start(first, a.window), window_last = attn_window_start(last, a.window);

    // queries: lane c has column c; features 16 s + 8 half and up
    uint4v q[S];
    {
        const uint16_t* src = a.q + ((int64_t)head * D + 8 * half) * a.ldq + seq.t0 + (query < seq.nq ? query : seq.nq - 1);
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                q[s][i] = src[(int64_t)(16 * s + 2 * i) * a.ldq] | (unsigned)src[(int64_t)(16 * s + 2 * i + 1) * a.ldq] << 16;
    }

    // the first key of tile v
    const int key_sinks = -shift, key_window = (tiles.window - tiles.sinks) * ATTN_TILE_KEYS - shift;
    const auto first_key = [&](int v) __attribute__((always_inline)) { return v * ATTN_TILE_KEYS + (v < tiles.sinks ? key_sinks : key_window); };
    // whether not all of the workgroup's queries see all 64 keys from j on
    const int wg_window = attn_window_start(wg_last, a.window);
    const auto partial = [&](int j) __attribute__((always_inline)) {
        return j < 0 || j + ATTN_TILE_KEYS - 1 > wg_first || (j < wg_window && j + ATTN_TILE_KEYS - 1 >= a.sinks);
    };
    // of 32 keys from j on: whether any of the wavefront's queries sees any, or not all see all
    const auto is_needed = [&](int j) __attribute__((always_inline)) { return j <= last && j + 31 >= 0 && (j + 31 >= window_first || j < a.sinks); };
    const auto is_masked = [&](int j) __attribute__((always_inline)) { return j < 0 || j + 31 > first || (j < window_last && j + 31 >= a.sinks); };

    // ---- staging: memory -> registers -> LDS, a part at a time, to be spread among the products
    const int page = 1 << a.page_shift;
    const int64_t chunk = page_head_bytes(page, D), page_bytes = chunk * a.heads;
    const char* pages = CACHE ? a.cache + h * chunk : nullptr;
    const attn_table table = attn_scalar(CACHE ? a.table + (int64_t)b * a.table_ld : nullptr);
    const int kind0 = W == 8 ? wave >> 2 : 0, brings = wave & 3, member = tid & 255;
    uint4v unit[KINDS][CACHE ? 1 : UNITS];
    unsigned word[KINDS][CACHE ? UNITS : 1], codes[KINDS] = {};
    int page_id = -1;                                      // cache: of the wavefront's keys of the next tile to load
    bool known = false, known_before = false;              // whether there is such a page: of the tile just loaded, of the one before
    const char* from[KINDS];                               // of the next tile to load, the same for all lanes of a wavefront
    const char* scales_from[KINDS];
    int64_t row_step[KINDS];                               // prompt: bytes of 32 rows
    unsigned lane_off[KINDS], scale_off[KINDS];            // a lane's bytes past these
    int lds_off[KINDS];
#pragma unroll
    for (int n = 0; n < KINDS; ++n) {
        const int kind = kind0 + n;
        if constexpr (CACHE) {
            const int row = kind ? ((lane >> 4) & 1) * 8 + ((lane >> 1) & 7) : r, part = kind ? (lane & 1) + 2 * half : lane >> 4;
            lane_off[n] = (D == 64 ? lane * 16 : lane * (D / 8)) + kind * page * (D / 2);
            scale_off[n] = page * D + (kind * page + row) * SB;
            lds_off[n] = kind ? Stage::K_BYTES + (brings * 16 + row) * VP + part * 16 : (brings * 16 + row) * KP + part * 16;
        } else {
            const int64_t ld = kind ? a.ldv : a.ldk;
            const int f = member >> 3;                     // rows f + 32 i have the same attn_unit
            row_step[n] = 64 * ld;
            lane_off[n] = 2 * ((unsigned)f * (unsigned)ld + (member & 7) * 8);
            lds_off[n] = (kind ? Stage::K_BYTES : 0) + f * 128 + ((member & 7) ^ attn_unit(f)) * 16;
        }
    }
    const auto find_page = [&](int j) __attribute__((always_inline)) {
        if constexpr (CACHE) {
            const int idx = (j + brings * 16) >> a.page_shift;
            page_id = table[idx < a.table_width ? idx : a.table_width - 1];   // (keys past the last page are hidden)
        }
    };
    // The last columns of a prompt end a tile, not begin one: what would lie past them is taken from before, where the tile before has it
    // already (and these are hidden).  Keys of the tile whose first key would be j begin at:
    const int prompt_last = CACHE || TINY ? INT32_MAX : (int)(a.tokens - ATTN_TILE_KEYS - seq.t0);
    const auto begins = [&](int j) __attribute__((always_inline)) { return j < prompt_last ? j : prompt_last; };
    // the tile whose keys are j and up; next: those of the tile after it
    const auto load_begin = [&](int j, int next) __attribute__((always_inline)) {
        if constexpr (CACHE) {
            const int at = (j + brings * 16) & (page - 1);     // a wavefront brings 16 keys (and their values)
            known = (unsigned)page_id < (unsigned)a.pages;
            const char* base = pages + (known ? page_id : 0) * page_bytes;
#pragma unroll
            for (int n = 0; n < KINDS; ++n) {
                from[n] = base + code_offset(D, at, 0);
                scales_from[n] = base + at * SB;
            }
            find_page(next);
        } else {
            const int64_t tile = seq.t0 + j;
#pragma unroll
            for (int n = 0; n < KINDS; ++n) from[n] = reinterpret_cast<const char*>((kind0 + n ? a.v : a.k) + (int64_t)h * D * (kind0 + n ? a.ldv : a.ldk) + tile);
        }
    };
    const auto load_part = [&](int i) __attribute__((always_inline)) {
        if constexpr (CACHE) {
            if (i >= KINDS) return;
            const unsigned* src = reinterpret_cast<const unsigned*>(from[i] + lane_off[i]);
#pragma unroll
            for (int s = 0; s < UNITS; ++s) word[i][s] = src[s];
            const char* sc = scales_from[i] + scale_off[i];
            codes[i] = SB == 2 ? *reinterpret_cast<const uint16_t*>(sc) : *reinterpret_cast<const unsigned*>(sc);
        } else {
            const int n = i / UNITS, u = i % UNITS;
            if constexpr (TINY) {
                // 16 bytes, whatever they hold past the last column (a NaN in there only costs time); what would end past the last
                // row's last column is loaded further down and moved
                const char* at = from[n] + u * row_step[n] + lane_off[n];
                const char* last = reinterpret_cast<const char*>(kind0 + n ? a.v : a.k) + row_step[n] / 32 * ((int64_t)a.heads * D - 1) + 2 * (a.tokens - 8);
                const int over = at > last ? (int)(at - last) : 0;
                unsigned __int128 x;
                __builtin_memcpy(&x, at - over, 16);
                if (over) x = over < 16 ? x >> 8 * over : 0;
                __builtin_memcpy(&unit[n][u], &x, 16);
            } else {
                __builtin_memcpy(&unit[n][u], from[n] + u * row_step[n] + lane_off[n], 16);
            }
        }
    };
    const auto store_begin = [&](bool clean) __attribute__((always_inline)) {
        if constexpr (CACHE)
            if (!known_before)                             // a page that is not there reads as NaN
#pragma unroll
                for (int n = 0; n < KINDS; ++n) codes[n] = 0xffffffffu;
        if (!clean || kind0 + KINDS == 1) return;
        constexpr int n = KINDS - 1;
        bool found = false;
        if constexpr (CACHE) {
#pragma unroll
            for (int s = 0; s < UNITS; ++s)
                if ((codes[n] >> 8 * s & 255) > most_scale(BF)) {
                    found = true;
                    codes[n] &= ~(255u << 8 * s);
                    word[n][s] = 0;
                }
        } else {
            constexpr unsigned EXP = BF ? 0x7f80u : 0x7c00u;
#pragma unroll
            for (int i = 0; i < UNITS; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const unsigned x = unit[n][i][k];
                    const bool lo_bad = (x & EXP) == EXP, hi_bad = (x >> 16 & EXP) == EXP;
                    found |= lo_bad | hi_bad;
                    unit[n][i][k] = x & (lo_bad ? 0xffff0000u : ~0u) & (hi_bad ? 0xffffu : ~0u);
                }
        }
        if (found) special = 1;
    };
    const auto store_part = [&](int i, int buffer) __attribute__((always_inline)) {
        const int n = i / UNITS, u = i % UNITS;
        char* dst = smem + buffer + lds_off[n];
        if constexpr (CACHE) *reinterpret_cast<uint4v*>(dst + u * 64) = attn_unpack<BF>(word[n][u], codes[n] >> 8 * u & 255);
        else *reinterpret_cast<uint4v*>(dst + u * 4096) = unit[n][u];
    };

    // ---- products
    const attn_lds lds = (attn_lds)smem;
    int k_at[2], v_at[4];
    if constexpr (CACHE) {
        k_at[0] = c * KP + half * 16;
        v_at[0] = Stage::K_BYTES + (4 * half + (r >> 2)) * VP + (16 * (lane >> 4 & 1) + (r & 3) * 4) * 2;
    } else {
        // rows 8 x + 4 half + i of the scores' tile are to be keys 16 .. + 8 half + 4 x + i: the two middle groups of
        // four of every 16 change places
        const int f = 8 * half + (r >> 2), at = 16 * (lane >> 4 & 1) + ((r & 1) << 1 | (r >> 1 & 1)) * 4;   // the first of four keys
        k_at[0] = f * 128 + ((at >> 3) ^ attn_unit(f)) * 16 + (at & 4) * 2;
        k_at[1] = (f + 4) * 128 + ((at >> 3) ^ attn_unit(f + 4)) * 16 + (at & 4) * 2;
#pragma unroll
        for (int g = 0; g < 4; ++g) v_at[g] = Stage::K_BYTES + c * 128 + ((2 * g + half) ^ attn_unit(c)) * 16;
    }
    // the first operand of the scores of keys 32 sub and up, at step s; buf: the tile's buffer, in bytes
    const auto key_operand = [&](int buf, int sub, int s) __attribute__((always_inline)) {
        if constexpr (CACHE) {
            return *(const __attribute__((address_space(3))) uint4v*)(lds + buf + k_at[0] + sub * 32 * KP + s * 32);
        } else {
            const uint2 one = attn_transposed(lds + buf + (k_at[0] ^ sub * 64) + s * 2048);
            const uint2 two = attn_transposed(lds + buf + (k_at[1] ^ sub * 64) + s * 2048);
            return uint4v{one.x, one.y, two.x, two.y};
        }
    };
    // that of the second product: features 32 t and up, keys 16 g and up
    const auto value_operand = [&](int buf, int g, int t) __attribute__((always_inline)) {
        if constexpr (CACHE) {
            const uint2 one = attn_transposed(lds + buf + v_at[0] + g * 16 * VP + t * 64), two = attn_transposed(lds + buf + v_at[0] + (g * 16 + 8) * VP + t * 64);
            return uint4v{one.x, one.y, two.x, two.y};
        } else {
            return *(const __attribute__((address_space(3))) uint4v*)(lds + buf + v_at[g] + t * 4096);
        }
    };

    float16v o[DT] = {}, sc[2] = {};                       // two sets of scores, each of 32 keys ..
    uint4v w[2][2] = {};                                   // .. and of weights
    float m = -FLT_MAX, l = 0;

    // half SUB of a tile, keys j and up, whose scores are in sc[SUB]: its weights; beside it the other half's scores (of the
    // next tile, where SUB is 1), the product of the weights before, and a part of the staging.  part: the tile is a partial one; keys
    // below `hide` are another tile's.
    const auto step = [&](auto which, int j, int hide, bool part, int next_buf, int last_buf, int stage_buf, int j_before, int j_after) __attribute__((always_inline)) {
        constexpr int SUB = decltype(which)::value;
        const auto stage = [&](int i) __attribute__((always_inline)) {
            if constexpr (SUB == 0) store_part(i, stage_buf);
            else load_part(i);
        };
        if (part) {
            // nothing to compute where neither these keys nor their neighbours in order are needed
            if (!(is_needed(j) || is_needed(j_before) || is_needed(j_after))) {
#pragma unroll
                for (int i = 0; i < PARTS; ++i) stage(i);
                w[SUB][0] = w[SUB][1] = uint4v{};
                return;
            }
            if (is_masked(j) || (!CACHE && j < hide))
                attn_hide<16>(
                    j + (CACHE ? 4 : 8) * half, p, lo, CACHE ? 0 : hide, a.sinks, j < a.sinks,
                    [](int i) __attribute__((always_inline)) { return CACHE ? 8 * (i >> 2) + (i & 3) : 16 * (i >> 3) + (i & 7); },
                    [&](int i) __attribute__((always_inline)) { sc[SUB][i] = -INFINITY; });
        }
        // Pieces of all that, in an order that keeps both units busy: per step of the reduction an operand of each product is
        // read ATTN_AHEAD steps before its use, two products are issued, and a share of the vector work follows: the maximum, whether
        // to follow it, and the weights two at a time
        float16v& x = sc[SUB];
        float top = 0, shrink = 1;
        bool grown = false;
        const auto piece = [&](int u) __attribute__((always_inline)) {
            if (u == 0) {
                top = attn_max3(x[0], x[1], x[2]);
#pragma unroll
                for (int i = 3; i < 15; i += 2) top = attn_max3(top, x[i], x[i + 1]);
                top = attn_max3(top, x[15], x[15]);
            } else if (u == 1) {
                const float2v both = attn_pair32(top);
                top = attn_max3(both[0], both[1], both[1]) * a.scale;
                grown = top > m + (ATTN_SLACK + ATTN_LIFT<BF>);
                const float now = grown ? top - ATTN_LIFT<BF> : m;
                shrink = attn_exp2(m - now);
                m = now;
                l *= shrink;
            } else {
                const int i = 2 * (u - 2);
                const float y = attn_exp2(__builtin_fmaf(x[i], a.scale, -m)), z = attn_exp2(__builtin_fmaf(x[i + 1], a.scale, -m));
                l += y + z;
                w[SUB][i >> 3][(i & 7) >> 1] = attn_pack<BF>(y, z);
            }
        };
        uint4v ks[S], xs[S];
        const auto fetch = [&](int s) __attribute__((always_inline)) {
            ks[s] = key_operand(next_buf, 1 - SUB, s);
            xs[s] = value_operand(last_buf, 2 * (1 - SUB) + s / DT, s % DT);
        };
        sc[1 - SUB] = float16v{};
#pragma unroll
        for (int s = 0; s < ATTN_AHEAD; ++s) fetch(s);
#pragma unroll
        for (int s = 0; s < S; ++s) {
            if (s + ATTN_AHEAD < S) fetch(s + ATTN_AHEAD);
            sc[1 - SUB] = attn_mma32<BF>(ks[s], q[s], sc[1 - SUB]);
            o[s % DT] = attn_mma32<BF>(xs[s], w[1 - SUB][s / DT], o[s % DT]);
#pragma unroll
            for (int i = s * PARTS / S; i < (s + 1) * PARTS / S; ++i) stage(i);
#pragma unroll
            for (int u = s * 10 / S; u < (s + 1) * 10 / S; ++u) piece(u);
            __builtin_amdgcn_sched_barrier(0);
        }
        // the weights are worked out before the branch, among the products
        asm volatile("" : "+v"(w[SUB][0]), "+v"(w[SUB][1]), "+v"(l));
        if (__any(grown))
#pragma unroll
            for (int t = 0; t < DT; ++t) o[t] *= shrink;
    };

    // the first step's product is one of zeros, with the third buffer's values
    for (int e = tid * 16; e < Stage::V_BYTES; e += 64 * W * 16)
        *reinterpret_cast<uint4v*>(smem + 2 * Stage::BYTES + Stage::K_BYTES + e) = uint4v{};
    if (tid == 0) special = 0;
    // past the last tile that one is brought again, to a buffer that is not read any more
    const auto clamped = [&](int v) __attribute__((always_inline)) { return first_key(v < v_end ? v : v_end - 1); };
    int own = clamped(v_begin), own_next = clamped(v_begin + 1);       // the tiles' own keys ..
    int j = begins(own), j_next = begins(own_next);                    // .. and what is brought
    if (v_begin < v_end) {
        find_page(j);
        load_begin(j, j_next);
#pragma unroll
        for (int i = 0; i < PARTS; ++i) load_part(i);
        known_before = known;
    }
    __syncthreads();
    if (v_begin < v_end) {
        store_begin(partial(j));
#pragma unroll
        for (int i = 0; i < PARTS; ++i) store_part(i, 0);
        load_begin(j_next, begins(clamped(v_begin + 2)));
#pragma unroll
        for (int i = 0; i < PARTS; ++i) load_part(i);
        known_before = known;
    }
    __syncthreads();
    if (v_begin < v_end)
#pragma unroll
        for (int s = 0; s < S; ++s) sc[0] = attn_mma32<BF>(key_operand(0, 0, s), q[s], sc[0]);
    int buf = 0, before = 2 * Stage::BYTES, j_before = INT32_MAX;
    bool part = partial(j) || j != own;
    for (int v = v_begin; v < v_end; ++v) {
        const int after = buf == 2 * Stage::BYTES ? 0 : buf + Stage::BYTES;
        const bool part_next = partial(j_next) || j_next != own_next;
        store_begin(part_next);
        step(std::integral_constant<int, 0>{}, j, own, part, buf, before, after, j_before, j + 32);
        __syncthreads();
        const int own_then = clamped(v + 2), j_then = begins(own_then);
        load_begin(j_then, clamped(v + 3));
        step(std::integral_constant<int, 1>{}, j + 32, own, part, after, buf, 0, j, j_next);
        known_before = known;
        j_before = j + 32;
        j = j_next;
        j_next = j_then;
        own = own_next;
        own_next = own_then;
        part = part_next;
        before = buf;
        buf = after;
    }
    if (v_begin < v_end)
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int t = 0; t < DT; ++t) o[t] = attn_mma32<BF>(value_operand(before, 2 + g, t), w[1][g], o[t]);

    if constexpr (!CACHE && !TINY) {
        float most = 0;                                    // infinity or NaN where a sum is not finite
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int e = 0; e < 16; e += 2)
                most = __builtin_elementwise_maximum(__builtin_elementwise_maximum(__builtin_fabsf(o[t][e]), __builtin_fabsf(o[t][e + 1])), most);
        if (__any(!(most < INFINITY) && l < INFINITY)) attn_infinite_sums<BF, D>(o, a.v + (int64_t)h * D * a.ldv + seq.t0, a.ldv, v_begin, v_end, first_key, partial);
    }
    if (special)
        for (int v = v_begin; v < v_end; ++v) {
            const int from_key = first_key(v);
            if (!partial(from_key)) continue;
            for (int k = from_key; k < from_key + ATTN_TILE_KEYS; ++k) {
                if (!attn_sees(k, p, lo, a.sinks)) continue;
                if constexpr (CACHE) {
                    const int id = a.table[(int64_t)b * a.table_ld + (k >> a.page_shift)];
                    const bool there = (unsigned)id < (unsigned)a.pages;
                    const char* sc8 = pages + (there ? id : 0) * page_bytes + (int64_t)page * D + (int64_t)(page + (k & (page - 1))) * SB;
#pragma unroll
                    for (int t = 0; t < DT; ++t)
                        if (!there || (unsigned char)sc8[t] > most_scale(BF)) o[t] += __builtin_nanf("");
                } else {
#pragma unroll
                    for (int t = 0; t < DT; ++t)
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const int d = 32 * t + 8 * (e >> 2) + 4 * half + (e & 3);
                            const float f = attn_widen<BF>(a.v[((int64_t)h * D + d) * a.ldv + seq.t0 + k]);
                            if (!(__builtin_fabsf(f) < INFINITY)) o[t][e] += f;
                        }
                }
            }
        }

    const float2v both = attn_pair32(l);
    l = both[0] + both[1];
    if (!works || query >= seq.nq) return;
    if (seq.bad) l = __builtin_nanf("");
    const int64_t token = seq.t0 + query;
    if (a.splits == 1) {
        const float f = p < 0 ? 0 : 1 / l;
        uint16_t* dst = a.out + ((int64_t)head * D + 4 * half) * a.ldo + token;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) dst[(int64_t)(32 * t + 8 * (i >> 2) + (i & 3)) * a.ldo] = attn_narrow<BF>(o[t][i] * f);
    } else {
        const int64_t at = ((int64_t)split * a.heads * a.group + head) * a.tokens + token;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                *reinterpret_cast<float4v*>(a.part_o + at * D + 32 * t + 8 * (i >> 2) + 4 * half) = float4v{o[t][i], o[t][i + 1], o[t][i + 2], o[t][i + 3]};
        if (half == 0) {
            a.part_ml[2 * at] = p < 0 ? -INFINITY : m;
            a.part_ml[2 * at + 1] = l;
        }
    }
}

// ---- join of the parts
//
// A wavefront takes one token of one query head, its lanes two features each, and reads the parts' sums along the features, all of
// them at once; a workgroup's results leave along the tokens.  Where there are few rows, the parts of a row are shared by the
// workgroup's four wavefronts instead.  Bound by latency where it matters: 128 rows of 32 parts 4.2 us.
template <bool BF, int D, bool FEW>
__global__ __launch_bounds__(FEW ? 256 : 1024) void attention_join_kernel(AttnArgs a)
{
    constexpr int TOKENS = FEW ? 1 : 16;
    __shared__ float tile[FEW ? 4 : TOKENS][D + 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t token0 = (int64_t)blockIdx.x * TOKENS;
    const int head = blockIdx.y;
    const int64_t stride = (int64_t)a.heads * a.group * a.tokens;
    const bool has = 2 * lane < D;
    const int c = FEW ? 0 : wave;
    if (token0 + c < a.tokens) {
        const int64_t at = (int64_t)head * a.tokens + token0 + c;
        float top = -FLT_MAX, total = 0;
        for (int i = 0; i < a.splits; i += 64) {
            const int part = i + lane;
            const float m = part < a.splits ? a.part_ml[2 * (at + part * stride)] : -FLT_MAX;
            top = fmaxf(top, m);
        }
#pragma unroll
        for (int by = 1; by < 64; by *= 2) top = fmaxf(top, __shfl_xor(top, by));
        float2v x = {0, 0};
        const bool none = a.part_ml[2 * at] == -INFINITY;
#pragma unroll 8
        for (int i = FEW ? wave : 0; i < a.splits; i += FEW ? 4 : 1) {
            const float f = attn_exp2(a.part_ml[2 * (at + i * stride)] - top);
            const float2v y = has ? *reinterpret_cast<const float2v*>(a.part_o + (at + i * stride) * D + 2 * lane) : float2v{0, 0};
            total += a.part_ml[2 * (at + i * stride) + 1] * f;
            x[0] += y[0] * f;
            x[1] += y[1] * f;
        }
        if constexpr (FEW) {
            if (has) {
                tile[wave][2 * lane] = x[0];
                tile[wave][2 * lane + 1] = x[1];
            }
            if (lane == 0) tile[wave][D] = total;
            __syncthreads();
            if (threadIdx.x < D) {
                const int d = threadIdx.x;
                const float y = (tile[0][d] + tile[1][d]) + (tile[2][d] + tile[3][d]), sum = (tile[0][D] + tile[1][D]) + (tile[2][D] + tile[3][D]);
                a.out[((int64_t)head * D + d) * a.ldo + token0] = attn_narrow<BF>(none ? 0 : y / sum);
            }
        } else if (has) {
            tile[c][2 * lane] = none ? 0 : x[0] / total;
            tile[c][2 * lane + 1] = none ? 0 : x[1] / total;
        }
    }
    if constexpr (!FEW) {
        __syncthreads();
#pragma unroll
        for (int e = threadIdx.x; e < TOKENS * D; e += 1024) {
            const int c = e & 15, d = e >> 4;
            if (token0 + c < a.tokens) a.out[((int64_t)head * D + d) * a.ldo + token0 + c] = attn_narrow<BF>(tile[c][d]);
        }
    }
}

}  // namespace shflbw
