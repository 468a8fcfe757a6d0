// Norms of queries and keys per head and the rotation by position, in one pass over both.
//
//     y = x / sqrt(mean(x^2) + eps) * weight;   (a, b) -> (a cos t - b sin t, a sin t + b cos t),  t = position * frequency
//
// A lane has one token's pairs of a head, or a part of them where tokens are few, and neighbouring lanes neighbouring tokens, so that
// the norm is a lane's own sum (of a few lanes) and loads are contiguous along the tokens.  All heads of a token turn by the
// same angles: a workgroup works them out once, into the LDS, and takes several heads.  The angle is a product in 64 bits, taken to
// one turn there (a position of 2^20 in 32 bits leaves 0.03 radians), its sine and cosine in 32.
//
// Everything between the loads and the one rounding at the store is in 32 bits.  Squares of bfloat16 may be more than 32 bits hold, or, with an
// eps that is as small, less: such columns' sums are done again in 64, and the factor is applied in two steps.
#include <hip/hip_runtime.h>

#include <cstdint>

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
// the features of pair n: those past 2 * pairs are pairs of neighbours that are not turned
struct RotPair {
    int a, b;
};
__device__ __forceinline__ RotPair rot_features(int n, int pairs, int interleaved)
{
    if (interleaved || n >= pairs) return RotPair{2 * n, 2 * n + 1};
    return RotPair{n, n + pairs};
}
// cosine and sine of pair n at a token's position
__device__ __forceinline__ float2 rot_angle(const RotateArgs& a, int n, int64_t token)
{
    const int row = a.axes ? a.axes[n] : 0;
    if ((unsigned)row >= (unsigned)a.position_rows) return float2{__builtin_nanf(""), __builtin_nanf("")};
    const double half_turns = (double)a.positions[row * a.ldp + token] * a.frequencies[n] * 0.31830988618379067154;
    float2 r;
    sincospif((float)(half_turns - 2 * __builtin_rint(half_turns * 0.5)), &r.y, &r.x);
    return r;
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

// T tokens and 64 / T parts of a head's pairs to a wavefront
template <bool BF, int D, int T>
__global__ __launch_bounds__(256) void norm_rotate_kernel(RotateArgs a)
{
    constexpr int F = 64 / T, P = D / 2 / F;
    __shared__ float2 angle[D / 2][T], weight[2][D / 2];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, t = lane % T, part = lane / T;
    const int64_t token0 = (int64_t)blockIdx.x * T, token = token0 + t < a.tokens ? token0 + t : a.tokens - 1;
    for (int e = threadIdx.x; e < a.pairs * T; e += 256) {
        const int64_t at = token0 + e % T;
        angle[e / T][e % T] = rot_angle(a, e / T, at < a.tokens ? at : a.tokens - 1);
    }
    if (threadIdx.x < D) {
        const int kind = threadIdx.x / (D / 2), n = threadIdx.x % (D / 2);
        const RotPair f = rot_features(n, a.pairs, a.interleaved);
        weight[kind][n] = a.weight[kind] ? float2{rot_widen<BF>(a.weight[kind][f.a]), rot_widen<BF>(a.weight[kind][f.b])} : float2{1, 1};
    }
    __syncthreads();
    for (int h = blockIdx.y * 4 + wave; h < a.all_heads; h += gridDim.y * 4) {
        const int kind = h >= a.q_heads, head = kind ? h - a.q_heads : h;
        const uint16_t* src = a.in[kind] + (int64_t)head * D * a.ld_in[kind] + token;
        uint16_t* dst = a.out[kind] + (int64_t)head * D * a.ld_out[kind] + token;
        unsigned x[P];
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const RotPair f = rot_features(part * P + i, a.pairs, a.interleaved);
            x[i] = src[f.a * a.ld_in[kind]] | (unsigned)src[f.b * a.ld_in[kind]] << 16;
        }
        RotFactor by = {1, 1};
        if (a.norm) {
            float sum = 0;
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const float u = rot_widen<BF>(x[i] & 0xffffu), v = rot_widen<BF>(x[i] >> 16);
                sum += u * u + v * v;
            }
#pragma unroll
            for (int step = T; step < 64; step *= 2) sum += __shfl_xor(sum, step);
            // (the lanes of a token have the same sum and go the same way)
            if (sum > 0x1p-60f && sum < 0x1p120f) {
                by.second = (float)(1 / __builtin_sqrt((double)sum / D + a.eps));
            } else {
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
                const float2 c = angle[n][t];
                const float turned = u * c.x - v * c.y;
                v = u * c.y + v * c.x;
                u = turned;
            }
            if (token0 + t < a.tokens) {
                dst[f.a * a.ld_out[kind]] = rot_narrow<BF>(u);
                dst[f.b * a.ld_out[kind]] = rot_narrow<BF>(v);
            }
        }
    }
}

template <bool BF, int D>
int launch(const RotateArgs& a, hipStream_t stream)
{
    const int T = a.tokens <= 4 ? 4 : a.tokens <= 16 ? 16 : 64;
    const int64_t blocks = (a.tokens + T - 1) / T;
    if (blocks > 0x7fffffffLL) return fail(SHFLBW_ERR_BAD_SHAPE, "grid too large");
    // heads to a workgroup: as many as leave 1024 workgroups
    const int64_t most = (a.all_heads + 3) / 4, wanted = (1024 + blocks - 1) / blocks;
    const dim3 grid((unsigned)blocks, (unsigned)(wanted < most ? wanted : most));
    if (T == 4) hipLaunchKernelGGL((norm_rotate_kernel<BF, D, 4>), grid, dim3(256), 0, stream, a);
    else if (T == 16) hipLaunchKernelGGL((norm_rotate_kernel<BF, D, 16>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((norm_rotate_kernel<BF, D, 64>), grid, dim3(256), 0, stream, a);
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
    typedef int (*launcher)(const RotateArgs&, hipStream_t);
    static const launcher table[2][3] = {{&launch<false, 64>, &launch<false, 96>, &launch<false, 128>},
                                         {&launch<true, 64>, &launch<true, 96>, &launch<true, 128>}};
    return table[r->dtype == SHFLBW_BF16][D / 32 - 2](a, static_cast<hipStream_t>(stream));
}
