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
// product (relative 2^-12 or 2^-9 of each, beside the same rounding of the result).  Keys read from the cache are
// exact in 16 bits but for binary16 blocks below 2^-21, whose values are rounded to multiples of 2^-24.
//
// A query whose mask leaves nothing gets zeros.  Infinities and NaN in keys or values that a query does not see leave
// it alone; those it sees reach its result.
#pragma once
#include <hip/hip_runtime.h>

#include <cfloat>
#include <cstdint>

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
        t0 = a.starts[b];
        t1 = a.starts[b + 1];
    }
    t0 = t0 < 0 ? 0 : t0;
    t1 = t1 > a.tokens ? a.tokens : t1;
    s.t0 = t0;
    s.nq = t1 > t0 ? (int)(t1 - t0) : 0;
    s.bad = false;
    if constexpr (CACHE) {
        const int64_t most = (int64_t)a.table_width << a.page_shift;
        const int len = a.lengths[b];
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

// ---- few queries over the cache
//
// A workgroup takes one sequence, key head and part of the keys, and up to 16 NT columns: a column is one query head
// of the key head's group, of one query.  Its wavefronts take tiles of 32 keys in turn, each with its own maximum, sum
// and accumulators, and join through the LDS at the end.  Bound by the cache's bytes: a value is read once, as four bits.
// The keys' words unpack in the registers of the lane that hands them to the matrix instruction; the
// values' words belong to one key each (they share its scale) where the second product wants eight keys of one
// feature per lane, so they go through a tile of LDS that only this wavefront uses and come back by transposing reads.
// Loads are one tile ahead, page numbers two.
template <bool BF, int D, int NT, int W>
__global__ __launch_bounds__(64 * W) void attention_decode_kernel(AttnArgs a)
{
    constexpr int S = D / 32, DT = D / 16;
    constexpr int VP = 2 * D + 32;                        // LDS pitch of a key's values: 8 rows x 32 bytes in 64 banks
    constexpr int OP = D + 4;                             // pitch of a column's sums, in floats
    constexpr int SB = scale_bytes(D);
    constexpr int V_BYTES = W * 32 * VP, O_BYTES = W * 16 * OP * 4, Q_BYTES = NT * 16 * D * 2;
    constexpr int BYTES = V_BYTES > O_BYTES ? (V_BYTES > Q_BYTES ? V_BYTES : Q_BYTES) : (O_BYTES > Q_BYTES ? O_BYTES : Q_BYTES);
    __shared__ __attribute__((aligned(16))) char smem[BYTES];
    __shared__ float stat[W][16 * NT][2];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int quarter = lane >> 4, r = lane & 15;
    const int split = blockIdx.x % a.splits, rest = blockIdx.x / a.splits;
    const int cb = rest % a.col_blocks, pair = rest / a.col_blocks;
    const int b = pair / a.heads, h = pair % a.heads;

    const AttnSeq seq = attn_sequence<true>(a, b);
    const int col0 = cb * 16 * NT, cols = seq.nq * a.group;
    if (col0 >= cols) return;
    const int last_col = (cols < col0 + 16 * NT ? cols : col0 + 16 * NT) - 1;
    const int p0 = seq.len - seq.nq;
    const int p_first = p0 + col0 / a.group, p_last = p0 + last_col / a.group;
    const AttnTiles tiles = attn_tiles(p_first, p_last, a.window, a.sinks, 0, ATTN_DECODE_KEYS);
    const int v_begin = split * a.split_tiles;
    const int v_end = tiles.count - v_begin < a.split_tiles ? tiles.count : v_begin + a.split_tiles;

    const int page = 1 << a.page_shift;
    const int64_t chunk = page_head_bytes(page, D);
    const int32_t* table = a.table + (int64_t)b * a.table_ld;

    struct Raw {
        unsigned k[2][S], v[2][S], ks[2], vs[2];
    };
    // page of tile v; tiles past the end read what the last one does
    auto page_of = [&](int v) __attribute__((always_inline)) {
        const int c = v < v_end ? v : v_end - 1;
        return table[tiles.real(c) * ATTN_DECODE_KEYS >> a.page_shift];
    };
    auto load = [&](int v, int id) __attribute__((always_inline)) {
        Raw x;
        const bool known = (unsigned)id < (unsigned)a.pages;
        const int at = tiles.real(v) * ATTN_DECODE_KEYS & (page - 1);
        const char* base = a.cache + ((int64_t)(known ? id : 0) * a.heads + h) * chunk;
        const char* codes = base + code_offset(D, at, lane);
#pragma unroll
        for (int kind = 0; kind < 2; ++kind, codes += page * D / 2) {
            unsigned(&w)[2][S] = kind ? x.v : x.k;
            if constexpr (D == 64) {
                const uint4v t = *reinterpret_cast<const uint4v*>(codes);
                w[0][0] = t[0]; w[0][1] = t[1]; w[1][0] = t[2]; w[1][1] = t[3];
            } else {
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int s = 0; s < S; ++s) w[u][s] = reinterpret_cast<const unsigned*>(codes + u * D * 8)[s];
            }
        }
        const char* scales = base + (int64_t)page * D;
        const int vr = ((lane >> 4) & 1) * 8 + ((lane >> 1) & 7);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const char* ks = scales + (at + 16 * u + r) * SB;
            const char* vs = scales + (page + at + 16 * u + vr) * SB;
            x.ks[u] = SB == 2 ? *reinterpret_cast<const uint16_t*>(ks) : *reinterpret_cast<const unsigned*>(ks);
            x.vs[u] = SB == 2 ? *reinterpret_cast<const uint16_t*>(vs) : *reinterpret_cast<const unsigned*>(vs);
            if (!known) x.ks[u] = x.vs[u] = 0xffffffffu;   // a page that is not there reads as NaN
        }
        return x;
    };

    int v = v_begin + wave;
    Raw raw = {};
    int id = 0;
    if (v < v_end) {
        raw = load(v, page_of(v));
        id = page_of(v + W);
    }

    // queries: through the LDS once, columns x features, then as operands in registers
    uint4v q[NT][S];
    {
        uint16_t* qs = reinterpret_cast<uint16_t*>(smem);
        for (int e = threadIdx.x; e < NT * 16 * D; e += 64 * W) {
            const int c = e % (16 * NT), f = e / (16 * NT);
            const int col = col0 + c;
            uint16_t x = 0;
            if (col < cols) x = a.q[((int64_t)(h * a.group + col % a.group) * D + f) * a.ldq + seq.t0 + col / a.group];
            qs[c * D + f] = x;
        }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int s = 0; s < S; ++s) q[n][s] = *reinterpret_cast<const uint4v*>(qs + (16 * n + r) * D + 32 * s + 8 * quarter);
        __syncthreads();
    }
    int p[NT], lo[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int col = col0 + 16 * n + r;
        p[n] = col < cols ? p0 + col / a.group : -1;
        lo[n] = attn_window_start(p[n], a.window);
    }

    float4v o[NT][DT] = {};
    float m[NT], l[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) { m[n] = -FLT_MAX; l[n] = 0; }

    char* vt = smem + wave * 32 * VP;
    const int vw = (((lane >> 4) & 1) * 8 + ((lane >> 1) & 7)) * VP + ((lane & 1) + 2 * (lane >> 5)) * 16;
    const attn_lds vr = (attn_lds)vt + (4 * quarter + (r >> 2)) * VP + (r & 3) * 8;

    for (; v < v_end; v += W) {
        Raw next = raw;
        if (v + W < v_end) {
            next = load(v + W, id);
            id = page_of(v + 2 * W);
        }
        const int j0 = tiles.real(v) * ATTN_DECODE_KEYS;
        const bool masked = j0 + 31 > p_first || (j0 < attn_window_start(p_last, a.window) && j0 + 31 >= a.sinks);

        // values of keys that only some columns see must not reach the others as 0 * NaN: such blocks become zeros
        // here, and NaN where they are seen
        if (masked) {
            unsigned special[2] = {0, 0};
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int s = 0; s < S; ++s)
                    if ((raw.vs[u] >> 8 * s & 255) == 255) {
                        special[u] |= 1u << s;
                        raw.vs[u] &= ~(255u << 8 * s);
                        raw.v[u][s] = 0;
                    }
            if (__any(special[0] | special[1])) {
                for (int u = 0; u < 2; ++u)
                    for (int i = 0; i < 16; ++i) {
                        const int from = (i >> 3) * 16 + (i & 7) * 2;   // the first lane that holds this key
                        const unsigned which = __builtin_amdgcn_readlane(u ? special[1] : special[0], from);
                        if (!which) continue;
#pragma unroll
                        for (int n = 0; n < NT; ++n)
                            if (attn_sees(j0 + 16 * u + i, p[n], lo[n], a.sinks))
#pragma unroll
                                for (int t = 0; t < DT; ++t)
                                    if (which >> (t / 2) & 1) o[n][t] += __builtin_nanf("");
                    }
            }
        }

#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int s = 0; s < S; ++s)
                *reinterpret_cast<uint4v*>(vt + vw + 16 * u * VP + s * 64) = attn_unpack<BF>(raw.v[u][s], raw.vs[u] >> 8 * s & 255);

        float4v sc[NT][2] = {};
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int s = 0; s < S; ++s) {
                const uint4v k = attn_unpack<BF>(raw.k[u][s], raw.ks[u] >> 8 * s & 255);
#pragma unroll
                for (int n = 0; n < NT; ++n) sc[n][u] = attn_mma16<BF>(k, q[n][s], sc[n][u]);
            }

        uint4v w[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float x[8], top = -INFINITY;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[i] = sc[n][i >> 2][i & 3] * a.scale;
                if (masked && !attn_sees(j0 + (i >> 2) * 16 + quarter * 4 + (i & 3), p[n], lo[n], a.sinks)) x[i] = -INFINITY;
                top = fmaxf(top, x[i]);
            }
            float2v t = attn_pair16(top);
            t = attn_pair32(fmaxf(t[0], t[1]));
            top = fmaxf(t[0], t[1]);
            if (__any(top > m[n])) {
                const float now = fmaxf(m[n], top), shrink = attn_exp2(m[n] - now);
                m[n] = now;
                l[n] *= shrink;
#pragma unroll
                for (int t2 = 0; t2 < DT; ++t2) o[n][t2] *= shrink;
            }
            float sum = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[i] = attn_exp2(x[i] - m[n]);
                sum += x[i];
            }
            l[n] += sum;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[n][i] = attn_pack<BF>(x[2 * i], x[2 * i + 1]);
        }

        asm volatile("" ::: "memory");
#pragma unroll
        for (int t = 0; t < DT; ++t) {
            const uint2 first = attn_transposed(vr + t * 32), second = attn_transposed(vr + 16 * VP + t * 32);
            const uint4v x = {first.x, first.y, second.x, second.y};
#pragma unroll
            for (int n = 0; n < NT; ++n) o[n][t] = attn_mma16<BF>(x, w[n], o[n][t]);
        }
        asm volatile("" ::: "memory");
        raw = next;
    }

    // join the wavefronts
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
        float top = -FLT_MAX;
#pragma unroll
        for (int i = 0; i < W; ++i) top = fmaxf(top, stat[i][16 * n + r][0]);
        const float f = attn_exp2(m[n] - top);
#pragma unroll
        for (int t = 0; t < DT; ++t) *reinterpret_cast<float4v*>(sums + (wave * 16 + r) * OP + 16 * t + 4 * quarter) = o[n][t] * f;
        __syncthreads();
        for (int e = threadIdx.x; e < 16 * D; e += 64 * W) {
            const int c = e / D, d = e % D, col = col0 + 16 * n + c;
            if (col >= cols) continue;
            float most = -FLT_MAX, total = 0, x = 0;
            for (int i = 0; i < W; ++i) most = fmaxf(most, stat[i][16 * n + c][0]);
            for (int i = 0; i < W; ++i) {
                total += stat[i][16 * n + c][1] * attn_exp2(stat[i][16 * n + c][0] - most);
                x += sums[(i * 16 + c) * OP + d];
            }
            const int pos = p0 + col / a.group, head = h * a.group + col % a.group;
            const int64_t token = seq.t0 + col / a.group;
            if (seq.bad) x = total = __builtin_nanf("");
            if (a.splits == 1) {
                a.out[((int64_t)head * D + d) * a.ldo + token] = attn_narrow<BF>(pos < 0 ? 0 : x / total);
            } else {
                const int64_t row = ((int64_t)split * a.heads * a.group + head) * a.tokens + token;
                a.part_o[row * D + d] = x;
                if (d == 0) {
                    a.part_ml[2 * row] = pos < 0 ? -INFINITY : most;
                    a.part_ml[2 * row + 1] = total;
                }
            }
        }
        __syncthreads();
    }
}

// ---- tiles of queries
//
// A workgroup takes one sequence and key head and 8 items, one per wavefront: 32 neighbouring queries of one of the
// group's heads; heads vary fastest, so that grouped heads share the tiles of keys and values.  Tiles of 64 keys are brought to the LDS
// by all wavefronts, the next while this one is worked on: from the cache unpacked, [key][feature]; from a prompt as they lie,
// [feature][key].  What lies the wrong way for its product is turned by transposing reads.
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

template <bool BF, int D, bool CACHE>
__global__ __launch_bounds__(64 * ATTN_WAVES, 2) void attention_tile_kernel(AttnArgs a)
{
    using Stage = AttnStage<BF, D, CACHE>;
    constexpr int S = D / 16, DT = D / 32, KP = Stage::KP, VP = Stage::VP;
    constexpr int SB = scale_bytes(D);
    constexpr int UNITS = D / 32;                          // 16-byte units of a tile per thread (prompt), words (cache)
    __shared__ __attribute__((aligned(16))) char smem[2][Stage::BYTES];
    __shared__ int special[2];                             // tile of the buffer that holds an infinity or a NaN among its values

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int half = lane >> 5, c = lane & 31;
    // a sequence and key head's workgroups on one XCD, whose L2 holds its keys and values; those with most keys first
    const int per_pair = a.col_blocks * a.splits;
    const int pair = (int)(blockIdx.x % 8 + blockIdx.x / 8 / per_pair * 8), inner = blockIdx.x / 8 % per_pair;
    if (pair >= a.batch * a.heads) return;
    const int blk = a.col_blocks - 1 - inner / a.splits, split = inner % a.splits;
    const int b = pair / a.heads, h = pair % a.heads;

    const AttnSeq seq = attn_sequence<CACHE>(a, b);
    const int blocks = (seq.nq + ATTN_TILE_QUERIES - 1) / ATTN_TILE_QUERIES;
    const int64_t items = (int64_t)blocks * a.group, item0 = (int64_t)blk * ATTN_WAVES;
    if (item0 >= items) return;
    const int64_t item_last = items < item0 + ATTN_WAVES ? items - 1 : item0 + ATTN_WAVES - 1;
    const int shift = CACHE ? 0 : (int)(seq.t0 & 7);       // tiles of a prompt begin at multiples of 8 columns
    const int p0 = seq.len - seq.nq;
    const auto position = [&](int64_t query) { return p0 + (int)(query < seq.nq ? query : seq.nq - 1); };
    const int wg_first = position(item0 / a.group * ATTN_TILE_QUERIES);
    const int wg_last = position(item_last / a.group * ATTN_TILE_QUERIES + ATTN_TILE_QUERIES - 1);
    const AttnTiles tiles = attn_tiles(wg_first, wg_last, a.window, a.sinks, shift, ATTN_TILE_KEYS);
    const int v_begin = split * (a.splits > 1 ? a.split_tiles : 0);
    const int v_end = a.splits == 1 || tiles.count - v_begin < a.split_tiles ? tiles.count : v_begin + a.split_tiles;

    const bool works = item0 + wave <= item_last;
    const int64_t item = works ? item0 + wave : item_last;
    const int head = h * a.group + (int)(item % a.group);
    const int query = (int)(item / a.group) * ATTN_TILE_QUERIES + c;
    const int first = position(query - c), last = position(query - c + ATTN_TILE_QUERIES - 1), p = position(query);
    const int lo = attn_window_start(p, a.window);
    const int64_t token = seq.t0 + (query < seq.nq ? query : seq.nq - 1);

    // queries: lane c has column c; features 16 s + 8 half and up
    uint4v q[S];
    {
        const uint16_t* src = a.q + ((int64_t)head * D + 8 * half) * a.ldq + token;
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                q[s][i] = src[(int64_t)(16 * s + 2 * i) * a.ldq] | (unsigned)src[(int64_t)(16 * s + 2 * i + 1) * a.ldq] << 16;
    }

    // ---- staging
    const int page = 1 << a.page_shift;
    const int64_t chunk = page_head_bytes(page, D);
    const int32_t* table = CACHE ? a.table + (int64_t)b * a.table_ld : nullptr;
    const int kind = tid >> 8, sub = tid >> 6 & 3;         // cache: keys or values, 16 of a tile's keys
    const int row = kind ? ((lane >> 4) & 1) * 8 + ((lane >> 1) & 7) : lane & 15;      // the thread's key among these
    const int part = kind ? (lane & 1) + 2 * (lane >> 5) : lane >> 4;                  // and its words' 8 features of 32
    uint4v unit[CACHE ? 1 : UNITS];
    unsigned word[CACHE ? UNITS : 1], codes = 0;
    const auto load = [&](int v) __attribute__((always_inline)) {
        const int t = tiles.real(v);
        if constexpr (CACHE) {
            const int key = t * ATTN_TILE_KEYS + sub * 16;
            const int idx = key >> a.page_shift, at = key & (page - 1);
            const int id = idx < a.table_width ? table[idx] : -1;
            const bool known = (unsigned)id < (unsigned)a.pages;
            const char* base = a.cache + ((int64_t)(known ? id : 0) * a.heads + h) * chunk;
            const unsigned* src = reinterpret_cast<const unsigned*>(base + (int64_t)kind * page * D / 2 + code_offset(D, at, lane));
#pragma unroll
            for (int s = 0; s < UNITS; ++s) word[s] = src[s];
            const char* sc = base + (int64_t)page * D + (int64_t)(kind * page + at + row) * SB;
            codes = SB == 2 ? *reinterpret_cast<const uint16_t*>(sc) : *reinterpret_cast<const unsigned*>(sc);
            if (!known) codes = 0xffffffffu;               // a page that is not there reads as NaN
        } else {
#pragma unroll
            for (int i = 0; i < UNITS; ++i) {
                const int e = tid + 512 * i, f = (e >> 3) % D;
                const bool is_v = e >= 8 * D;
                const int64_t at = seq.t0 - shift + (int64_t)t * ATTN_TILE_KEYS + (e & 7) * 8;
                const uint16_t* src = (is_v ? a.v : a.k) + ((int64_t)h * D + f) * (is_v ? a.ldv : a.ldk);
                uint4v x = {0, 0, 0, 0};
                if (at + 8 <= a.tokens) {
                    __builtin_memcpy(&x, src + at, 16);
                } else {
                    for (int j = 0; j < 8; ++j)
                        if (at + j < a.tokens) x[j >> 1] |= (unsigned)src[at + j] << 16 * (j & 1);
                }
                unit[i] = x;
            }
        }
    };
    const auto store = [&](int v) __attribute__((always_inline)) {
        char* buf = smem[v & 1];
        bool found = false;
        if constexpr (CACHE) {
            char* dst = buf + (kind ? Stage::K_BYTES + (sub * 16 + row) * VP : (sub * 16 + row) * KP) + part * 16;
#pragma unroll
            for (int s = 0; s < UNITS; ++s) {
                found |= kind && (codes >> 8 * s & 255) == 255;
                *reinterpret_cast<uint4v*>(dst + s * 64) = attn_unpack<BF>(word[s], codes >> 8 * s & 255);
            }
        } else {
            constexpr unsigned EXP = BF ? 0x7f80u : 0x7c00u;
#pragma unroll
            for (int i = 0; i < UNITS; ++i) {
                const int e = tid + 512 * i, f = (e >> 3) % D;
                const bool is_v = e >= 8 * D;
                *reinterpret_cast<uint4v*>(buf + (is_v ? Stage::K_BYTES : 0) + f * 128 + ((e & 7) ^ attn_unit(f)) * 16) = unit[i];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    found |= is_v && ((unit[i][j] & EXP) == EXP || (unit[i][j] >> 16 & EXP) == EXP);
            }
        }
        if (found) special[v & 1] = v;
    };

    float16v o[DT] = {};
    float m = -FLT_MAX, l = 0;

    if (tid < 2) special[tid] = -1;
    if (v_begin < v_end) load(v_begin);
    __syncthreads();
    if (v_begin < v_end) store(v_begin);

    for (int v = v_begin; v < v_end; ++v) {
        __syncthreads();
        if (v + 1 < v_end) load(v + 1);
        const int j0 = tiles.real(v) * ATTN_TILE_KEYS - shift, j1 = j0 + ATTN_TILE_KEYS - 1;
        const bool needed = works && j0 <= last && j1 >= 0 && (j1 >= attn_window_start(first, a.window) || j0 < a.sinks);
        if (needed) {
            const char* kb = smem[v & 1];
            const char* vb = kb + Stage::K_BYTES;
            const bool masked = j0 < 0 || j1 > first || (j0 < attn_window_start(last, a.window) && j1 >= a.sinks);
            float16v sc[2] = {};
#pragma unroll
            for (int s = 0; s < S; ++s)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    uint4v x;
                    if constexpr (CACHE) {
                        x = *reinterpret_cast<const uint4v*>(kb + (32 * t + c) * KP + (2 * s + half) * 16);
                    } else {
                        // rows 8 x + 4 half + i of the scores' tile are to be keys 16 .. + 8 half + 4 x + i: the two
                        // middle groups of four of every 16 change places
                        const int i = lane & 15, f = 16 * s + 8 * half + (i >> 2);
                        const int at = 32 * t + 16 * (lane >> 4 & 1) + ((i & 1) << 1 | (i >> 1 & 1)) * 4;   // first of four keys
                        const uint2 one = attn_transposed((attn_lds)kb + f * 128 + ((at >> 3) ^ attn_unit(f)) * 16 + (at & 4) * 2);
                        const uint2 two = attn_transposed((attn_lds)kb + (f + 4) * 128 + ((at >> 3) ^ attn_unit(f + 4)) * 16 + (at & 4) * 2);
                        x = uint4v{one.x, one.y, two.x, two.y};
                    }
                    sc[t] = attn_mma32<BF>(x, q[s], sc[t]);
                }
            // key of the scores' register i of tile t
            const auto key = [&](int t, int i) __attribute__((always_inline)) {
                return j0 + 32 * t + (CACHE ? 8 * (i >> 2) + 4 * half + (i & 3) : 16 * (i >> 3) + 8 * half + (i & 7));
            };
            float top = -INFINITY;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    if (masked && !attn_sees(key(t, i), p, lo, a.sinks)) sc[t][i] = -INFINITY;
                    top = fmaxf(top, sc[t][i]);
                }
            const float2v both = attn_pair32(top);
            top = fmaxf(both[0], both[1]) * a.scale;
            if (__any(top > m)) {
                const float now = fmaxf(m, top), shrink = attn_exp2(m - now);
                m = now;
                l *= shrink;
#pragma unroll
                for (int t = 0; t < DT; ++t) o[t] *= shrink;
            }
            uint4v w[4];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 16; i += 2) {
                    const float x = attn_exp2(__builtin_fmaf(sc[t][i], a.scale, -m)), y = attn_exp2(__builtin_fmaf(sc[t][i + 1], a.scale, -m));
                    l += x + y;
                    w[2 * t + (i >> 3)][(i & 7) >> 1] = attn_pack<BF>(x, y);
                }
            // a value at keys that only some of the queries see must not reach the others as 0 * NaN: infinities and
            // NaN are added where they are seen, and are zeros in the product
            const bool apart = masked && __builtin_amdgcn_readfirstlane(special[v & 1]) == v;
            if (apart) {
                for (int n = 0; n < ATTN_TILE_KEYS; ++n) {
                    const bool seen = attn_sees(j0 + n, p, lo, a.sinks);
#pragma unroll
                    for (int t = 0; t < DT; ++t)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int d = 32 * t + 8 * (i >> 2) + 4 * half + (i & 3);
                            const uint16_t x = *reinterpret_cast<const uint16_t*>(
                                CACHE ? vb + n * VP + d * 2 : vb + d * 128 + ((n >> 3) ^ attn_unit(d)) * 16 + (n & 7) * 2);
                            const float f = attn_widen<BF>(x);
                            if (seen && !(__builtin_fabsf(f) < INFINITY)) o[t][i] += f;
                        }
                }
            }
#pragma unroll
            for (int g = 0; g < 4; ++g)
#pragma unroll
                for (int t = 0; t < DT; ++t) {
                    uint4v x;
                    if constexpr (CACHE) {
                        const int i = lane & 15;
                        const attn_lds at = (attn_lds)vb + (16 * g + 4 * half + (i >> 2)) * VP + (32 * t + 16 * (lane >> 4 & 1) + (i & 3) * 4) * 2;
                        const uint2 one = attn_transposed(at), two = attn_transposed(at + 8 * VP);
                        x = uint4v{one.x, one.y, two.x, two.y};
                    } else {
                        const int d = 32 * t + c;
                        x = *reinterpret_cast<const uint4v*>(vb + d * 128 + ((2 * g + half) ^ attn_unit(d)) * 16);
                    }
                    if (apart) {
                        constexpr unsigned EXP = BF ? 0x7f80u : 0x7c00u;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            if ((x[j] & EXP) == EXP) x[j] &= 0xffff0000u;
                            if ((x[j] >> 16 & EXP) == EXP) x[j] &= 0xffffu;
                        }
                    }
                    o[t] = attn_mma32<BF>(x, w[g], o[t]);
                }
        }
        if (v + 1 < v_end) store(v + 1);
    }

    const float2v both = attn_pair32(l);
    l = both[0] + both[1];
    if (!works || query >= seq.nq) return;
    if (seq.bad) l = __builtin_nanf("");
    if (a.splits == 1) {
        const float f = p < 0 ? 0 : 1 / l;
        uint16_t* dst = a.out + ((int64_t)head * D + 4 * half) * a.ldo + token;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                dst[(int64_t)(32 * t + 8 * (i >> 2) + (i & 3)) * a.ldo] = attn_narrow<BF>(o[t][i] * f);
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
// A workgroup takes 16 tokens of one query head: the parts' sums are read along their features, the results leave along the tokens.
template <bool BF, int D>
__global__ __launch_bounds__(256) void attention_join_kernel(AttnArgs a)
{
    __shared__ uint16_t tile[D][17];
    const int64_t token0 = (int64_t)blockIdx.x * 16;
    const int head = blockIdx.y, heads = a.heads * a.group;
    const int64_t stride = (int64_t)heads * a.tokens;
    for (int e = threadIdx.x; e < 16 * D; e += 256) {
        const int c = e / D, d = e % D;
        if (token0 + c >= a.tokens) break;
        const int64_t at = (int64_t)head * a.tokens + token0 + c;
        float top = -FLT_MAX, total = 0, x = 0;
        for (int i = 0; i < a.splits; ++i) top = fmaxf(top, a.part_ml[2 * (at + i * stride)]);
        for (int i = 0; i < a.splits; ++i) {
            const float f = attn_exp2(a.part_ml[2 * (at + i * stride)] - top);
            total += a.part_ml[2 * (at + i * stride) + 1] * f;
            x += a.part_o[(at + i * stride) * D + d] * f;
        }
        tile[d][c] = attn_narrow<BF>(a.part_ml[2 * at] == -INFINITY ? 0 : x / total);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < 16 * D; e += 256) {
        const int c = e & 15, d = e >> 4;
        if (token0 + c < a.tokens) a.out[((int64_t)head * D + d) * a.ldo + token0 + c] = tile[d][c];
    }
}

}  // namespace shflbw
