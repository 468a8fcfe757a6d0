// The 4-bit cache of keys and values: tokens written into it and read back.
//
// Activations are features x tokens, so a thread takes one token's 32 features of a block at the stride of a row, and
// neighbouring threads take neighbouring tokens: every load and store of the 16-bit side is contiguous along the tokens.
// Bound by memory: 2 bytes of a value in or out, 17/32 in the cache (13/24 for heads of 96, whose scales are padded).  65536 tokens, 8 heads of
// 128 (f16): 340 MB each way, 79 us to write and 82 to read, 4.2 TB/s; a large copy moves 5.1.  Two tokens a thread, with half as many and
// wider accesses, took 192 us for both where one takes 162.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "attention.h"
#include "shflbw.h"
#include "shflbw_internal.h"

namespace shflbw {
namespace {

typedef _Float16 kv_half2 __attribute__((ext_vector_type(2)));
typedef __bf16 kv_bf2 __attribute__((ext_vector_type(2)));

struct KvArgs {
    const uint16_t* in[2];    // keys, values [heads * D][tokens]
    uint16_t* out[2];
    int64_t ld[2];
    char* cache;
    const int32_t* slots;
    int64_t tokens, slot_count;
    int heads, page_shift;
};

// where a token's block of 32 features lies
struct KvPlace {
    char* codes;              // of the page and head, of keys or values
    char* scale;              // the block's byte
    int token;                // in the page
};
template <int D>
__device__ __forceinline__ KvPlace kv_place(const KvArgs& a, int64_t slot, int h, int kind, int s)
{
    const int page = 1 << a.page_shift, t = (int)(slot & (page - 1));
    char* base = a.cache + ((slot >> a.page_shift) * a.heads + h) * page_head_bytes(page, D);
    return KvPlace{base + (int64_t)kind * page * D / 2, base + (int64_t)page * D + (int64_t)(kind * page + t) * scale_bytes(D) + s, t};
}

// A block's scale: floor(log2) of its largest magnitude is the exponent field of that value in 32 bits.  The conversion to
// 4 bits rounds to the nearest code, ties to the even one, and takes what is beyond 6 to 6.
template <bool BF, int D>
__global__ __launch_bounds__(256) void kv_write_kernel(KvArgs a)
{
    const int64_t token = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (token >= a.tokens) return;
    const int64_t slot = a.slots[token];
    if (slot < 0 || slot >= a.slot_count) return;
    const int s = blockIdx.y % (D / 32), h = blockIdx.y / (D / 32), kind = blockIdx.z;
    const uint16_t* src = a.in[kind] + (int64_t)(h * D + s * 32) * a.ld[kind] + token;
    unsigned x[16];
    unsigned most = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const unsigned lo = src[(int64_t)(2 * i) * a.ld[kind]], hi = src[(int64_t)(2 * i + 1) * a.ld[kind]];
        most = max(most, max(lo & 0x7fffu, hi & 0x7fffu));
        x[i] = lo | hi << 16;
    }
    const bool finite = most < (BF ? 0x7f80u : 0x7c00u);
    const float largest = BF ? __builtin_bit_cast(float, most << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)most);
    const int field = (int)(__builtin_bit_cast(unsigned, largest) >> 23) - 2;
    const unsigned code = field > 1 ? field : 1;
    const float scale = __builtin_bit_cast(float, code << 23);
    const KvPlace place = kv_place<D>(a, slot, h, kind, s);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        unsigned w = 0;
        const auto pair = [&](auto n) __attribute__((always_inline)) {
            constexpr int i = decltype(n)::value;
            if constexpr (BF) w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(kv_bf2, x[4 * q + i]), scale, i);
            else w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, __builtin_bit_cast(kv_half2, x[4 * q + i]), scale, i);
        };
        pair(std::integral_constant<int, 0>{});
        pair(std::integral_constant<int, 1>{});
        pair(std::integral_constant<int, 2>{});
        pair(std::integral_constant<int, 3>{});
        const int lane = kind ? value_lane(place.token, q) : key_lane(place.token, q);
        reinterpret_cast<unsigned*>(place.codes + code_offset(D, place.token, lane))[s] = finite ? w : 0;
    }
    *place.scale = finite ? (char)code : (char)255;
}

template <bool BF, int D>
__global__ __launch_bounds__(256) void kv_read_kernel(KvArgs a)
{
    const int64_t token = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (token >= a.tokens) return;
    const int64_t slot = a.slots[token];
    const bool known = slot >= 0 && slot < a.slot_count;
    const int s = blockIdx.y % (D / 32), h = blockIdx.y / (D / 32), kind = blockIdx.z;
    const KvPlace place = kv_place<D>(a, known ? slot : 0, h, kind, s);
    const unsigned code = known ? (unsigned)(unsigned char)*place.scale : 255u;
    const float scale = __builtin_bit_cast(float, code << 23);
    uint16_t* dst = a.out[kind] + (int64_t)(h * D + s * 32) * a.ld[kind] + token;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int lane = kind ? value_lane(place.token, q) : key_lane(place.token, q);
        const unsigned w = reinterpret_cast<const unsigned*>(place.codes + code_offset(D, place.token, lane))[s];
        const auto pair = [&](auto n) __attribute__((always_inline)) {
            constexpr int i = decltype(n)::value;
            unsigned x;
            if constexpr (BF) x = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, i));
            else x = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, i));
            dst[(int64_t)(8 * q + 2 * i) * a.ld[kind]] = (uint16_t)x;
            dst[(int64_t)(8 * q + 2 * i + 1) * a.ld[kind]] = (uint16_t)(x >> 16);
        };
        pair(std::integral_constant<int, 0>{});
        pair(std::integral_constant<int, 1>{});
        pair(std::integral_constant<int, 2>{});
        pair(std::integral_constant<int, 3>{});
    }
}

int launch_kv(bool write, const shflbw_kv_cache* c, const KvArgs& a, hipStream_t stream)
{
    const int64_t blocks = (a.tokens + 255) / 256, parts = (int64_t)a.heads * (c->head_dim / 32);
    if (blocks > 0x7fffffffLL) return fail(SHFLBW_ERR_BAD_SHAPE, "grid too large");   // (check_cache: parts are at most 65535)
    const dim3 grid((unsigned)blocks, (unsigned)parts, 2);
    typedef void (*kernel)(KvArgs);
    static const kernel table[2][2][3] = {
        {{&kv_read_kernel<false, 64>, &kv_read_kernel<false, 96>, &kv_read_kernel<false, 128>},
         {&kv_read_kernel<true, 64>, &kv_read_kernel<true, 96>, &kv_read_kernel<true, 128>}},
        {{&kv_write_kernel<false, 64>, &kv_write_kernel<false, 96>, &kv_write_kernel<false, 128>},
         {&kv_write_kernel<true, 64>, &kv_write_kernel<true, 96>, &kv_write_kernel<true, 128>}}};
    hipLaunchKernelGGL(table[write][c->dtype == SHFLBW_BF16][c->head_dim / 32 - 2], grid, dim3(256), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(SHFLBW_ERR_HIP, "kernel launch: %s", hipGetErrorString(e));
    return SHFLBW_OK;
}

}  // namespace
}  // namespace shflbw

extern "C" {

int shflbw_kv_write(const shflbw_kv_cache* cache, const void* k, int64_t ldk, const void* v, int64_t ldv, const int32_t* slots, int64_t tokens,
                    void* stream)
{
    using namespace shflbw;
    const int rc = check_cache(cache);
    if (rc < 0) return rc;
    if (tokens < 0) return fail(SHFLBW_ERR_BAD_SHAPE, "tokens < 0");
    if (tokens == 0) return SHFLBW_OK;
    if (!k || !v || !slots) return fail(SHFLBW_ERR_NULL_ARG, "k, v and slots must not be NULL");
    if (ldk < tokens || ldv < tokens) return fail(SHFLBW_ERR_BAD_SHAPE, "leading dimension too small");
    KvArgs a = {};
    a.in[0] = static_cast<const uint16_t*>(k);
    a.in[1] = static_cast<const uint16_t*>(v);
    a.ld[0] = ldk; a.ld[1] = ldv;
    a.cache = static_cast<char*>(cache->data);
    a.slots = slots;
    a.tokens = tokens;
    a.slot_count = (int64_t)cache->pages * cache->page_tokens;
    a.heads = cache->heads;
    a.page_shift = __builtin_ctz(cache->page_tokens);
    return launch_kv(true, cache, a, static_cast<hipStream_t>(stream));
}

int shflbw_kv_read(const shflbw_kv_cache* cache, const int32_t* slots, int64_t tokens, void* k, int64_t ldk, void* v, int64_t ldv, void* stream)
{
    using namespace shflbw;
    const int rc = check_cache(cache);
    if (rc < 0) return rc;
    if (tokens < 0) return fail(SHFLBW_ERR_BAD_SHAPE, "tokens < 0");
    if (tokens == 0) return SHFLBW_OK;
    if (!k || !v || !slots) return fail(SHFLBW_ERR_NULL_ARG, "k, v and slots must not be NULL");
    if (ldk < tokens || ldv < tokens) return fail(SHFLBW_ERR_BAD_SHAPE, "leading dimension too small");
    KvArgs a = {};
    a.out[0] = static_cast<uint16_t*>(k);
    a.out[1] = static_cast<uint16_t*>(v);
    a.ld[0] = ldk; a.ld[1] = ldv;
    a.cache = static_cast<char*>(cache->data);
    a.slots = slots;
    a.tokens = tokens;
    a.slot_count = (int64_t)cache->pages * cache->page_tokens;
    a.heads = cache->heads;
    a.page_shift = __builtin_ctz(cache->page_tokens);
    return launch_kv(false, cache, a, static_cast<hipStream_t>(stream));
}

}  // extern "C"
