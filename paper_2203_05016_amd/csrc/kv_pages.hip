// Which pages of the cache belong to which sequences: more tokens for sequences, sequences that continue others, pages moved to the
// front.  All of it stays on the device, and everything that takes free pages takes the lowest, so that results depend on the
// arguments alone: free (or used) pages are counted by blocks of PAGES_BLOCK of them, every block adds up the counts of those before it, and
// ranks inside a block come from ballots.  Atomic additions are of whole numbers, whose order does not show.
//
// Bound by latency (a launch for every step that needs all of the step before) but for the pages that are copied.
#include <hip/hip_runtime.h>

#include <climits>
#include <cstdint>

#include "attention.h"
#include "shflbw.h"
#include "shflbw_internal.h"

namespace shflbw {
namespace {

constexpr int PAGES_BLOCK = 4096;          // pages to a workgroup of 1024 threads
constexpr int COPY_BYTES = 16384;          // bytes of a page to a workgroup of 256 threads
constexpr int MOST_BLOCKS = 16384;         // of a launch whose workgroups take pieces in turn

typedef unsigned copy4 __attribute__((ext_vector_type(4)));

struct PagesArgs {
    const int32_t* table_in;
    int32_t* table_out;
    const int32_t *lengths_in, *uses_in;
    int32_t *lengths_out, *uses_out;
    const int32_t* which;                  // counts of an extension, parents of a fork
    int32_t *slots, *starts;
    char* data;
    int64_t ld_in, ld_out, tokens, page_bytes;
    int rows_in, rows, width, pages, page_shift, blocks, page_blocks;
    // workspace: see carve
    int32_t *counts, *list, *source, *rank, *moved, *totals, *base, *old_length, *first, *children;
};
// totals: what a call's steps tell each other
enum { WANTED, FREE, LIVE_BELOW, LIVE };

__device__ __forceinline__ bool in_cache(const PagesArgs& a, int page) { return (unsigned)page < (unsigned)a.pages; }
// entries of a row that belong to a sequence of `length` tokens
__device__ __forceinline__ int held(const PagesArgs& a, int64_t length)
{
    const int64_t n = length <= 0 ? 0 : (length + (1 << a.page_shift) - 1) >> a.page_shift;
    return n < a.width ? (int)n : a.width;
}
// the entry that is not full, or -1
__device__ __forceinline__ int open_entry(const PagesArgs& a, int length)
{
    if (length <= 0 || !(length & ((1 << a.page_shift) - 1))) return -1;
    const int j = length >> a.page_shift;
    return j < a.width ? j : -1;
}

// the sum of x over the threads before this one, and over all 1024 of them
struct Scan {
    int64_t before, all;
};
__device__ __forceinline__ Scan scan_block(int64_t x, int64_t* shared)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t sum = x;
#pragma unroll
    for (int by = 1; by < 64; by *= 2) {
        const int64_t y = __shfl_up(sum, by);
        if (lane >= by) sum += y;
    }
    if (lane == 63) shared[wave] = sum;
    __syncthreads();
    Scan r = {sum - x, 0};
#pragma unroll
    for (int w = 0; w < 16; ++w) {
        if (w < wave) r.before += shared[w];
        r.all += shared[w];
    }
    __syncthreads();
    return r;
}

// ---- ranks of pages: LIVE_PAGES ones that are used, otherwise free ones
template <bool LIVE_PAGES>
__device__ __forceinline__ bool counted(const int32_t* uses, int p, int pages) { return p < pages && (LIVE_PAGES ? uses[p] != 0 : uses[p] == 0); }

template <bool LIVE_PAGES>
__device__ __forceinline__ void count_pages(const PagesArgs& a, const int32_t* uses, int block, int64_t* shared)
{
    int n = 0;
#pragma unroll
    for (int i = 0; i < PAGES_BLOCK / 1024; ++i) n += counted<LIVE_PAGES>(uses, block * PAGES_BLOCK + i * 1024 + threadIdx.x, a.pages);
    const Scan s = scan_block(n, shared);
    if (threadIdx.x == 0) a.counts[block] = (int)s.all;
}
// calls f(page, whether it is counted, how many are before it) for every page of the block; returns how many there are in all
template <bool LIVE_PAGES, class F>
__device__ __forceinline__ int rank_pages(const PagesArgs& a, const int32_t* uses, int block, int64_t* shared, F&& f)
{
    int64_t mine = 0, rest = 0;
    for (int i = threadIdx.x; i < a.page_blocks; i += 1024) (i < block ? mine : rest) += a.counts[i];
    int before = (int)scan_block(mine, shared).all;
    const int total = before + (int)scan_block(rest, shared).all;
    // (both in one pass over the block: a page is looked at before f may change its count)
    bool is[PAGES_BLOCK / 1024];
#pragma unroll
    for (int i = 0; i < PAGES_BLOCK / 1024; ++i) is[i] = counted<LIVE_PAGES>(uses, block * PAGES_BLOCK + i * 1024 + threadIdx.x, a.pages);
#pragma unroll
    for (int i = 0; i < PAGES_BLOCK / 1024; ++i) {
        const Scan s = scan_block(is[i], shared);
        f(block * PAGES_BLOCK + i * 1024 + (int)threadIdx.x, is[i], before + (int)s.before, total);
        before += (int)s.all;
    }
    return total;
}

// the lowest totals[WANTED] free pages, in order; they are in use from here on
__global__ __launch_bounds__(1024) void pages_take_kernel(PagesArgs a, const int32_t* uses)
{
    __shared__ int64_t shared[16];
    const int wanted = a.totals[WANTED];
    const int total = rank_pages<false>(a, uses, blockIdx.x, shared, [&](int p, bool free, int rank, int) {
        if (p >= a.pages) return;
        const bool taken = free && rank < wanted;
        if (taken) a.list[rank] = p;
        a.uses_out[p] = taken ? 1 : uses[p];
    });
    if (blockIdx.x == 0 && threadIdx.x == 0) a.totals[FREE] = total;
}
// the page of rank `rank` among those taken, or -1
__device__ __forceinline__ int taken_page(const PagesArgs& a, int64_t rank) { return rank < a.totals[FREE] ? a.list[rank] : -1; }

// ---- more tokens
__device__ __forceinline__ void extend_rows(const PagesArgs& a, int64_t* shared)
{
    int64_t pages = 0, tokens = 0;
    for (int b0 = 0; b0 < a.rows; b0 += 1024) {
        const int b = b0 + threadIdx.x;
        int64_t need = 0, count = 0;
        if (b < a.rows) {
            const int length = a.lengths_in[b] > 0 ? a.lengths_in[b] : 0;
            count = a.which[b] > 0 ? a.which[b] : 0;
            need = held(a, length + count) - held(a, length);
            a.old_length[b] = length;
            const int64_t now = length + count;
            a.lengths_out[b] = now < INT_MAX ? (int)now : INT_MAX;
        }
        const Scan p = scan_block(need, shared), t = scan_block(count, shared);
        if (b < a.rows) {
            const int64_t start = tokens + t.before, base = pages + p.before;
            a.starts[b] = start < INT_MAX ? (int)start : INT_MAX;
            a.base[b] = base < INT_MAX ? (int)base : INT_MAX;
        }
        pages += p.all;
        tokens += t.all;
    }
    if (threadIdx.x == 0) {
        a.starts[a.rows] = tokens < INT_MAX ? (int)tokens : INT_MAX;
        a.totals[WANTED] = pages < INT_MAX ? (int)pages : INT_MAX;
    }
}
__global__ __launch_bounds__(1024) void extend_count_kernel(PagesArgs a)
{
    __shared__ int64_t shared[16];
    if ((int)blockIdx.x < a.page_blocks) count_pages<false>(a, a.uses_in, blockIdx.x, shared);
    else extend_rows(a, shared);
}
// entry j of a sequence that had `old` of them
__device__ __forceinline__ int extended(const PagesArgs& a, int b, int j, int old)
{
    return j < old ? a.table_in[b * a.ld_in + j] : taken_page(a, (int64_t)a.base[b] + j - old);
}
__global__ __launch_bounds__(256) void extend_apply_kernel(PagesArgs a)
{
    const int64_t entries = (int64_t)a.rows * a.width, step = (int64_t)gridDim.x * 256;
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < entries + a.tokens; e += step) {
        if (e < entries) {
            const int b = (int)(e / a.width), j = (int)(e % a.width), old = held(a, a.old_length[b]);
            a.table_out[b * a.ld_out + j] = j < held(a, a.lengths_out[b]) ? extended(a, b, j, old) : -1;
            continue;
        }
        const int64_t t = e - entries;
        int slot = -1;
        if (t < a.starts[a.rows]) {
            int low = 0, high = a.rows;                    // starts[low] <= t < starts[high]
            while (high - low > 1) {
                const int mid = low + (high - low) / 2;
                if (a.starts[mid] <= t) low = mid;
                else high = mid;
            }
            const int64_t at = a.old_length[low] + t - a.starts[low], j = at >> a.page_shift;
            const int page = j < a.width ? extended(a, low, (int)j, held(a, a.old_length[low])) : -1;
            if (in_cache(a, page)) slot = (page << a.page_shift) + (int)(at & ((1 << a.page_shift) - 1));
        }
        a.slots[t] = slot;
    }
}

// ---- sequences that continue others
//
// A row's children and the lowest of them; what every child wants of fresh pages (its open page, where it is not the lowest).
__device__ __forceinline__ int load_shared(const int32_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ bool has_parent(const PagesArgs& a, int parent) { return (unsigned)parent < (unsigned)a.rows_in; }
__global__ __launch_bounds__(1024) void fork_count_kernel(PagesArgs a)
{
    __shared__ int64_t shared[16];
    if (blockIdx.x) {                                      // the counts, to be changed
        for (int64_t p = (int64_t)(blockIdx.x - 1) * 1024 + threadIdx.x; p < a.pages; p += (int64_t)(gridDim.x - 1) * 1024) a.uses_out[p] = a.uses_in[p];
        return;
    }
    for (int b = threadIdx.x; b < a.rows_in; b += 1024) {
        __hip_atomic_store(a.first + b, INT_MAX, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(a.children + b, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __threadfence();
    __syncthreads();
    for (int i = threadIdx.x; i < a.rows; i += 1024) {
        const int parent = a.which[i];
        if (!has_parent(a, parent)) continue;
        atomicMin(a.first + parent, i);
        atomicAdd(a.children + parent, 1);
    }
    __threadfence();
    __syncthreads();
    int64_t pages = 0;
    for (int i0 = 0; i0 < a.rows; i0 += 1024) {
        const int i = i0 + threadIdx.x;
        bool need = false;
        if (i < a.rows) {
            const int parent = a.which[i];
            const int length = has_parent(a, parent) && a.lengths_in[parent] > 0 ? a.lengths_in[parent] : 0, j = open_entry(a, length);
            a.lengths_out[i] = length;
            need = j >= 0 && load_shared(a.first + parent) != i && in_cache(a, a.table_in[parent * a.ld_in + j]);
        }
        const Scan s = scan_block(need, shared);
        if (i < a.rows) a.base[i] = need ? (int)(pages + s.before) : -1;
        pages += s.all;
    }
    if (threadIdx.x == 0) a.totals[WANTED] = (int)pages;
}
// Every old entry's page is named by as many entries as its row has children, an open one by the lowest's: the count changes by that less one.
__global__ __launch_bounds__(256) void fork_table_kernel(PagesArgs a)
{
    const int64_t old = (int64_t)a.rows_in * a.width, all = old + (int64_t)a.rows * a.width, step = (int64_t)gridDim.x * 256;
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < all; e += step) {
        if (e < old) {
            const int b = (int)(e / a.width), j = (int)(e % a.width);
            if (j >= held(a, a.lengths_in[b])) continue;
            const int page = a.table_in[b * a.ld_in + j], children = a.children[b];
            const int change = (j == open_entry(a, a.lengths_in[b]) && children > 1 ? 1 : children) - 1;
            if (change && in_cache(a, page)) atomicAdd(a.uses_out + page, change);
        } else {
            const int i = (int)((e - old) / a.width), j = (int)((e - old) % a.width), parent = a.which[i];
            const bool has = has_parent(a, parent) && j < held(a, a.lengths_in[parent]);
            a.table_out[i * a.ld_out + j] = has ? a.table_in[parent * a.ld_in + j] : -1;
        }
    }
}
__global__ __launch_bounds__(1024) void pages_count_kernel(PagesArgs a)
{
    __shared__ int64_t shared[16];
    count_pages<false>(a, a.uses_out, blockIdx.x, shared);
}
// piece `part` of page `from` to page `to`
__device__ __forceinline__ void copy_piece(const PagesArgs& a, int from, int to, int part)
{
    const int64_t begin = (int64_t)part * COPY_BYTES;
    const char* src = a.data + from * a.page_bytes;
    char* dst = a.data + to * a.page_bytes;
    copy4 x[COPY_BYTES / 4096];
#pragma unroll
    for (int i = 0; i < COPY_BYTES / 4096; ++i) {
        const int64_t at = begin + i * 4096 + threadIdx.x * 16;
        if (at < a.page_bytes) x[i] = *reinterpret_cast<const copy4*>(src + at);
    }
#pragma unroll
    for (int i = 0; i < COPY_BYTES / 4096; ++i) {
        const int64_t at = begin + i * 4096 + threadIdx.x * 16;
        if (at < a.page_bytes) *reinterpret_cast<copy4*>(dst + at) = x[i];
    }
}
__global__ __launch_bounds__(256) void fork_copy_kernel(PagesArgs a, int parts)
{
    for (int64_t n = blockIdx.x; n < (int64_t)a.rows * parts; n += gridDim.x) {
        const int i = (int)(n / parts), part = (int)(n % parts), rank = a.base[i];
        if (rank < 0) continue;
        const int parent = a.which[i], j = open_entry(a, a.lengths_in[parent]), to = taken_page(a, rank);
        if (part == 0 && threadIdx.x == 0) a.table_out[i * a.ld_out + j] = to;
        if (to >= 0) copy_piece(a, a.table_in[parent * a.ld_in + j], to, part);
    }
}

// ---- pages in use to the front
//
// With n of them: those from n on have ranks totals[LIVE_BELOW] and up among the pages in use, and as many pages below n are free; the i-th goes to the i-th.
__global__ __launch_bounds__(1024) void compact_count_kernel(PagesArgs a)
{
    __shared__ int64_t shared[16];
    count_pages<true>(a, a.uses_in, blockIdx.x, shared);
}
__global__ __launch_bounds__(1024) void compact_rank_kernel(PagesArgs a)
{
    __shared__ int64_t shared[16];
    rank_pages<true>(a, a.uses_in, blockIdx.x, shared, [&](int p, bool live, int rank, int total) {
        if (p == total || (p == a.pages - 1 && total == a.pages)) {
            a.totals[LIVE_BELOW] = p == total ? rank : total;
            a.totals[LIVE] = total;
        }
        if (p >= a.pages) return;
        const int uses = a.uses_in[p];
        if (p < total) {
            if (live) a.uses_out[p] = uses;
            else a.list[p - rank] = p;                     // (its count comes with the page that moves here)
        } else {
            a.rank[p] = live ? rank : -1;
            a.uses_out[p] = 0;
            if (live) {
                a.source[rank] = p;
                a.moved[rank] = uses;
            }
        }
    });
}
__global__ __launch_bounds__(256) void compact_apply_kernel(PagesArgs a, int parts, int table_blocks)
{
    const int below = a.totals[LIVE_BELOW], live = a.totals[LIVE];
    if ((int)blockIdx.x < table_blocks) {
        for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < (int64_t)a.rows * a.width; e += (int64_t)table_blocks * 256) {
            const int64_t b = e / a.width, j = e % a.width;
            int page = a.table_in[b * a.ld_in + j];
            if (page >= live && page < a.pages && a.rank[page] >= 0) page = a.list[a.rank[page] - below];
            a.table_out[b * a.ld_out + j] = page;
        }
        return;
    }
    const int64_t pieces = (int64_t)(live - below) * parts;
    for (int64_t n = blockIdx.x - table_blocks; n < pieces; n += gridDim.x - table_blocks) {
        const int i = (int)(n / parts), part = (int)(n % parts), from = a.source[below + i], to = a.list[i];
        if (part == 0 && threadIdx.x == 0) a.uses_out[to] = a.moved[below + i];
        copy_piece(a, from, to, part);
    }
}

// ---- calls
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
unsigned few_blocks(int64_t pieces) { return (unsigned)(pieces < 1 ? 1 : pieces < MOST_BLOCKS ? pieces : MOST_BLOCKS); }

int64_t workspace_bytes_of(int64_t pages, int64_t sequences)
{
    return 4 * (4 * pages + ceil_div(pages, PAGES_BLOCK) + 4 * sequences + 4);
}
void carve(PagesArgs& a, void* workspace, int64_t sequences)
{
    int32_t* at = static_cast<int32_t*>(workspace);
    const auto take = [&](int64_t n) { int32_t* p = at; at += n; return p; };
    a.totals = take(4);
    a.list = take(a.pages);
    a.source = take(a.pages);
    a.rank = take(a.pages);
    a.moved = take(a.pages);
    a.counts = take(a.page_blocks);
    a.base = take(sequences);
    a.old_length = take(sequences);
    a.first = take(sequences);
    a.children = take(sequences);
}

struct Span {
    const void* base;
    int64_t count;             // of 4 bytes
};
Span table_span(const shflbw_kv_pages* p) { return Span{p->table, p->sequences ? (p->sequences - 1) * p->table_ld + p->table_pages : 0}; }
bool overlap(const Span& x, const Span& y)
{
    const uintptr_t a = reinterpret_cast<uintptr_t>(x.base), b = reinterpret_cast<uintptr_t>(y.base);
    return x.count && y.count && a < b + 4 * y.count && b < a + 4 * x.count;
}
int check_pages(const shflbw_kv_pages* p)
{
    if (!p) return fail(SHFLBW_ERR_NULL_ARG, "pages is NULL");
    if (p->sequences < 0 || p->table_pages < 1 || p->table_ld < p->table_pages) return fail(SHFLBW_ERR_BAD_SHAPE, "sequences < 0, table_pages < 1 or table_ld < table_pages");
    if (!p->uses || (p->sequences && !p->table)) return fail(SHFLBW_ERR_NULL_ARG, "table and uses must not be NULL");
    return SHFLBW_OK;
}
// Checks what the three calls have in common and fills in a.  in_place: tables and lengths may be the same.  lengths: they are needed.
int begin(PagesArgs& a, const shflbw_kv_cache* c, const shflbw_kv_pages* in, const shflbw_kv_pages* out, bool in_place, bool lengths, void* workspace,
          int64_t workspace_bytes)
{
    int rc = check_cache(c);
    if (rc < 0 || (rc = check_pages(in)) < 0 || (rc = check_pages(out)) < 0) return rc;
    if (in->table_pages != out->table_pages) return fail(SHFLBW_ERR_BAD_SHAPE, "tables of different width");
    if (in_place && in->sequences != out->sequences) return fail(SHFLBW_ERR_BAD_SHAPE, "different numbers of sequences");
    if ((int64_t)in->table_pages * c->page_tokens > INT_MAX - 1024) return fail(SHFLBW_ERR_BAD_SHAPE, "more than 2^31 tokens in a sequence's pages");
    if (lengths && ((in->sequences && !in->lengths) || (out->sequences && !out->lengths))) return fail(SHFLBW_ERR_NULL_ARG, "lengths must not be NULL");
    const Span from[3] = {table_span(in), {in->lengths, lengths ? in->sequences : 0}, {in->uses, c->pages}};
    const Span to[3] = {table_span(out), {out->lengths, lengths ? out->sequences : 0}, {out->uses, c->pages}};
    for (int i = 0; i < 3; ++i)
        for (int j = 0; j < 3; ++j) {
            const bool same = i == j && from[j].base == to[i].base && (i == 2 || (in_place && (i == 1 || in->table_ld == out->table_ld)));
            if (overlap(to[i], from[j]) && !same) return fail(SHFLBW_ERR_BAD_SHAPE, "arrays of out overlap those of in");
            if (i != j && overlap(to[i], to[j])) return fail(SHFLBW_ERR_BAD_SHAPE, "arrays of out overlap each other");
        }
    const int64_t sequences = in->sequences > out->sequences ? in->sequences : out->sequences;
    if (!workspace || workspace_bytes < workspace_bytes_of(c->pages, sequences))
        return fail(SHFLBW_ERR_NULL_ARG, "the call needs a workspace of %lld bytes", (long long)workspace_bytes_of(c->pages, sequences));
    if (reinterpret_cast<uintptr_t>(workspace) % 16) return fail(SHFLBW_ERR_BAD_SHAPE, "the workspace must be 16-byte aligned");
    a.table_in = in->table;
    a.table_out = out->table;
    a.lengths_in = in->lengths;
    a.lengths_out = out->lengths;
    a.uses_in = in->uses;
    a.uses_out = out->uses;
    a.ld_in = in->table_ld;
    a.ld_out = out->table_ld;
    a.rows_in = in->sequences;
    a.rows = out->sequences;
    a.width = in->table_pages;
    a.pages = c->pages;
    a.page_shift = __builtin_ctz(c->page_tokens);
    a.page_blocks = (int)ceil_div(c->pages, PAGES_BLOCK);
    a.data = static_cast<char*>(c->data);
    a.page_bytes = page_head_bytes(c->page_tokens, c->head_dim) * c->heads;
    carve(a, workspace, sequences);
    return SHFLBW_OK;
}
int launched()
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SHFLBW_OK : fail(SHFLBW_ERR_HIP, "kernel launch: %s", hipGetErrorString(e));
}

}  // namespace
}  // namespace shflbw

extern "C" {

int64_t shflbw_kv_pages_workspace(const shflbw_kv_cache* cache, int sequences)
{
    using namespace shflbw;
    const int rc = check_cache(cache);
    if (rc < 0) return rc;
    if (sequences < 0) return fail(SHFLBW_ERR_BAD_SHAPE, "sequences < 0");
    return workspace_bytes_of(cache->pages, sequences);
}

int shflbw_kv_extend(const shflbw_kv_cache* cache, const shflbw_kv_pages* in, const shflbw_kv_pages* out, const int32_t* counts, int32_t* slots,
                     int32_t* starts, int64_t tokens, void* workspace, int64_t workspace_bytes, void* stream)
{
    using namespace shflbw;
    PagesArgs a = {};
    const int rc = begin(a, cache, in, out, true, true, workspace, workspace_bytes);
    if (rc < 0) return rc;
    if (tokens < 0 || tokens > INT_MAX) return fail(SHFLBW_ERR_BAD_SHAPE, "tokens must be 0 to 2^31 - 1");
    if (!starts || (tokens && !slots) || (a.rows && !counts)) return fail(SHFLBW_ERR_NULL_ARG, "counts, slots and starts must not be NULL");
    a.which = counts;
    a.slots = slots;
    a.starts = starts;
    a.tokens = tokens;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    hipLaunchKernelGGL(extend_count_kernel, dim3(a.page_blocks + 1), dim3(1024), 0, st, a);
    hipLaunchKernelGGL(pages_take_kernel, dim3(a.page_blocks), dim3(1024), 0, st, a, a.uses_in);
    hipLaunchKernelGGL(extend_apply_kernel, dim3(few_blocks(ceil_div((int64_t)a.rows * a.width + tokens, 256))), dim3(256), 0, st, a);
    return launched();
}

int shflbw_kv_fork(const shflbw_kv_cache* cache, const shflbw_kv_pages* in, const shflbw_kv_pages* out, const int32_t* parents, void* workspace,
                   int64_t workspace_bytes, void* stream)
{
    using namespace shflbw;
    PagesArgs a = {};
    const int rc = begin(a, cache, in, out, false, true, workspace, workspace_bytes);
    if (rc < 0) return rc;
    if (a.rows && !parents) return fail(SHFLBW_ERR_NULL_ARG, "parents must not be NULL");
    a.which = parents;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const int parts = (int)ceil_div(a.page_bytes, COPY_BYTES);
    hipLaunchKernelGGL(fork_count_kernel, dim3(a.uses_in == a.uses_out ? 1 : 1 + few_blocks(ceil_div(a.pages, 1024))), dim3(1024), 0, st, a);
    hipLaunchKernelGGL(fork_table_kernel, dim3(few_blocks(ceil_div(((int64_t)a.rows_in + a.rows) * a.width, 256))), dim3(256), 0, st, a);
    hipLaunchKernelGGL(pages_count_kernel, dim3(a.page_blocks), dim3(1024), 0, st, a);
    hipLaunchKernelGGL(pages_take_kernel, dim3(a.page_blocks), dim3(1024), 0, st, a, a.uses_out);
    hipLaunchKernelGGL(fork_copy_kernel, dim3(few_blocks((int64_t)a.rows * parts)), dim3(256), 0, st, a, parts);
    return launched();
}

int shflbw_kv_compact(const shflbw_kv_cache* cache, const shflbw_kv_pages* in, const shflbw_kv_pages* out, void* workspace, int64_t workspace_bytes,
                      void* stream)
{
    using namespace shflbw;
    PagesArgs a = {};
    const int rc = begin(a, cache, in, out, true, false, workspace, workspace_bytes);
    if (rc < 0) return rc;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const int parts = (int)ceil_div(a.page_bytes, COPY_BYTES), table_blocks = (int)few_blocks(ceil_div((int64_t)a.rows * a.width, 256));
    // at most half of the pages move
    const unsigned copy_blocks = few_blocks((int64_t)(a.pages / 2) * parts);
    hipLaunchKernelGGL(compact_count_kernel, dim3(a.page_blocks), dim3(1024), 0, st, a);
    hipLaunchKernelGGL(compact_rank_kernel, dim3(a.page_blocks), dim3(1024), 0, st, a);
    hipLaunchKernelGGL(compact_apply_kernel, dim3(table_blocks + copy_blocks), dim3(256), 0, st, a, parts, table_blocks);
    return launched();
}

}  // extern "C"
