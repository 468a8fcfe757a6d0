// Which pages of the cache belong to which sequences: more tokens for sequences, sequences that continue others, pages moved to the
// front.  All of it stays on the device, and everything that takes free pages takes the lowest, so that results depend on the
// arguments alone: free (or used) pages are counted by blocks of PAGES_BLOCK of them, every block adds up the counts of those before it, and
// ranks inside a block come from ballots.  Atomic additions are of whole numbers, whose order does not show.
//
// Bound by latency (a launch for every step that needs all of the step before, 3 to 5 us each on the GPU, of which most is the chain of loads and barriers) but
// for the pages that are copied.  64 sequences, one token more, 8192 pages: 7.7 us; 256 prompts of up to 8192 tokens, 65536 pages: 15.4; 512 sequences continued by
// 8 each, 16000 pages, 15 MB copied: 17; 2000 of 8000 pages of 70 KB to the front: 51 us, 5.4 TB/s, where part of it lies in
// the memory-side cache, 65, 4.3 TB/s, where nothing does (a large copy 5.2).
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
// What one workgroup does alone, in fewer launches: pages that it ranks, rows that it has in the LDS, entries and slots that it works out.  16 rows of
// 64 pages forked 9.4 us, one token more 6.5, where five and three launches take 20 and 12; 128 rows 16.9 and 10.2, in several launches 12.2 and 9.3.
constexpr int FEW_PAGES = 16384;
constexpr int FEW_ROWS = 2048;
constexpr int64_t FEW_ENTRIES = 8192;
static_assert(PAGES_BLOCK == 4 * 1024, "rank_flags takes four runs of 1024");

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
    int rows_in, rows, width, pages, page_shift, page_blocks;
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

// ---- sums over a workgroup of 1024 threads
//
// A wavefront's running sum by moves between lanes' registers; `shared` is 64 numbers of LDS that nothing else uses.
template <int CTRL, int ROWS>
__device__ __forceinline__ int moved_lanes(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, true); }
__device__ __forceinline__ int wave_sum(int x)               // over this lane and those before it
{
    x += moved_lanes<0x111, 0xf>(x);                         // by 1, 2, 4, 8 in rows of 16
    x += moved_lanes<0x112, 0xf>(x);
    x += moved_lanes<0x114, 0xf>(x);
    x += moved_lanes<0x118, 0xf>(x);
    x += moved_lanes<0x142, 0xa>(x);                         // the last of row 0 to 1, of 2 to 3
    x += moved_lanes<0x143, 0xc>(x);                         // the last of 1 to 2 and 3
    return x;
}
template <int CTRL, int ROWS>
__device__ __forceinline__ int64_t moved_lanes64(int64_t x)
{
    const unsigned low = (unsigned)moved_lanes<CTRL, ROWS>((int)x);
    return (int64_t)moved_lanes<CTRL, ROWS>((int)(x >> 32)) << 32 | low;
}
__device__ __forceinline__ int64_t wave_sum64(int64_t x)
{
    x += moved_lanes64<0x111, 0xf>(x);
    x += moved_lanes64<0x112, 0xf>(x);
    x += moved_lanes64<0x114, 0xf>(x);
    x += moved_lanes64<0x118, 0xf>(x);
    x += moved_lanes64<0x142, 0xa>(x);
    x += moved_lanes64<0x143, 0xc>(x);
    return x;
}
// the sum of x over the threads before this one, and over all
struct Scan {
    int64_t before, all;
};
__device__ __forceinline__ Scan scan_block(int64_t x, int64_t* shared)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t sum = wave_sum64(x);
    if (lane == 63) shared[wave] = sum;
    __syncthreads();
    const int64_t mine = lane < 16 ? shared[lane] : 0, waves = wave_sum64(mine);
    const Scan r = {__shfl(waves - mine, wave) + sum - x, __shfl(waves, 15)};
    __syncthreads();
    return r;
}
__device__ __forceinline__ int sum_block(int x, int64_t* shared)
{
    int* counts = reinterpret_cast<int*>(shared);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sum = wave_sum(x);
    if (lane == 63) counts[wave] = sum;
    __syncthreads();
    const int all = __builtin_amdgcn_readlane(wave_sum(lane < 16 ? counts[lane] : 0), 63);
    __syncthreads();
    return all;
}
// Four runs of 1024 flags, a thread's at its own number in each: how many are set before each of the thread's, and in all.
struct Ranks {
    int before[4], all;
};
__device__ __forceinline__ Ranks rank_flags(const bool (&flag)[4], int64_t* shared)
{
    int* counts = reinterpret_cast<int*>(shared);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Ranks r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint64_t set = __ballot(flag[i]);
        r.before[i] = (int)__builtin_amdgcn_mbcnt_hi((unsigned)(set >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)set, 0));
        if (lane == 0) counts[i * 16 + wave] = __popcll(set);
    }
    __syncthreads();
    const int mine = counts[lane], sum = wave_sum(mine);
#pragma unroll
    for (int i = 0; i < 4; ++i) r.before[i] += __builtin_amdgcn_readlane(sum - mine, i * 16 + wave);
    r.all = __builtin_amdgcn_readlane(sum, 63);
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
    n = sum_block(n, shared);
    if (threadIdx.x == 0) a.counts[block] = n;
}
// Calls f(page, whether it is counted, how many are before it) for every page of the block, of which `before` are in earlier ones; returns how many are up to
// its end.  A page is looked at before f may change its count.
template <bool LIVE_PAGES, class F>
__device__ __forceinline__ int rank_block(const PagesArgs& a, const int32_t* uses, int block, int before, int64_t* shared, F&& f)
{
    bool is[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) is[i] = counted<LIVE_PAGES>(uses, block * PAGES_BLOCK + i * 1024 + threadIdx.x, a.pages);
    const Ranks r = rank_flags(is, shared);
#pragma unroll
    for (int i = 0; i < 4; ++i) f(block * PAGES_BLOCK + i * 1024 + (int)threadIdx.x, is[i], before + r.before[i]);
    return before + r.all;
}
// The counts of up to FEW_PAGES pages in registers of one workgroup, all brought at once; rank_few as rank_block over them, f being given the count too
struct FewUses {
    int of[FEW_PAGES / 1024];
};
__device__ __forceinline__ FewUses load_few(const PagesArgs& a, const int32_t* uses)
{
    FewUses u;
#pragma unroll
    for (int i = 0; i < FEW_PAGES / 1024; ++i) {
        const int p = i * 1024 + (int)threadIdx.x;
        u.of[i] = uses[p < a.pages ? p : a.pages - 1];
    }
    return u;
}
template <bool LIVE_PAGES, class F>
__device__ __forceinline__ int rank_few(const PagesArgs& a, const FewUses& u, int64_t* shared, F&& f)
{
    int before = 0;
#pragma unroll
    for (int b = 0; b < FEW_PAGES / PAGES_BLOCK; ++b) {
        if (b >= a.page_blocks) break;
        bool is[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) is[i] = b * PAGES_BLOCK + i * 1024 + (int)threadIdx.x < a.pages && (LIVE_PAGES ? u.of[4 * b + i] != 0 : u.of[4 * b + i] == 0);
        const Ranks r = rank_flags(is, shared);
#pragma unroll
        for (int i = 0; i < 4; ++i) f(b * PAGES_BLOCK + i * 1024 + (int)threadIdx.x, is[i], before + r.before[i], u.of[4 * b + i]);
        before += r.all;
    }
    return before;
}
// what is counted in the blocks before, and in all: of counts that count_pages left
struct Counted {
    int before, all;
};
__device__ __forceinline__ Counted counted_blocks(const PagesArgs& a, int block, int64_t* shared)
{
    int mine = 0, rest = 0;
    for (int i = threadIdx.x; i < a.page_blocks; i += 1024) (i < block ? mine : rest) += a.counts[i];
    const int before = sum_block(mine, shared);
    return Counted{before, before + sum_block(rest, shared)};
}

// the lowest `wanted` free pages, in order; they are in use from here on
__device__ __forceinline__ void take_page(const PagesArgs& a, int32_t* list, int wanted, int p, bool free, int rank, int uses)
{
    if (p >= a.pages) return;
    const bool taken = free && rank < wanted;
    if (taken) list[rank] = p;
    a.uses_out[p] = taken ? 1 : uses;
}
__global__ __launch_bounds__(1024) void pages_take_kernel(PagesArgs a, const int32_t* uses)
{
    __shared__ int64_t shared[64];
    const Counted n = counted_blocks(a, blockIdx.x, shared);
    const int wanted = a.totals[WANTED];
    rank_block<false>(a, uses, blockIdx.x, n.before, shared, [&](int p, bool free, int rank) {
        if (p < a.pages) take_page(a, a.list, wanted, p, free, rank, uses[p]);
    });
    if (blockIdx.x == 0 && threadIdx.x == 0) a.totals[FREE] = n.all;
}
// by one workgroup, without the counts of another launch
__global__ __launch_bounds__(1024) void pages_take_few_kernel(PagesArgs a, const int32_t* uses)
{
    __shared__ int64_t shared[64];
    const FewUses u = load_few(a, uses);
    const int wanted = a.totals[WANTED];
    const int free = rank_few<false>(a, u, shared, [&](int p, bool is_free, int rank, int n) { take_page(a, a.list, wanted, p, is_free, rank, n); });
    if (threadIdx.x == 0) a.totals[FREE] = free;
}
// the page of rank `rank` among those taken, or -1
__device__ __forceinline__ int taken_page(const PagesArgs& a, int64_t rank, int free) { return rank < free ? a.list[rank] : -1; }

// ---- more tokens
__device__ __forceinline__ int64_t extend_rows(const PagesArgs& a, int64_t* shared)   // returns the pages that are wanted
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
    if (threadIdx.x == 0) a.starts[a.rows] = tokens < INT_MAX ? (int)tokens : INT_MAX;
    return pages;
}
// What a row had and where its new pages are: entry j is the old one below `old`, a fresh one below `now`
struct ExtendedRow {
    int length, old, now;
    int64_t base;
};
__device__ __forceinline__ ExtendedRow extended_row(const PagesArgs& a, int b)
{
    ExtendedRow r;
    r.length = a.old_length[b];
    r.old = held(a, r.length);
    r.now = held(a, a.lengths_out[b]);
    r.base = (int64_t)a.base[b] - r.old;
    return r;
}
__device__ __forceinline__ int extended_entry(const PagesArgs& a, const ExtendedRow& r, int b, int j, int free)
{
    return j < r.old ? a.table_in[b * a.ld_in + j] : j < r.now ? taken_page(a, r.base + j, free) : -1;
}
// the slot of new token t of row b
__device__ __forceinline__ int extended_slot(const PagesArgs& a, const ExtendedRow& r, int b, int64_t t, int free)
{
    const int64_t at = r.length + (t - a.starts[b]), j = at >> a.page_shift;
    const int page = j < a.width ? extended_entry(a, r, b, (int)j, free) : -1;
    return in_cache(a, page) ? (page << a.page_shift) + (int)(at & ((1 << a.page_shift) - 1)) : -1;
}
// A row's entries and its tokens' slots, by `step` threads of which this is `first`.  Row a.rows is that of the slots past the last token.
__device__ __forceinline__ void extend_row(const PagesArgs& a, int b, int free, int first, int step)
{
    if (b == a.rows) {
        for (int64_t t = (int64_t)a.starts[b] + first; t < a.tokens; t += step) a.slots[t] = -1;
        return;
    }
    const ExtendedRow r = extended_row(a, b);
    for (int j = first; j < a.width; j += step) a.table_out[b * a.ld_out + j] = extended_entry(a, r, b, j, free);
    const int64_t start = a.starts[b], end = a.starts[b + 1] < a.tokens ? a.starts[b + 1] : a.tokens;
    for (int64_t t = start + first; t < end; t += step) a.slots[t] = extended_slot(a, r, b, t, free);
}
__global__ __launch_bounds__(1024) void extend_count_kernel(PagesArgs a)
{
    __shared__ int64_t shared[64];
    if ((int)blockIdx.x < a.page_blocks) count_pages<false>(a, a.uses_in, blockIdx.x, shared);
    else {
        const int64_t pages = extend_rows(a, shared);
        if (threadIdx.x == 0) a.totals[WANTED] = pages < INT_MAX ? (int)pages : INT_MAX;
    }
}
__global__ __launch_bounds__(256) void extend_apply_kernel(PagesArgs a, int parts)
{
    for (int64_t n = blockIdx.x; n < ((int64_t)a.rows + 1) * parts; n += gridDim.x)
        extend_row(a, (int)(n / parts), a.totals[FREE], (int)(n % parts) * 256 + threadIdx.x, parts * 256);
}
// All of it by one workgroup: what the steps tell each other stays in the LDS.
__global__ __launch_bounds__(1024) void extend_few_kernel(PagesArgs a)
{
    __shared__ int64_t shared[64];
    __shared__ int32_t list[FEW_PAGES], base[FEW_ROWS], old_length[FEW_ROWS], length[FEW_ROWS], starts[FEW_ROWS + 1];
    const FewUses uses = load_few(a, a.uses_in);
    PagesArgs b = a;
    b.list = list;
    b.base = base;
    b.old_length = old_length;
    b.lengths_out = length;
    b.starts = starts;
    const int64_t pages = extend_rows(b, shared);
    const int wanted = pages < INT_MAX ? (int)pages : INT_MAX;
    const int free = rank_few<false>(a, uses, shared, [&](int p, bool is_free, int rank, int n) { take_page(a, list, wanted, p, is_free, rank, n); });
    __syncthreads();
    for (int i = threadIdx.x; i <= a.rows; i += 1024) {
        if (i < a.rows) a.lengths_out[i] = length[i];
        a.starts[i] = starts[i];
    }
    // four entries at a time, whose loads travel together, whatever rows they are of
    const int entries = a.rows * a.width, all = entries + (int)a.tokens;     // (FEW_ENTRIES at most)
    for (int e0 = threadIdx.x; e0 < all; e0 += 4096) {
        int x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int e = e0 + k * 1024;
            x[k] = -1;
            if (e < entries) {
                const int row = (unsigned)e / (unsigned)a.width;
                x[k] = extended_entry(b, extended_row(b, row), row, e - row * a.width, free);
            } else if (e < all && e - entries < starts[a.rows]) {
                int low = 0, high = a.rows;                // starts[low] <= t < starts[high]
                while (high - low > 1) {
                    const int mid = (low + high) / 2;
                    if (starts[mid] <= e - entries) low = mid;
                    else high = mid;
                }
                x[k] = extended_slot(b, extended_row(b, low), low, e - entries, free);
            }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int e = e0 + k * 1024;
            if (e < entries) {
                const int row = (unsigned)e / (unsigned)a.width;
                a.table_out[row * a.ld_out + e - row * a.width] = x[k];
            } else if (e < all) {
                a.slots[e - entries] = x[k];
            }
        }
    }
}

// ---- sequences that continue others
//
// A row's children and the lowest of them; what every child wants of fresh pages (its open page, where it is not the lowest).
__device__ __forceinline__ int load_shared(const int32_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ bool has_parent(const PagesArgs& a, int parent) { return (unsigned)parent < (unsigned)a.rows_in; }
__device__ __forceinline__ void fork_children(const PagesArgs& a, int* first, int* children)   // of one workgroup, in the LDS
{
    for (int b = threadIdx.x; b < a.rows_in; b += 1024) {
        first[b] = INT_MAX;
        children[b] = 0;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.rows; i += 1024) {
        const int parent = a.which[i];
        if (!has_parent(a, parent)) continue;
        atomicMin(first + parent, i);
        atomicAdd(children + parent, 1);
    }
    __syncthreads();
}
// the new lengths, and what every child wants: its rank among those that want a page, or -1.  Returns how many do.
template <class First>
__device__ __forceinline__ int fork_wants(const PagesArgs& a, First&& first, int64_t* shared)
{
    int wanted = 0;
    for (int i0 = 0; i0 < a.rows; i0 += 4096) {
        bool need[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int i = i0 + k * 1024 + (int)threadIdx.x;
            need[k] = false;
            if (i >= a.rows) continue;
            const int parent = a.which[i];
            const int length = has_parent(a, parent) && a.lengths_in[parent] > 0 ? a.lengths_in[parent] : 0, j = open_entry(a, length);
            a.lengths_out[i] = length;
            need[k] = j >= 0 && first(parent) != i && in_cache(a, a.table_in[parent * a.ld_in + j]);
        }
        const Ranks r = rank_flags(need, shared);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int i = i0 + k * 1024 + (int)threadIdx.x;
            if (i < a.rows) a.base[i] = need[k] ? wanted + r.before[k] : -1;
        }
        wanted += r.all;
    }
    return wanted;
}
__global__ __launch_bounds__(1024) void fork_count_kernel(PagesArgs a)
{
    __shared__ int64_t shared[64];
    __shared__ int first[FEW_ROWS], children[FEW_ROWS];
    if (blockIdx.x) {                                      // the counts, to be changed
        for (int64_t p = (int64_t)(blockIdx.x - 1) * 1024 + threadIdx.x; p < a.pages; p += (int64_t)(gridDim.x - 1) * 1024) a.uses_out[p] = a.uses_in[p];
        return;
    }
    int wanted;
    if (a.rows_in <= FEW_ROWS) {
        fork_children(a, first, children);
        for (int b = threadIdx.x; b < a.rows_in; b += 1024) a.children[b] = children[b];
        wanted = fork_wants(a, [&](int b) __attribute__((always_inline)) { return first[b]; }, shared);
    } else {
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
        wanted = fork_wants(a, [&](int b) __attribute__((always_inline)) { return load_shared(a.first + b); }, shared);
    }
    if (threadIdx.x == 0) a.totals[WANTED] = wanted;
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
    __shared__ int64_t shared[64];
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
        const int parent = a.which[i], j = open_entry(a, a.lengths_in[parent]), to = taken_page(a, rank, a.totals[FREE]);
        if (part == 0 && threadIdx.x == 0) a.table_out[i * a.ld_out + j] = to;
        if (to >= 0) copy_piece(a, a.table_in[parent * a.ld_in + j], to, part);
    }
}

// All but the copies by one workgroup, with the counts and the rows' children in the LDS.
__global__ __launch_bounds__(1024) void fork_few_kernel(PagesArgs a)
{
    __shared__ int64_t shared[64];
    __shared__ int uses[FEW_PAGES], first[FEW_ROWS], children[FEW_ROWS];
    for (int p = threadIdx.x; p < a.pages; p += 1024) uses[p] = a.uses_in[p];
    fork_children(a, first, children);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int b = wave; b < a.rows_in; b += 16) {           // (as fork_table_kernel)
        const int length = a.lengths_in[b], n = held(a, length), open = open_entry(a, length), named = children[b];
        for (int j = lane; j < n; j += 64) {
            const int page = a.table_in[b * a.ld_in + j], change = (j == open && named > 1 ? 1 : named) - 1;
            if (change && in_cache(a, page)) atomicAdd(uses + page, change);
        }
    }
    for (int i = wave; i < a.rows; i += 16) {
        const int parent = a.which[i], n = has_parent(a, parent) ? held(a, a.lengths_in[parent]) : 0;
        for (int j = lane; j < a.width; j += 64) a.table_out[i * a.ld_out + j] = j < n ? a.table_in[parent * a.ld_in + j] : -1;
    }
    const int wanted = fork_wants(a, [&](int b) __attribute__((always_inline)) { return first[b]; }, shared);
    __syncthreads();
    int free = 0;
    for (int block = 0; block < a.page_blocks; ++block)
        free = rank_block<false>(a, uses, block, free, shared, [&](int p, bool is_free, int rank) {
            if (p < a.pages) take_page(a, a.list, wanted, p, is_free, rank, uses[p]);
        });
    if (threadIdx.x == 0) a.totals[FREE] = free;
}

// ---- pages in use to the front
//
// With n of them: those from n on have ranks totals[LIVE_BELOW] and up among the pages in use, and as many pages below n are free; the i-th goes to the i-th.
__global__ __launch_bounds__(1024) void compact_count_kernel(PagesArgs a)
{
    __shared__ int64_t shared[64];
    count_pages<true>(a, a.uses_in, blockIdx.x, shared);
}
__device__ __forceinline__ void place_page(const PagesArgs& a, int total, int p, bool live, int rank, int uses)   // of `total` pages in use
{
    if (p == total || (p == a.pages - 1 && total == a.pages)) {
        a.totals[LIVE_BELOW] = p == total ? rank : total;
        a.totals[LIVE] = total;
    }
    if (p >= a.pages) return;
    if (p < total) {
        if (live) a.uses_out[p] = uses;
        else a.list[p - rank] = p;                         // (its count comes with the page that moves here)
    } else {
        a.rank[p] = live ? rank : -1;
        a.uses_out[p] = 0;
        if (live) {
            a.source[rank] = p;
            a.moved[rank] = uses;
        }
    }
}
__global__ __launch_bounds__(1024) void compact_rank_kernel(PagesArgs a)
{
    __shared__ int64_t shared[64];
    const Counted n = counted_blocks(a, blockIdx.x, shared);
    rank_block<true>(a, a.uses_in, blockIdx.x, n.before, shared, [&](int p, bool live, int rank) { place_page(a, n.all, p, live, rank, p < a.pages ? a.uses_in[p] : 0); });
}
// by one workgroup, without the counts of another launch
__global__ __launch_bounds__(1024) void compact_few_kernel(PagesArgs a)
{
    __shared__ int64_t shared[64];
    const FewUses uses = load_few(a, a.uses_in);
    int n = 0;
#pragma unroll
    for (int i = 0; i < FEW_PAGES / 1024; ++i) n += i * 1024 + (int)threadIdx.x < a.pages && uses.of[i] != 0;
    const int total = sum_block(n, shared);
    rank_few<true>(a, uses, shared, [&](int p, bool live, int rank, int count) { place_page(a, total, p, live, rank, count); });
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
// Checks what the three calls have in common and fills in a.  in_place: tables and lengths may be the same.  lengths: they are needed.  which: counts or
// parents, one for each row of out, if the call has such; kernels read them again when they have written rows of out, so that they may not be part of it.
// more: what else the call writes.
int begin(PagesArgs& a, const shflbw_kv_cache* c, const shflbw_kv_pages* in, const shflbw_kv_pages* out, bool in_place, bool lengths, const int32_t* which,
          const Span (&more)[2], void* workspace, int64_t workspace_bytes)
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
    const Span chosen = {which, which ? out->sequences : 0};
    for (int i = 0; i < 3; ++i) {
        if (overlap(to[i], chosen)) return fail(SHFLBW_ERR_BAD_SHAPE, "arrays of out overlap counts or parents");
        for (const Span& x : more)
            if (overlap(x, from[i]) || overlap(x, to[i]) || overlap(x, chosen)) return fail(SHFLBW_ERR_BAD_SHAPE, "slots or starts overlap another array");
    }
    if (overlap(more[0], more[1])) return fail(SHFLBW_ERR_BAD_SHAPE, "slots and starts overlap");
    const int64_t sequences = in->sequences > out->sequences ? in->sequences : out->sequences, work = workspace_bytes_of(c->pages, sequences);
    if (!workspace || workspace_bytes < work) return fail(SHFLBW_ERR_NULL_ARG, "the call needs a workspace of %lld bytes", (long long)work);
    if (reinterpret_cast<uintptr_t>(workspace) % 16) return fail(SHFLBW_ERR_BAD_SHAPE, "the workspace must be 16-byte aligned");
    const int64_t page_bytes = page_head_bytes(c->page_tokens, c->head_dim) * c->heads;
    const Span own[2] = {{workspace, work / 4}, {c->data, c->pages * page_bytes / 4}};
    if (overlap(own[0], own[1])) return fail(SHFLBW_ERR_BAD_SHAPE, "the workspace overlaps the cache");
    for (const Span& x : own) {
        bool any = overlap(x, chosen) || overlap(x, more[0]) || overlap(x, more[1]);
        for (int i = 0; i < 3; ++i) any |= overlap(x, from[i]) || overlap(x, to[i]);
        if (any) return fail(SHFLBW_ERR_BAD_SHAPE, "an array overlaps the workspace or the cache");
    }
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
    a.page_bytes = page_bytes;
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
    if (tokens < 0 || tokens > INT_MAX) return fail(SHFLBW_ERR_BAD_SHAPE, "tokens must be 0 to 2^31 - 1");
    const int rc = begin(a, cache, in, out, true, true, counts, {{slots, tokens}, {starts, out ? out->sequences + 1LL : 0}}, workspace, workspace_bytes);
    if (rc < 0) return rc;
    if (!starts || (tokens && !slots) || (a.rows && !counts)) return fail(SHFLBW_ERR_NULL_ARG, "counts, slots and starts must not be NULL");
    a.which = counts;
    a.slots = slots;
    a.starts = starts;
    a.tokens = tokens;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (a.pages <= FEW_PAGES && a.rows <= FEW_ROWS && (int64_t)a.rows * a.width + tokens <= FEW_ENTRIES) {
        hipLaunchKernelGGL(extend_few_kernel, dim3(1), dim3(1024), 0, st, a);
        return launched();
    }
    hipLaunchKernelGGL(extend_count_kernel, dim3(a.page_blocks + 1), dim3(1024), 0, st, a);
    hipLaunchKernelGGL(pages_take_kernel, dim3(a.page_blocks), dim3(1024), 0, st, a, a.uses_in);
    // workgroups to a row, for 1024 of its entries and slots each
    const int parts = (int)few_blocks(ceil_div((int64_t)a.rows * a.width + tokens, ((int64_t)a.rows + 1) * 1024));
    hipLaunchKernelGGL(extend_apply_kernel, dim3(few_blocks(((int64_t)a.rows + 1) * parts)), dim3(256), 0, st, a, parts);
    return launched();
}

int shflbw_kv_fork(const shflbw_kv_cache* cache, const shflbw_kv_pages* in, const shflbw_kv_pages* out, const int32_t* parents, void* workspace,
                   int64_t workspace_bytes, void* stream)
{
    using namespace shflbw;
    PagesArgs a = {};
    const int rc = begin(a, cache, in, out, false, true, parents, {}, workspace, workspace_bytes);
    if (rc < 0) return rc;
    if (a.rows && !parents) return fail(SHFLBW_ERR_NULL_ARG, "parents must not be NULL");
    a.which = parents;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const int parts = (int)ceil_div(a.page_bytes, COPY_BYTES);
    if (a.pages <= FEW_PAGES && a.rows_in <= FEW_ROWS && ((int64_t)a.rows_in + a.rows) * a.width <= FEW_ENTRIES) {
        hipLaunchKernelGGL(fork_few_kernel, dim3(1), dim3(1024), 0, st, a);
        hipLaunchKernelGGL(fork_copy_kernel, dim3(few_blocks((int64_t)a.rows * parts)), dim3(256), 0, st, a, parts);
        return launched();
    }
    hipLaunchKernelGGL(fork_count_kernel, dim3(a.uses_in == a.uses_out ? 1 : 1 + few_blocks(ceil_div(a.pages, 1024))), dim3(1024), 0, st, a);
    hipLaunchKernelGGL(fork_table_kernel, dim3(few_blocks(ceil_div(((int64_t)a.rows_in + a.rows) * a.width, 256))), dim3(256), 0, st, a);
    if (a.pages <= FEW_PAGES) {
        hipLaunchKernelGGL(pages_take_few_kernel, dim3(1), dim3(1024), 0, st, a, a.uses_out);
    } else {
        hipLaunchKernelGGL(pages_count_kernel, dim3(a.page_blocks), dim3(1024), 0, st, a);
        hipLaunchKernelGGL(pages_take_kernel, dim3(a.page_blocks), dim3(1024), 0, st, a, a.uses_out);
    }
    hipLaunchKernelGGL(fork_copy_kernel, dim3(few_blocks((int64_t)a.rows * parts)), dim3(256), 0, st, a, parts);
    return launched();
}

int shflbw_kv_compact(const shflbw_kv_cache* cache, const shflbw_kv_pages* in, const shflbw_kv_pages* out, void* workspace, int64_t workspace_bytes,
                      void* stream)
{
    using namespace shflbw;
    PagesArgs a = {};
    const int rc = begin(a, cache, in, out, true, false, nullptr, {}, workspace, workspace_bytes);
    if (rc < 0) return rc;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const int parts = (int)ceil_div(a.page_bytes, COPY_BYTES), table_blocks = (int)few_blocks(ceil_div((int64_t)a.rows * a.width, 256));
    // at most half of the pages move
    const unsigned copy_blocks = few_blocks((int64_t)(a.pages / 2) * parts);
    if (a.pages <= FEW_PAGES) {
        hipLaunchKernelGGL(compact_few_kernel, dim3(1), dim3(1024), 0, st, a);
    } else {
        hipLaunchKernelGGL(compact_count_kernel, dim3(a.page_blocks), dim3(1024), 0, st, a);
        hipLaunchKernelGGL(compact_rank_kernel, dim3(a.page_blocks), dim3(1024), 0, st, a);
    }
    hipLaunchKernelGGL(compact_apply_kernel, dim3(table_blocks + copy_blocks), dim3(256), 0, st, a, parts, table_blocks);
    return launched();
}

}  // extern "C"
