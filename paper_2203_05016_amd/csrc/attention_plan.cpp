// How a call of the attention operators is cut into workgroups.  Host code without HIP.
#include "attention.h"

#include <algorithm>

namespace shflbw {
namespace {

constexpr int CUS = 256;

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// a * b, or INT64_MAX where that is too much: more workgroups than any grid has
int64_t product(int64_t a, int64_t b)
{
    int64_t x;
    return __builtin_mul_overflow(a, b, &x) ? INT64_MAX : x;
}

// Keys that the queries of one workgroup see at most
int64_t keys_seen(int64_t max_length, int window, int sinks, int64_t queries)
{
    if (window == INT32_MAX) return max_length;
    return std::min<int64_t>(max_length, (int64_t)window + sinks + queries);
}

}  // namespace

AttnPlan plan_cache_attention(int batch, int heads, int group, int D, int64_t tokens, int max_queries, int64_t max_length, int window, int sinks)
{
    AttnPlan p = {};
    // no sequence has more queries than there are columns, whatever the caller's bound
    max_queries = (int)std::max<int64_t>(1, std::min<int64_t>(max_queries, tokens));
    const int64_t pairs = (int64_t)batch * heads, columns = (int64_t)group * max_queries;
    int64_t col_blocks = 1;
    // The kernel for few queries up to 64 columns (8 sequences of 4000 keys, 8 queries of 64 heads over 8 of 128: 27 us, in tiles of queries 42;
    // 24 of up to 3001, 5 queries: 34 and 100), and up to 128 in blocks of 32, each of which reads the cache, while the GPU holds them: 16
    // queries of the same heads over 3000 keys, 16 sequences 47 us and 60, 64 of them over 1000 keys 103 and 74.
    const bool cuts = group <= 32;                 // blocks are of whole queries
    const int64_t blocks_of_32 = cuts ? ceil_div(max_queries, 32 / group) : 1;
    p.decode = columns <= 64 || (cuts && columns <= 128 && pairs * blocks_of_32 <= 2 * CUS);
    int64_t slots, least;   // workgroups the GPU holds at a time, and tiles that a part is worth
    if (p.decode) {
        p.col_tiles = (int)ceil_div(columns, 16);
        // 64 columns leave one wavefront per SIMD (D = 128): two blocks of 32, of whole queries, read the cache twice and are faster.  16
        // sequences of 3000 keys on average, 8 queries of 64 heads over 8 of 128: 48 -> 35 us; 32 of them 66 -> 54; of 64 features
        // 28 -> 24; but 24 of 2100, 5 queries, in 48 columns 34 and in two blocks 41.
        if (p.col_tiles >= 4 && cuts) {
            p.col_tiles = 2;
            col_blocks = blocks_of_32;
        }
        // Workgroups of 8 wavefronts while all of them are on the GPU at a time, of 4 beyond: 64 sequences of 2500 keys on average, 8 heads
        // of 128: 40 us with 8, 44 with 4; 128 of 1028, 16 heads of 64: 35 and 29.
        const int residency = decode_residency(p.col_tiles, D);
        p.waves = residency > 1 && pairs * col_blocks <= CUS * (residency / 2) ? 8 : 4;
        slots = p.waves == 8 ? CUS * (residency / 2) : CUS * residency;
        least = 4 * p.waves;
    } else {
        const int64_t items = ceil_div(max_queries, ATTN_TILE_QUERIES) * group;
        // 8 wavefronts share what they bring; 4 where there are no more items (4 sequences of up to 9000 keys, 1024 queries, 32 heads over 8 of
        // 96 410 us with 8, 428 with 4)
        p.waves = items > 4 ? 8 : 4;
        col_blocks = ceil_div(items, p.waves);
        slots = p.waves == 4 && D < 128 ? 2 * CUS : CUS;   // what the LDS holds of three tiles
        least = 4;   // 633 queries of 1 sequence of 1222 keys, 4 heads of 128: 25 us in parts of 4 tiles, 31 of 8
    }
    const int tile = p.decode ? ATTN_DECODE_KEYS : ATTN_TILE_KEYS;
    const int64_t base = product(pairs, col_blocks);
    // tiles of the longest sequence: window and sinks each may begin inside a tile
    const int64_t tiles = keys_seen(max_length, window, sinks, max_queries) / tile + 3;
    // One cut for all sequences, by max_length.  Where that is the table's capacity, parts past a sequence's keys have no work: one of 30000 keys, 64
    // heads over 8 of 128, 16.3 us cut by its length and 24.6 by a table of 131072; 16 of 3000 on average 20.1 and 30.7 by one of 32768.
    // Keys are cut into parts where workgroups are few, into as many as fill the GPU once (what is left over costs a whole round: 24
    // sequences of 3000 keys, 8 heads of 128, 5 queries of 64 heads 48 us in 3 parts of 4 wavefronts, 41 in 2).  The join takes 4
    // to 5 us, so parts are not worth it under twice their least length.
    int64_t splits = base > 0 && tiles >= 2 * least ? std::min(slots / base, tiles / least) : 1;
    splits = std::max<int64_t>(splits, 1);
    p.split_tiles = (int)ceil_div(tiles, splits);
    p.splits = (int)ceil_div(tiles, p.split_tiles);
    p.groups = product(base, p.splits);
    p.col_blocks = (int)std::min<int64_t>(col_blocks, INT32_MAX);   // (more are more groups than a launch takes)
    p.workspace = p.splits > 1 ? (int64_t)p.splits * heads * group * tokens * (D + 2) * 4 : 0;
    return p;
}

AttnPlan plan_prompt(int sequences, int heads, int group, int D, int64_t max_tokens, int window, int sinks, int64_t tokens)
{
    AttnPlan p = {};
    p.tiny = tokens < ATTN_TILE_KEYS;    // whole tiles of keys would reach past the rows
    const int64_t items = ceil_div(max_tokens, ATTN_TILE_QUERIES) * group, pairs = (int64_t)sequences * heads;
    // Workgroups of 8 wavefronts share what they bring to the LDS; of 4 where 8 leave CUs without work, for heads of 64 (tile_residency), and
    // for heads of 96, of which a CU holds two, where their keys are few: 8 prompts of 4096, 8 heads, windows of 64, 512 and 1024 61, 99 and 147 us
    // in these, 70, 114 and 152 in workgroups of 8; without a window, 4 of up to 4096, 32 over 8 heads, 487 and 452 (the bound of 1536 keys lies between).
    const bool few_keys = keys_seen(max_tokens, window, sinks, 0) < 1536;
    // Fewer than 64 columns: in workgroups of 4.
    p.waves = !p.tiny && D > 64 && !(D == 96 && few_keys) && product(ceil_div(items, 8), pairs) >= CUS ? 8 : 4;
    const int64_t col_blocks = ceil_div(items, p.waves);
    p.col_blocks = (int)std::min<int64_t>(col_blocks, INT32_MAX);
    p.splits = 1;
    p.split_tiles = INT32_MAX;
    p.groups = product(pairs, col_blocks);
    return p;
}

}  // namespace shflbw
