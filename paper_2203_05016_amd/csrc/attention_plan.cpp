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

// The keys' cut into parts: of `base` workgroups, `slots` of which the GPU holds, each part worth `least` tiles or more
void cut(AttnPlan& p, int64_t base, int64_t slots, int64_t least, int64_t tiles)
{
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
}

// The tile kernel over the cache, for `items` of each of `pairs`, that see up to `keys`
AttnPlan plan_tiles(int64_t pairs, int64_t items, int D, int64_t keys)
{
    AttnPlan p = {};
    // 8 wavefronts share what they bring; 4 where there are no more items (4 sequences of up to 9000 keys, 1024 queries, 32 heads over 8 of
    // 96 410 us with 8, 428 with 4)
    p.waves = items > 4 ? 8 : 4;
    const int64_t col_blocks = ceil_div(items, p.waves);
    // (parts of 4 tiles: 633 queries of 1 sequence of 1222 keys, 4 heads of 128: 25 us in parts of 4 tiles, 31 of 8)
    cut(p, product(pairs, col_blocks), p.waves == 4 && D < 128 ? 2 * CUS : CUS /* what the LDS holds of three tiles */, 4, keys / ATTN_TILE_KEYS + 3);
    p.col_blocks = (int)std::min<int64_t>(col_blocks, INT32_MAX);   // (more are more groups than a launch takes)
    return p;
}

// The prefixes' part: max_sharing queries of each of `pairs`, all of which see all `keys`.  Up to 192 columns by the kernel for few queries in blocks of 32
// (64 heads over 8 of 128, one prefix of 8000: 24 sequences 30.4 us, in tiles of queries 37.6; 16 prefixes of 3000 with 24 each 99 and 100), up to 256
// while the GPU holds the blocks (32: 30.3 and 40.7; 16 prefixes with 32 each 132 and 108); blocks of 48 where these are fewer by a fourth and the GPU is
// full (16 prefixes with 12 sequences each 59 us, in blocks of 32 66; with 16 81 and 71; one prefix with 12 30.0 and 25.7).
AttnPlan plan_prefix(int64_t pairs, int group, int D, int64_t max_sharing, int64_t keys)
{
    AttnPlan p = {};
    const int64_t columns = product(max_sharing, group);
    const int64_t twos = ceil_div(columns, 32), threes = ceil_div(columns, 48);
    if (group > 32 || columns > 256 || (columns > 192 && product(pairs, twos) > CUS)) return plan_tiles(pairs, ceil_div(columns, ATTN_TILE_QUERIES), D, keys);
    p.decode = true;
    p.col_tiles = columns <= 16 ? 1 : pairs * twos >= CUS && 4 * threes < 3 * twos ? 3 : 2;
    const int64_t col_blocks = ceil_div(max_sharing, 16 * p.col_tiles / group);
    const int residency = decode_residency(p.col_tiles, D);
    p.waves = residency > 1 && pairs * col_blocks <= CUS * (residency / 2) ? 8 : 4;
    cut(p, product(pairs, col_blocks), p.waves == 8 ? CUS * (residency / 2) : CUS * residency, 4 * p.waves, keys / ATTN_DECODE_KEYS + 3);
    p.col_blocks = (int)col_blocks;
    return p;
}

// Items of 32 queries of a head that `tokens` queries of `batch` sequences may be more than they would be in sequences of max_queries (2 or more) each: at most so
// many have max_queries that every other still has one
double uneven_items(int64_t batch, int64_t tokens, int64_t max_queries)
{
    const int64_t sequences = std::min(batch, tokens), items = ceil_div(max_queries, ATTN_TILE_QUERIES);
    const int64_t whole = std::min((tokens - sequences) / (max_queries - 1), sequences);
    return (double)(whole * items + sequences - whole) - (double)tokens / (double)max_queries * (double)items;
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
    // keys that the queries of one workgroup see: window and sinks each may begin inside a tile
    const int64_t keys = keys_seen(max_length, window, sinks, max_queries);
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
        const int64_t slots = p.waves == 8 ? CUS * (residency / 2) : CUS * residency;
        cut(p, product(pairs, col_blocks), slots, 4 * p.waves, keys / ATTN_DECODE_KEYS + 3);
        p.col_blocks = (int)std::min<int64_t>(col_blocks, INT32_MAX);
    } else {
        p = plan_tiles(pairs, ceil_div(max_queries, ATTN_TILE_QUERIES) * group, D, keys);
    }
    p.workspace = p.splits > 1 ? (int64_t)p.splits * heads * group * tokens * (D + 2) * 4 : 0;
    return p;
}

SharedPlan plan_shared_attention(int prefixes, int64_t max_sharing, int64_t max_prefix, int batch, int heads, int group, int D, int64_t tokens, int max_queries,
                                 int64_t max_length, bool keys_fit)
{
    SharedPlan p = {};
    max_queries = (int)std::max<int64_t>(1, std::min<int64_t>(max_queries, tokens));
    max_sharing = std::max<int64_t>(1, std::min<int64_t>(max_sharing, tokens));
    const auto parts = [&](int64_t n) { return product(n * (D + 2) * 4, (int64_t)heads * group * tokens); };
    // From 20 queries on, sequence by sequence: a prefix's parts, in 32 bits, are then more than its keys.  32 sequences behind 4096 tokens, 64 heads over 8 of
    // 128: 16 queries 137 us, prefix and own apart 116; 20 131 and 151, 32 129 and 180, 33 240 and 292; 8 of 512 504 and 752.
    // Sequences of few queries among those of many are items of 32 columns there that read their prefix for a few: not where, for all that the host knows (every sequence
    // has a query, and as many as can have the most), such items are so many that their keys come to over 75 for each column of q.  With prefix
    // and own apart, then without, 64 heads over 8 of 128, one prefix of 8001 tokens: 63 sequences of 1 query and one of 512 (849 keys a column) 375 us and 1910, 56 and
    // 8 of 512 (104) 1521 and 2359, 15 and one of 512 (220) 285 and 631; behind 1000 tokens 63 and one (106) 204 and 362, but 56 and 8 (13) 577 and 468; behind 200, 60 and
    // 4 of 200 (14) 120 and 89; 32 over 8 of 96 behind 4096, 31 and one of 1024 (116) 215 and 518.  What the
    // host does not know costs less: if the 56 others have none 1233 and 988; 32 of 10 and 32 of 30 queries (133) 525 and 480.
    // And few queries where reading the prefix again for every sequence, from the L2s, is less than parts and another launch: up to 2^27 values (bytes, as
    // the cache has them, are 17/32 of that).  64 heads over 8 of 128: 8 sequences behind 500 tokens 8.5 us and 18.8 apart, 32 behind 1000 12.0 and 22.7, behind 2000
    // (131 million) 20.7 and 23.6; 32 over 8 of 96, 8 prefixes of 3000 with 4 each (147 million) 20.2 and 18.0.
    const bool many = max_queries >= 20 && uneven_items(batch, tokens, max_queries) * (double)max_prefix <= 75.0 * (double)tokens;
    const int64_t again = product((int64_t)batch * heads * 2 * D, max_prefix);
    p.behind = keys_fit && (many || (max_queries < 20 && (int64_t)group * max_queries <= 64 && again <= 1LL << 27));
    if (p.behind) {
        const int64_t keys = max_prefix + ATTN_TILE_KEYS + max_length;
        p.own = many ? plan_tiles((int64_t)batch * heads, ceil_div(max_queries, ATTN_TILE_QUERIES) * group, D, keys)
                     : plan_cache_attention(batch, heads, group, D, tokens, max_queries, keys, INT32_MAX, 0);
        p.workspace = p.own.splits > 1 ? parts(p.own.splits) : 0;
        return p;
    }
    p.prefix = plan_prefix((int64_t)prefixes * heads, group, D, max_sharing, max_prefix);
    p.own = plan_cache_attention(batch, heads, group, D, tokens, max_queries, max_length, INT32_MAX, 0);
    // The kernel for few queries joins the prefixes' parts with what it finds, if there are no parts of its own keys: 64 sequences, 64 heads over 8 of 128, 16 parts
    // 46 us, by a kernel of its own 55; 8 with 32 parts 28.2 and 30.1; 128 of 32 over 8 of 96 27 and 33; 8 queries of each of 64 113 and 115.
    p.joins = p.own.decode && p.own.splits == 1 && p.prefix.splits <= ATTN_JOINED;
    p.workspace = parts((int64_t)p.prefix.splits + (p.joins ? 0 : p.own.splits));
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
