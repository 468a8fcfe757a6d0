// How a call of the attention operators is cut into workgroups.  Host code without HIP.
#include "attention.h"

#include <algorithm>

namespace shflbw {
namespace {

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Keys that the queries of one workgroup see at most
int64_t keys_seen(int64_t max_length, int window, int sinks, int64_t queries)
{
    if (window == INT32_MAX) return max_length;
    return std::min<int64_t>(max_length, (int64_t)window + sinks + queries);
}

// Wavefronts of the tile kernel's workgroups: 8 share what they bring to the LDS, 4 where that leaves CUs without work
void tile_shape(AttnPlan& p, int64_t items, int64_t pairs)
{
    p.waves = ceil_div(items, 8) * pairs >= 256 ? 8 : 4;
    p.col_blocks = (int)ceil_div(items, p.waves);
}

}  // namespace

AttnPlan plan_cache_attention(int batch, int heads, int group, int D, int64_t tokens, int max_queries, int64_t max_length, int window, int sinks)
{
    AttnPlan p = {};
    const int64_t columns = (int64_t)group * max_queries;
    p.decode = columns <= 64;
    const int tile = p.decode ? ATTN_DECODE_KEYS : ATTN_TILE_KEYS;
    if (p.decode) {
        p.col_tiles = (int)ceil_div(columns, 16);
        p.col_blocks = 1;
    } else {
        const int64_t items = ceil_div(max_queries, ATTN_TILE_QUERIES) * group;
        tile_shape(p, items, (int64_t)batch * heads);
    }
    const int64_t base = (int64_t)batch * heads * p.col_blocks;
    // tiles of the longest sequence: window and sinks each may begin inside a tile
    const int64_t tiles = keys_seen(max_length, window, sinks, max_queries) / tile + 3;
    // enough workgroups for two on each of 256 CUs, but no part under 8 tiles (decoding: one per wavefront)
    int64_t splits = std::min(ceil_div(512, std::max<int64_t>(base, 1)), std::max<int64_t>(tiles / 8, 1));
    p.split_tiles = (int)ceil_div(tiles, splits);
    p.splits = (int)ceil_div(tiles, p.split_tiles);
    p.groups = base * p.splits;
    p.workspace = p.splits > 1 ? (int64_t)p.splits * heads * group * tokens * (D + 2) * 4 : 0;
    return p;
}

AttnPlan plan_prompt(int sequences, int heads, int group, int64_t max_tokens)
{
    AttnPlan p = {};
    const int64_t items = ceil_div(max_tokens, ATTN_TILE_QUERIES) * group;
    tile_shape(p, items, (int64_t)sequences * heads);
    p.splits = 1;
    p.split_tiles = INT32_MAX;
    p.groups = (int64_t)sequences * heads * p.col_blocks;
    return p;
}

}  // namespace shflbw
