// How attention is cut into workgroups and how the cache lies in memory, for tests/test_attention_plan.py.
#include "attention.h"

using namespace shflbw;

namespace {
void put(const AttnPlan& p, long* out)
{
    const long all[] = {p.decode, p.col_tiles, p.waves, p.col_blocks, p.splits, p.split_tiles, (long)p.groups, (long)p.workspace};
    for (int i = 0; i < 8; ++i) out[i] = all[i];
}
}  // namespace

extern "C" void probe_cache_plan(int batch, int heads, int group, int D, long tokens, int max_queries, long max_length, int window, int sinks, long* out)
{
    put(plan_cache_attention(batch, heads, group, D, tokens, max_queries, max_length, window, sinks), out);
}
extern "C" void probe_prompt_plan(int sequences, int heads, int group, int D, long max_tokens, int window, int sinks, long* out)
{
    put(plan_prompt(sequences, heads, group, D, max_tokens, window, sinks), out);
}
extern "C" int probe_place(int block, int pairs, int heads, int per_pair, int* inner)
{
    const AttnPlace at = attn_place(block, pairs, heads, per_pair);
    *inner = at.inner;
    return at.pair;
}
// byte of the first of a token's words of q, of keys (0) or values (1), from the codes' start; bytes of a head in a page
extern "C" int probe_code(int D, int token, int q, int values) { return code_offset(D, token, values ? value_lane(token, q) : key_lane(token, q)); }
extern "C" long probe_head_bytes(int page, int D) { return (long)page_head_bytes(page, D); }
