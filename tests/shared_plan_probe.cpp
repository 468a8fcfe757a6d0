// How attention over shared prefixes is cut into workgroups, for tests/test_shared_plan.py.
#include "attention.h"

using namespace shflbw;

namespace {
long* put(const AttnPlan& p, long* out)
{
    const long all[] = {p.decode, p.col_tiles, p.waves, p.col_blocks, p.splits, p.split_tiles, (long)p.groups, p.tiny};
    for (long x : all) *out++ = x;
    return out;
}
}  // namespace

// both parts, whether both are one call, whether the own part's kernel joins, and the workspace
extern "C" void probe_shared_plan(int prefixes, long max_sharing, long max_prefix, int batch, int heads, int group, int D, long tokens, int max_queries, long max_length,
                                  int keys_fit, long* out)
{
    const SharedPlan p = plan_shared_attention(prefixes, max_sharing, max_prefix, batch, heads, group, D, tokens, max_queries, max_length, keys_fit != 0);
    out = put(p.own, put(p.prefix, out));
    *out++ = p.behind;
    *out++ = p.joins;
    *out++ = (long)p.workspace;
}
extern "C" int probe_most_joined() { return ATTN_JOINED; }
