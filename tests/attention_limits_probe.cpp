// What the plans of attention calls say, for tests/test_attention_limits.py.
#include "attention.h"

using namespace shflbw;

// wavefronts per workgroup, whether the form for fewer than 64 columns, blocks of columns; returns whether there is such a kernel
extern "C" int probe_prompt_kernel(int sequences, int heads, int group, int D, long max_tokens, int window, int sinks, long tokens, int* out)
{
    const AttnPlan p = plan_prompt(sequences, heads, group, D, max_tokens, window, sinks, tokens);
    out[0] = p.waves;
    out[1] = p.tiny;
    out[2] = p.col_blocks;
    return !p.decode && tile_kernel_exists(D, false, p.waves, p.tiny);
}
// blocks of columns, workgroups and whether the kernel for few queries
extern "C" void probe_cache_blocks(int batch, int heads, int group, int D, long tokens, int max_queries, long max_length, long* out)
{
    const AttnPlan p = plan_cache_attention(batch, heads, group, D, tokens, max_queries, max_length, INT32_MAX, 0);
    out[0] = p.col_blocks;
    out[1] = (long)p.groups;
    out[2] = p.decode;
}
