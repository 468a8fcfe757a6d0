// What kernel a prompt's plan names, for tests/test_attention_limits.py.
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
