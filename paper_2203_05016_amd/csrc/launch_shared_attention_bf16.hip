// Launchers of attention over shared prefixes for bfloat16 operands.
#define SHFLBW_LAUNCH_BF true
#define SHFLBW_LAUNCH_SHARED run_shared_attention_bf16
#include "launch_attention.inc"
