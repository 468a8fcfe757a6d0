// Launchers of attention over shared prefixes for binary16 operands.
#define SHFLBW_LAUNCH_BF false
#define SHFLBW_LAUNCH_SHARED run_shared_attention_f16
#include "launch_attention.inc"
