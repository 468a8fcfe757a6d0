// Attention launchers for bfloat16 operands.
#define SHFLBW_LAUNCH_BF true
#define SHFLBW_LAUNCH_NAME run_attention_bf16
#include "launch_attention.inc"
