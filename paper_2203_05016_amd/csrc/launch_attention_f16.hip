// Attention launchers for binary16 operands.
#define SHFLBW_LAUNCH_BF false
#define SHFLBW_LAUNCH_NAME run_attention_f16
#include "launch_attention.inc"
