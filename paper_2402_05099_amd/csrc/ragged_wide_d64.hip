// Causal attention of packed tokens, 128-row tiles, D = 64 (ragged_wide_impl.h).
#define HG_RW_D 64
#define HG_RW_KERNEL ragged_wide_kernel_d64
#define HG_RW_LAUNCH launch_ragged_wide_d64
#include "ragged_wide_impl.h"
