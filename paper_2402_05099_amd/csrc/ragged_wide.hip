// Causal attention of packed tokens, 128-row tiles, D = 128 (ragged_wide_impl.h).
#define HG_RW_D 128
#define HG_RW_KERNEL ragged_wide_kernel
#define HG_RW_LAUNCH launch_ragged_wide
#include "ragged_wide_impl.h"
