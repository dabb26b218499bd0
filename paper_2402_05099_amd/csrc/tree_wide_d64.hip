// Attention of trees of drafted tokens over a paged cache, 128-row tiles, D = 64 (ragged_wide_impl.h).
#define HG_RW_D 64
#define HG_RW_TREE true
#define HG_RW_KERNEL tree_wide_kernel_d64
#define HG_RW_LAUNCH launch_tree_wide_d64
#include "ragged_wide_impl.h"
