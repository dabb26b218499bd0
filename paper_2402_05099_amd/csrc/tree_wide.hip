// Attention of trees of drafted tokens over a paged cache, 128-row tiles, D = 128 (ragged_wide_impl.h).
#define HG_RW_D 128
#define HG_RW_TREE true
#define HG_RW_KERNEL tree_wide_kernel
#define HG_RW_LAUNCH launch_tree_wide
#include "ragged_wide_impl.h"
