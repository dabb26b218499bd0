// The same for trees of drafted tokens (ragged_rows_kernels.h).
#define HG_ROWS_TREE true
#define HG_ROWS_KERNEL tree_rows_kernel
#define HG_JOIN_KERNEL tree_join_kernel
#define HG_ROWS_LAUNCH launch_tree_rows
#define HG_JOIN_LAUNCH launch_tree_join
#include "ragged_rows_kernels.h"
