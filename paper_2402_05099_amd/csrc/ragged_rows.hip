// What remains of chunks behind their tiles, or all there is of them, and the join of parts (ragged_rows_kernels.h).
#define HG_ROWS_TREE false
#define HG_ROWS_KERNEL ragged_rows_kernel
#define HG_JOIN_KERNEL ragged_join_kernel
#define HG_ROWS_LAUNCH launch_ragged_rows
#define HG_JOIN_LAUNCH launch_ragged_join
#include "ragged_rows_kernels.h"
