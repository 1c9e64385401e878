// The second projection's kernels of the 8-bit grouped GEMM.
#define GG_SECOND_PROJECTION
#include "moe_i8_grouped.hip"
