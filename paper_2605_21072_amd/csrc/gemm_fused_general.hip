// The rest of gemm_fused.hip's builds, in a file of their own so that the two compile side by side: packed INT4 weights, and the
// general form (outlier blocks of any width, any N, any alignment).
#define QARVD_FUSED_GENERAL 1
#include "gemm_fused.hip"
