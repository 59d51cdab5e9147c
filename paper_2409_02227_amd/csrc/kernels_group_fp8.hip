// Grouped products of fp8 inputs.
#include "grouped.h"
gdy::GroupKernel gdy::group_fp8(int over_k, int tb, int tile) { return group_kernels<DT_FP8>(over_k, tb, tile); }
