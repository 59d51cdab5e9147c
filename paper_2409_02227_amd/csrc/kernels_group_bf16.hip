// Grouped products of bf16 inputs.
#include "grouped.h"
gdy::GroupKernel gdy::group_bf16(int over_k, int tb, int tile) { return group_kernels<DT_BF16>(over_k, tb, tile); }
