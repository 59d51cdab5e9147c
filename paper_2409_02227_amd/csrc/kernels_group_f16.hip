// Grouped products of f16 inputs.
#include "grouped.h"
gdy::GroupKernel gdy::group_f16(int over_k, int tb, int tile) { return group_kernels<DT_F16>(over_k, tb, tile); }
