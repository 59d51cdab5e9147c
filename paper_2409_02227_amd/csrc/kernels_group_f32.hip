// Grouped products of f32 inputs.
#include "grouped.h"
gdy::GroupKernel gdy::group_f32(int over_k, int tb, int tile) { return group_kernels<DT_F32>(over_k, tb, tile); }
