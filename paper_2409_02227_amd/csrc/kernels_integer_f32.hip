// Products of 8-bit integers with results in f32.
#include "integer.h"
gdy::GroupKernel gdy::integer_f32(int tb, int tile) { return integer_kernels<DT_I8_F32>(tb, tile); }
