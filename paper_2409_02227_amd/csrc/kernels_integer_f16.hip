// Products of 8-bit integers with results in f16.
#include "integer.h"
gdy::GroupKernel gdy::integer_f16(int tb, int tile) { return integer_kernels<DT_I8_F16>(tb, tile); }
