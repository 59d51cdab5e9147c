// Products of 8-bit integers with results in bf16.
#include "integer.h"
gdy::GroupKernel gdy::integer_bf16(int tb, int tile) { return integer_kernels<DT_I8_BF16>(tb, tile); }
