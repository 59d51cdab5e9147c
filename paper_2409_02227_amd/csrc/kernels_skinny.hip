// GEMMs of at most 16 rows with epilogues, and grouped products in tiles of 16 rows.
#include "skinny.h"
const void* gdy::skinny_ep(int dt, int tb) {
  switch (dt) {
    case DT_BF16: return skinny_kernel<DT_BF16>(tb);
    case DT_F16: return skinny_kernel<DT_F16>(tb);
    case DT_FP8: return skinny_kernel<DT_FP8>(tb);
    default: return skinny_kernel<DT_F32>(tb);
  }
}
gdy::GroupKernel gdy::group_few(int dt, int tb) {
  switch (dt) {
    case DT_BF16: return few_kernel<DT_BF16>(tb);
    case DT_F16: return few_kernel<DT_F16>(tb);
    case DT_FP8: return few_kernel<DT_FP8>(tb);
    default: return few_kernel<DT_F32>(tb);
  }
}
