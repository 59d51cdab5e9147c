// Activation gradients and the sums of bias gradients.
#include "act_grad.h"
const void* gdy::act_grad_kernel(int dt) {
  switch (dt) {
    case DT_BF16: return reinterpret_cast<const void*>(&act_grad<DT_BF16>);
    case DT_F16: return reinterpret_cast<const void*>(&act_grad<DT_F16>);
    case DT_F32: return reinterpret_cast<const void*>(&act_grad<DT_F32>);
    default: return nullptr;
  }
}
const void* gdy::bias_sum_kernel(bool many) {
  return many ? reinterpret_cast<const void*>(&bias_sums<16, 64>) : reinterpret_cast<const void*>(&bias_sums<64, 4>);
}
const void* gdy::group_sum_kernel(bool many) {
  return many ? reinterpret_cast<const void*>(&group_sums<16, 64>) : reinterpret_cast<const void*>(&group_sums<64, 4>);
}
