// fp32 GEMMs with epilogues.
#include "go_kernel_ep.h"
const void* gdy::ep_f32(int family) {
  return family == 1   ? reinterpret_cast<const void*>(&go_gemm_ep<DT_F32>)
         : family == 0 ? reinterpret_cast<const void*>(&split_reduce_ep<DT_F32>)
                       : nullptr;
}
