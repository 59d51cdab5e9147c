// bf16 GEMMs with epilogues.
#include "go_kernel_ep.h"
const void* gdy::ep_bf16(int family) {
  return family == 1   ? reinterpret_cast<const void*>(&go_gemm_ep<DT_BF16>)
         : family == 2 ? reinterpret_cast<const void*>(&go_gemm_p_ep<DT_BF16>)
                       : reinterpret_cast<const void*>(&split_reduce_ep<DT_BF16>);
}
