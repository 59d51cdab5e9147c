// fp8 GEMMs with epilogues.
#include "go_kernel_ep.h"
const void* gdy::ep_fp8(int family) {
  return family == 1   ? reinterpret_cast<const void*>(&go_gemm_ep<DT_FP8>)
         : family == 2 ? reinterpret_cast<const void*>(&go_gemm_p_ep<DT_FP8>)
                       : reinterpret_cast<const void*>(&split_reduce_ep<DT_FP8>);
}
