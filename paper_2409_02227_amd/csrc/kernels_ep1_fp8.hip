// fp8 GEMMs with epilogues: launches of one tile and layout.
#include "go_kernel_ep.h"
const void* gdy::ep_lone_fp8(int family, int code, bool copies) { return ep_lone<DT_FP8>(family, code, copies); }
