// f32 GEMMs with epilogues: launches of one tile and layout.
#include "go_kernel_ep.h"
const void* gdy::ep_lone_f32(int family, int code, bool copies) { return ep_lone<DT_F32>(family, code, copies); }
