// go_kernel_ep.h -- launches whose members carry epilogues (epilogue.h).  One
// kernel per family and input type runs members of every tile and layout, as the
// joint kernels of go_kernel_u.h and go_kernel_p.h do without: the same loops on
// the same tiles, so an element's fp32 sum is that of the plain launch.
#pragma once
#include "go_kernel_u.h"

namespace gdy {

template <int DT>
__global__ void __launch_bounds__(256)
go_gemm_ep(KLaunch L, KEpis E) {
  (void)E;  // read by MemberEpi
  __shared__ __attribute__((aligned(1024))) uint8_t smem_raw[kJointLds];
  lds_u8* smem = (lds_u8*)smem_raw;
  int gi, lwg, nwg;
  locate(L, gi, lwg, nwg);
  if (gi < 0) return;
  const KArgs& p = L.g[gi];
  if (p.ew) {
    ew_member<256>(p, lwg, nwg);
    return;
  }
  const MemberEpi ep = {uniform(gi)};
  switch (p.code >> 3) {
    case 0: joint_tiles<DT, 0, 0, MemberEpi>(p, lwg, nwg, smem, ep); break;
    case 1: joint_tiles<DT, 0, 1, MemberEpi>(p, lwg, nwg, smem, ep); break;
    case 2: joint_tiles<DT, 1, 0, MemberEpi>(p, lwg, nwg, smem, ep); break;
    default: joint_tiles<DT, 1, 1, MemberEpi>(p, lwg, nwg, smem, ep);
  }
}

template <int DT>
__global__ void __launch_bounds__(512)
go_gemm_p_ep(KLaunch L, KEpis E) {
  (void)E;  // read by MemberEpi
  __shared__ __attribute__((aligned(1024))) uint8_t smem_raw[kPLds];
  lds_u8* smem = (lds_u8*)smem_raw;
  int gi, lwg, nwg;
  locate(L, gi, lwg, nwg);
  if (gi < 0) return;
  const KArgs& p = L.g[gi];
  if (p.ew) {
    ew_member<512>(p, lwg, nwg);
    return;
  }
  const MemberEpi ep = {uniform(gi)};
  switch (p.code) {
    case 0: p_tiles<DT, 0, 0, true, MemberEpi>(p, lwg, nwg, smem, ep); break;
    case 1: p_tiles<DT, 0, 1, true, MemberEpi>(p, lwg, nwg, smem, ep); break;
    case 2: p_tiles<DT, 1, 0, true, MemberEpi>(p, lwg, nwg, smem, ep); break;
    default: p_tiles<DT, 1, 1, true, MemberEpi>(p, lwg, nwg, smem, ep);
  }
}

}  // namespace gdy
