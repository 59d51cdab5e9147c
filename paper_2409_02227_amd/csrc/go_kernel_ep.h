// go_kernel_ep.h -- launches whose members carry epilogues (epilogue.h): the loops and
// tiles of the joint kernels of go_kernel_u.h and go_kernel_p.h, so an element's
// fp32 sum is that of the plain launch.  Members of one tile and layout run on a
// kernel of their own; go_gemm_ep and go_gemm_p_ep run mixed ones, as the joint
// kernels do.
#pragma once
#include "go_kernel_u.h"

namespace gdy {

// Member gi's arguments, read from the argument block for each work item (as
// MemberEpi): nothing of them is kept through an epilogue.
__device__ __forceinline__ KArgs member_args(int gi) {
  typedef const __attribute__((address_space(4))) uint8_t* Ptr;
  Ptr args = (Ptr)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(args));
  const auto* q = (const __attribute__((address_space(4))) KArgs*)(args + offsetof(KLaunch, g)) + gi;
  KArgs p = {};
  p.a = q->a, p.b = q->b;
  p.m = q->m, p.n = q->n, p.k = q->k;
  p.lda = q->lda, p.ldb = q->ldb;
  p.a_bytes = q->a_bytes, p.b_bytes = q->b_bytes;
  p.tiles_m = q->tiles_m, p.tiles_n = q->tiles_n, p.batch = q->batch;
  p.a_dma = q->a_dma, p.b_dma = q->b_dma, p.group_m = q->group_m, p.xcd_remap = q->xcd_remap;
  p.code = q->code, p.rows128 = q->rows128;
  p.split = q->split, p.split_kt = q->split_kt, p.ws = q->ws;
  p.stride_a = q->stride_a, p.stride_b = q->stride_b;
  return p;
}

// A workgroup of NT threads: its member's work items, each by T::run, or an add's.
template <int NT, class T>
__device__ __forceinline__ void ep_member(const KLaunch& L, lds_u8* smem) {
  int gi, lwg, nwg;
  locate(L, gi, lwg, nwg);
  if (gi < 0) return;
  if (L.g[gi].ew) {
    ew_member<NT>(L.g[gi], lwg, nwg);
    return;
  }
  gi = uniform(gi), lwg = uniform(lwg), nwg = uniform(nwg);
  for (int tb = lwg;; tb += nwg) {
    const KArgs p = member_args(gi);
    if (tb >= p.tiles_m * p.tiles_n * p.batch * p.split) break;
    if (tb != lwg) __syncthreads();  // the epilogue's rows before are read
    T::run(p, tb, gi, smem);
  }
}

template <int DT> struct MixedU {
  static __device__ __forceinline__ void run(const KArgs& p, int tb, int gi, lds_u8* smem) {
    // fp8's loops leave registers for one row ahead and no linear path
    typedef MemberEpi<DT == DT_FP8 ? 1 : 2, DT != DT_FP8> E;
    switch (p.code >> 3) {
      case 0: joint_tiles<DT, 0, 0, E>(p, tb, 1 << 30, smem, E{gi}); break;
      case 1: joint_tiles<DT, 0, 1, E>(p, tb, 1 << 30, smem, E{gi}); break;
      case 2: joint_tiles<DT, 1, 0, E>(p, tb, 1 << 30, smem, E{gi}); break;
      default: joint_tiles<DT, 1, 1, E>(p, tb, 1 << 30, smem, E{gi});
    }
  }
};
template <int DT> struct MixedP {
  static __device__ __forceinline__ void run(const KArgs& p, int tb, int gi, lds_u8* smem) {
    typedef MemberEpi<2, false> E;
    switch (p.code) {
      case 0: p_tiles<DT, 0, 0, true, E>(p, tb, 1 << 30, smem, E{gi}); break;
      case 1: p_tiles<DT, 0, 1, true, E>(p, tb, 1 << 30, smem, E{gi}); break;
      case 2: p_tiles<DT, 1, 0, true, E>(p, tb, 1 << 30, smem, E{gi}); break;
      default: p_tiles<DT, 1, 1, true, E>(p, tb, 1 << 30, smem, E{gi});
    }
  }
};
template <int DT, int TA, int TB> struct LoneP {
  static __device__ __forceinline__ void run(const KArgs& p, int tb, int gi, lds_u8* smem) {
    p_tiles<DT, TA, TB, false, MemberEpi<2>>(p, tb, 1 << 30, smem, MemberEpi<2>{gi});
  }
};
template <int DT, int TA, int TB, int BM, int BN, int WM, int WN, int STAGES, bool ANY> struct LoneU {
  static __device__ __forceinline__ void run(const KArgs& p, int tb, int gi, lds_u8* smem) {
    u_tiles<DT, TA, TB, BM, BN, WM, WN, STAGES, ANY, true, false, MemberEpi<2>>(p, tb, 1 << 30, smem, MemberEpi<2>{gi});
  }
};

// The kernels take KEpis, which MemberEpi reads from the argument block.  Two workgroups
// a CU: registers are held to 256 (mixed members of 154 x 5120 x 4608, backward, bf16:
// 278 registers and one workgroup 89 us, 256 61).
template <int DT>
__global__ void __launch_bounds__(256, 2) go_gemm_ep(KLaunch L, KEpis) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[kJointLds];
  ep_member<256, MixedU<DT>>(L, (lds_u8*)smem);
}
template <int DT>
__global__ void __launch_bounds__(512) go_gemm_p_ep(KLaunch L, KEpis) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[kPLds];
  ep_member<512, MixedP<DT>>(L, (lds_u8*)smem);
}
// One tile and layout.
template <int DT, int TA, int TB>
__global__ void __launch_bounds__(512) go_gemm_p_ep1(KLaunch L, KEpis) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[kPLds];
  ep_member<512, LoneP<DT, TA, TB>>(L, (lds_u8*)smem);
}
template <int DT, int TA, int TB, int BM, int BN, int WM, int WN, int STAGES, bool ANY>
__global__ void __launch_bounds__(WM * WN * 64, (UCfg<DT, BM, BN, WM, WN, STAGES>::LDS > 80 * 1024 ? 1 : 2))
go_gemm_ep1(KLaunch L, KEpis) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[UCfg<DT, BM, BN, WM, WN, STAGES>::LDS];
  ep_member<WM * WN * 64, LoneU<DT, TA, TB, BM, BN, WM, WN, STAGES, ANY>>(L, (lds_u8*)smem);
}

// Members of joint code `code`; copies: both operands of all of them take copies.
template <int DT, int TA, int TB, int BM, int BN, int WM, int WN, int STAGES>
const void* ep1_kernel(bool copies) {
  if (copies)
    return reinterpret_cast<const void*>(&go_gemm_ep1<DT, TA, TB, BM, BN, WM, WN, STAGES, false>);
  return reinterpret_cast<const void*>(&go_gemm_ep1<DT, TA, TB, BM, BN, WM, WN, STAGES, true>);
}
template <int DT, int TA, int TB> const void* ep1_tile(int tile, bool copies) {
  switch (tile) {
    case 0: return ep1_kernel<DT, TA, TB, 128, 128, 2, 2, 2>(copies);
    case 2: return ep1_kernel<DT, TA, TB, 64, 64, 2, 2, 4>(copies);
    case 4: return ep1_kernel<DT, TA, TB, 32, 64, 1, 4, 4>(copies);
    case 5: return reinterpret_cast<const void*>(&go_gemm_ep1<DT, TA, TB, 128, 128, 2, 2, 4, false>);
    default:  // as joint_tiles
      if constexpr (TA == 0)
        return tile == 1 ? ep1_kernel<DT, TA, TB, 64, 128, 2, 2, 3>(copies) : ep1_kernel<DT, TA, TB, 32, 128, 1, 4, 4>(copies);
      else
        return nullptr;
  }
}
template <int DT> const void* ep_lone(int family, int code, bool copies) {
  if constexpr (DT != DT_F32)
    if (family == 2) switch (code) {
        case 0: return reinterpret_cast<const void*>(&go_gemm_p_ep1<DT, 0, 0>);
        case 1: return reinterpret_cast<const void*>(&go_gemm_p_ep1<DT, 0, 1>);
        case 2: return reinterpret_cast<const void*>(&go_gemm_p_ep1<DT, 1, 0>);
        default: return reinterpret_cast<const void*>(&go_gemm_p_ep1<DT, 1, 1>);
      }
  switch (code >> 3) {
    case 0: return ep1_tile<DT, 0, 0>(code & 7, copies);
    case 1: return ep1_tile<DT, 0, 1>(code & 7, copies);
    case 2: return ep1_tile<DT, 1, 0>(code & 7, copies);
    default: return ep1_tile<DT, 1, 1>(code & 7, copies);
  }
}

}  // namespace gdy
