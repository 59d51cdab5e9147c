// grouped.h -- products grouped by expert.  Row counts are known to the device
// alone: group e holds the rows [offsets[e], offsets[e+1]) of A.
//   over rows: C[rows of e] = epilogue(A[rows of e] op(B_e))
//   over K:    C_e = A[rows of e]^T B[rows of e]  (+ R_e)
// A workgroup computes one tile: it finds the group and the tile from the offsets
// (a scan over them in every wave, 64 groups at a time), and runs the tile loop of
// go_kernel_u.h or go_kernel_p.h on that tile alone, so that every extent is the
// tile's own and reads and writes past the group's rows are dropped by the buffer
// unit.  The grid covers the most tiles that the rows can make; the workgroups
// that find none end at once.  Offsets are clamped to 0 .. rows on reading, so no
// value of theirs leads outside the operands.
#pragma once
#include "go_kernel_u.h"

namespace gdy {

// Inclusive sum over the lanes up to this one.
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // row_shr:1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast:15 into rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast:31 into rows 2 and 3
  return x;
}

// This lane's group: its rows within 0 .. rows.
struct GroupRows {
  int lo, count;
};
__device__ __forceinline__ GroupRows group_rows(const int32_t* offsets, int groups, int rows, int e) {
  GroupRows g = {0, 0};
  if (e < groups) {
    g.lo = min(max(offsets[e], 0), rows);
    g.count = min(max(offsets[e + 1], g.lo), rows) - g.lo;
  }
  return g;
}

// Row tiles of `bm` rows over all groups (at most max_slots).
__device__ __forceinline__ int total_slots(const int32_t* offsets, int groups, int rows, int bm, int max_slots) {
  const int lane = threadIdx.x & 63;
  int n = 0;
  for (int e0 = 0; e0 < groups; e0 += 64) {
    const GroupRows g = group_rows(offsets, groups, rows, e0 + lane);
    const int s = wave_scan((g.count + bm - 1) / bm);
    n += __builtin_amdgcn_readlane(s, 63);
  }
  return min(n, max_slots);
}

// The group that holds row tile `slot`; false: none does.
struct GroupSlot {
  int e, lo, count;  // the group and its rows
  int first;         // its first slot
};
__device__ __forceinline__ bool find_slot(const int32_t* offsets, int groups, int rows, int bm, int slot,
                                          GroupSlot& out) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int e0 = 0; e0 < groups; e0 += 64) {
    const GroupRows g = group_rows(offsets, groups, rows, e0 + lane);
    const int t = (g.count + bm - 1) / bm;
    const int s = before + wave_scan(t);
    const uint64_t past = __ballot(s > slot);
    if (past) {
      const int l = (int)__builtin_ctzll(past);
      out.e = e0 + l;
      out.lo = __builtin_amdgcn_readlane(g.lo, l);
      out.count = __builtin_amdgcn_readlane(g.count, l);
      out.first = __builtin_amdgcn_readlane(s - t, l);
      return true;
    }
    before = __builtin_amdgcn_readlane(s, 63);
  }
  return false;
}

// The first slot of group e.
__device__ __forceinline__ int first_slot(const int32_t* offsets, int groups, int rows, int bm, int e) {
  const int lane = threadIdx.x & 63;
  int n = 0;
  for (int e0 = 0; e0 < e; e0 += 64) {
    const GroupRows g = group_rows(offsets, groups, rows, e0 + lane);
    const int s = wave_scan(e0 + lane < e ? (g.count + bm - 1) / bm : 0);
    n += __builtin_amdgcn_readlane(s, 63);
  }
  return n;
}

// Tile `t` of tm x tn: eight tile rows at a time, so that neighbours share rows of
// A and columns of B in an L2.
__device__ __forceinline__ void group_tile(int t, int tm, int tn, int& i, int& j) {
  const int band = 8 * tn, q = t / band, first = q * 8, here = min(tm - first, 8), r = t - q * band;
  i = first + r % here;
  j = r / here;
}

// A tile of a grouped product, and where its results go.  As MemberEpi, the argument
// block is read again when the sums are done.
struct GroupEpi {
  static constexpr bool on = true, linear = true;
  static constexpr int ahead = 2;
  int e, row, n0, m, n, slot;  // group, first row and column in C, extent, row of partial sums
  int os;                      // bytes of an element of C
  bool over_k;
  __device__ __forceinline__ EpiOut operator()(int, int) const {
    typedef const __attribute__((address_space(4))) KGroup* Ptr;
    Ptr g = (Ptr)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(g));
    const int64_t at = over_k ? e : 0;  // groups of C, R (over K)
    EpiOut o;
    o.ldc = g->ldc, o.m = m, o.n = n;
    o.c = g->c + at * g->stride_c + ((int64_t)row * o.ldc + n0) * os;
    o.c_bytes = ((m - 1) * o.ldc + n) * os;
    o.c_vec = g->c_vec != 0;
    o.scale = g->scale * (g->scales ? g->scales[e] : 1.0f);
    o.ldr = g->epi.ldr, o.ldaux = g->epi.ldaux, o.act = g->epi.act;
    o.bias_f32 = g->epi.bias_f32 != 0, o.grad = g->epi.grad != 0;
    o.res_vec = g->epi.res_vec != 0, o.aux_vec = g->epi.aux_vec != 0;
    o.bias = g->epi.bias ? g->epi.bias + e * g->epi.stride_bias + n0 * (o.bias_f32 ? 4 : os) : nullptr;
    o.res = g->epi.res ? g->epi.res + at * g->epi.stride_res + ((int64_t)row * o.ldr + n0) * os : nullptr;
    o.aux = g->epi.aux ? g->epi.aux + ((int64_t)row * o.ldaux + n0) * os : nullptr;
    o.part = g->epi.part ? g->epi.part + (int64_t)slot * g->n + n0 : nullptr;
    return o;
  }
};

// Arguments of one tile: m x n outputs from `k` of K.
template <int DT, int TA, int TB>
__device__ __forceinline__ KArgs tile_args(const KGroup& g, const uint8_t* a, const uint8_t* b, int m, int n, int k) {
  constexpr int ES = ElemSize<DT>::v;
  KArgs p = {};
  p.a = a, p.b = b;
  p.m = m, p.n = n, p.k = k;
  p.lda = g.lda, p.ldb = g.ldb, p.ldc = g.ldc;
  // whole dwords (the operands that the 256 x 256 kernel takes start on one)
  p.a_bytes = k == 0 ? 0 : (((TA == 0 ? (m - 1) * g.lda + k : (k - 1) * g.lda + m) * ES + 3) & ~3);
  p.b_bytes = k == 0 ? 0 : (((TB == 1 ? (n - 1) * g.ldb + k : (k - 1) * g.ldb + n) * ES + 3) & ~3);
  p.tiles_m = p.tiles_n = p.group_m = p.batch = p.split = 1;
  p.a_dma = g.a_dma, p.b_dma = g.b_dma;
  return p;
}

// Tile families: the 256 x 256 kernel, and tiles of go_kernel_u.h.  The latter run the loop
// for any operands, also where both take copies: a K step's fragments are read in front of
// its MFMAs, not a K tile's ahead of them (u_tiles; plain 128 x 128 launches gain 10% by that), and
// the cost model of their tiles is fitted to that loop.
template <int DT, int TA, int TB> struct TileP {
  static constexpr int BM = 256, BN = 256, NT = 512, LDS = kPLds;
  static __device__ __forceinline__ void run(const KArgs& p, lds_u8* smem, const GroupEpi& e) {
    p_tiles<DT, TA, TB, true, GroupEpi>(p, 0, 1, smem, e);
  }
};
template <int DT, int TA, int TB, int BM_, int BN_, int WM, int WN, int STAGES> struct TileU {
  static constexpr int BM = BM_, BN = BN_, NT = WM * WN * 64, LDS = UCfg<DT, BM, BN, WM, WN, STAGES>::LDS;
  static __device__ __forceinline__ void run(const KArgs& p, lds_u8* smem, const GroupEpi& e) {
    u_tiles<DT, TA, TB, BM, BN, WM, WN, STAGES, true, false, true, GroupEpi>(p, 0, 1, smem, e);
  }
};

// Over rows.  The hardware deals workgroup b to XCD b % 8; each XCD takes a
// contiguous run of the tiles, so that a group's B is read by one or two L2s.  A CU
// holds one 256 x 256 tile: where an XCD's last tiles would leave half of its CUs idle
// they run as halves of 128 rows, on twice as many (8192 rows in 16 groups x 4096,
// 80 tiles an XCD: 170 -> 162 us).  The halves have partial sums of their own, so
// every 256-row tile has two rows of them.
template <int DT, int TB, class T>
__global__ void __launch_bounds__(T::NT) grouped_rows(KGroup g) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[T::LDS];
  constexpr int ES = ElemSize<DT>::v;
  const int bm = T::BM == 256 ? g.bm : T::BM;  // the 256 x 256 kernel has 128-row tiles too
  const bool two = T::BM == 256 && bm == 256;
  const int tn = (g.n + T::BN - 1) / T::BN;
  const int total = total_slots(g.offsets, g.groups, g.rows, bm, g.max_slots) * tn;
  const int per = (total + kXcds - 1) / kXcds;
  int j = (int)blockIdx.x / kXcds, half = -1;
  if (two) {
    const int rest = per % g.xcd_cus;
    if (2 * rest <= g.xcd_cus && j >= per - rest) {
      half = (j - (per - rest)) & 1;
      j = per - rest + (j - (per - rest)) / 2;
    }
  }
  const int id = ((int)blockIdx.x & (kXcds - 1)) * per + j;
  if (j >= per || id >= total) return;
  GroupSlot s;
  if (!find_slot(g.offsets, g.groups, g.rows, bm, id / tn, s)) return;
  int ti, tj;
  group_tile(id - s.first * tn, (s.count + bm - 1) / bm, tn, ti, tj);
  const int m0 = ti * bm + (half > 0 ? 128 : 0), n0 = tj * T::BN;
  GroupEpi e;
  e.e = uniform(s.e), e.row = uniform(s.lo + m0), e.n0 = uniform(n0);
  e.m = uniform(min(half >= 0 ? 128 : bm, s.count - m0)), e.n = uniform(min(T::BN, g.n - n0));
  e.slot = uniform(two ? 2 * (s.first + ti) + (half > 0) : s.first + ti);
  if (two && g.epi.part && (half < 0 || e.m <= 0) && (int)threadIdx.x < e.n)  // the sums of no half
    g.epi.part[(int64_t)(half < 0 ? e.slot + 1 : e.slot) * g.n + n0 + threadIdx.x] = 0.0f;
  if (e.m <= 0) return;
  e.os = OutSize<DT>::v, e.over_k = false;
  const uint8_t* a = g.a + (int64_t)e.row * g.lda * ES;
  const uint8_t* b = g.b + e.e * g.stride_b + (TB == 1 ? (int64_t)e.n0 * g.ldb : (int64_t)e.n0) * ES;
  T::run(tile_args<DT, 0, TB>(g, a, b, e.m, e.n, g.k), (lds_u8*)smem, e);
}

// Over K.  Every group's tiles are dealt to all XCDs, each a contiguous run of them, with no
// workgroup left idle: a 256 x 256 one would hold a CU (128 groups of 64 rows, 512 x 256, two
// tiles each: 38.6 us where each group took eight workgroups, now 16.2).
template <int DT, class T>
__global__ void __launch_bounds__(T::NT) grouped_k(KGroup g) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[T::LDS];
  constexpr int ES = ElemSize<DT>::v;
  const int tm = (g.m + T::BM - 1) / T::BM, tn = (g.n + T::BN - 1) / T::BN;
  const int tiles = tm * tn, group = (int)blockIdx.x / tiles, r = (int)blockIdx.x - group * tiles;
  const int x = r & (kXcds - 1);
  const int t = x * (tiles / kXcds) + min(x, tiles & (kXcds - 1)) + r / kXcds;
  const GroupRows rows = group_rows(g.offsets, g.groups, g.rows, group);
  int ti, tj;
  group_tile(t, tm, tn, ti, tj);
  GroupEpi e;
  e.e = uniform(group), e.row = uniform(ti * T::BM), e.n0 = uniform(tj * T::BN);
  e.m = min(T::BM, g.m - e.row), e.n = min(T::BN, g.n - e.n0), e.slot = 0;
  e.os = OutSize<DT>::v, e.over_k = true;
  const int64_t lo = uniform(rows.lo);
  const uint8_t* a = g.a + (lo * g.lda + e.row) * ES;
  const uint8_t* b = g.b + (lo * g.ldb + e.n0) * ES;
  T::run(tile_args<DT, 1, 0>(g, a, b, e.m, e.n, uniform(rows.count)), (lds_u8*)smem, e);
}

// ---- the kernels of one input type ------------------------------------------------
template <class T> GroupKernel group_kernel(const void* f) { return GroupKernel{f, T::BM, T::BN, T::NT}; }
#define GDY_GROUP_ROWS(DT, TB, ...) \
  group_kernel<__VA_ARGS__>(reinterpret_cast<const void*>(&grouped_rows<DT, TB, __VA_ARGS__>))
#define GDY_GROUP_K(DT, ...) group_kernel<__VA_ARGS__>(reinterpret_cast<const void*>(&grouped_k<DT, __VA_ARGS__>))

template <int DT, int TB> GroupKernel rows_kernel(int tile) {
  switch (tile) {
    case 0:
      if constexpr (DT != DT_F32) return GDY_GROUP_ROWS(DT, TB, TileP<DT, 0, TB>);
      else return GroupKernel{nullptr, 0, 0, 0};
    case 1: return GDY_GROUP_ROWS(DT, TB, TileU<DT, 0, TB, 128, 128, 2, 2, 2>);
    case 2: return GDY_GROUP_ROWS(DT, TB, TileU<DT, 0, TB, 64, 128, 2, 2, 3>);
    case 3: return GDY_GROUP_ROWS(DT, TB, TileU<DT, 0, TB, 32, 128, 1, 4, 4>);
    case 4: return GDY_GROUP_ROWS(DT, TB, TileU<DT, 0, TB, 32, 64, 1, 4, 4>);
    default: return GroupKernel{nullptr, 0, 0, 0};
  }
}
template <int DT> GroupKernel k_kernel(int tile) {
  switch (tile) {
    case 0:
      if constexpr (DT != DT_F32) return GDY_GROUP_K(DT, TileP<DT, 1, 0>);
      else return GroupKernel{nullptr, 0, 0, 0};
    case 1: return GDY_GROUP_K(DT, TileU<DT, 1, 0, 128, 128, 2, 2, 2>);
    case 2: return GDY_GROUP_K(DT, TileU<DT, 1, 0, 64, 64, 2, 2, 4>);
    default: return GroupKernel{nullptr, 0, 0, 0};
  }
}
template <int DT> GroupKernel group_kernels(int over_k, int tb, int tile) {
  return over_k ? k_kernel<DT>(tile) : tb ? rows_kernel<DT, 1>(tile) : rows_kernel<DT, 0>(tile);
}

}  // namespace gdy
