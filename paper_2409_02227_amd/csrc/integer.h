// integer.h -- products of 8-bit integers with a scale for each row of A and each column
// of C, dense or grouped by expert over rows:
//   C(i,j) = round(f(row_scale(i) * col_scale(j) * sum_k A(i,k) op(B)(k,j) + bias(j)) + R(i,j))
// The loops, tiles and group search of the grouped products (grouped.h, skinny.h) with
// integer MFMAs: their sums stay integers until the epilogue (epilogue.h), which makes
// them floats and applies the scales, so that no order of additions matters.
#pragma once
#include "skinny.h"

namespace gdy {

// A tile and where its results go: as GroupEpi, with the scales.
template <int DT> struct IntegerEpi : GroupEpi {
  static constexpr bool linear = OutSize<DT>::v == 2;
  __device__ __forceinline__ EpiOut operator()(int item, int tile_row) const {
    EpiOut o = GroupEpi::operator()(item, tile_row);
    typedef const __attribute__((address_space(4))) KInteger* Ptr;
    Ptr g = (Ptr)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(g));
    o.row_scales = g->row_scales ? g->row_scales + row : nullptr;
    o.col_scales = g->col_scales ? g->col_scales + e * g->stride_col_scales + n0 : nullptr;
    return o;
  }
};

// The tile of C that this workgroup computes, in tiles of bm x bn rows; false: none.  halves:
// whether the last tiles run as halves of 128 rows (grouped_rows).
template <int DT>
__device__ __forceinline__ bool integer_tile(const KGroup& g, int bm, int bn, bool halves, IntegerEpi<DT>& e) {
  const int tn = (g.n + bn - 1) / bn;
  const int total = (g.offsets ? total_slots(g.offsets, g.groups, g.rows, bm, g.max_slots) : (g.rows + bm - 1) / bm) * tn;
  const int per = (total + kXcds - 1) / kXcds;
  int j = (int)blockIdx.x / kXcds, half = -1;
  if (halves) {
    const int rest = per % g.xcd_cus;
    if (2 * rest <= g.xcd_cus && j >= per - rest) {
      half = (j - (per - rest)) & 1;
      j = per - rest + (j - (per - rest)) / 2;
    }
  }
  const int id = ((int)blockIdx.x & (kXcds - 1)) * per + j;
  if (j >= per || id >= total) return false;
  GroupSlot s = {0, 0, g.rows, 0};
  if (g.offsets && !find_slot(g.offsets, g.groups, g.rows, bm, id / tn, s)) return false;
  int ti, tj;
  group_tile(id - s.first * tn, (s.count + bm - 1) / bm, tn, ti, tj);
  const int m0 = ti * bm + (half > 0 ? 128 : 0);
  e.e = uniform(s.e), e.row = uniform(s.lo + m0), e.n0 = uniform(tj * bn);
  e.m = uniform(min(half >= 0 ? 128 : bm, s.count - m0)), e.n = uniform(min(bn, g.n - tj * bn));
  e.slot = 0, e.os = OutSize<DT>::v, e.over_k = false;
  return e.m > 0;
}

template <int DT, int TB, class T>
__global__ void __launch_bounds__(T::NT) integer_rows(KInteger q) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[T::LDS];
  const KGroup& g = q.g;
  const int bm = T::BM == 256 ? g.bm : T::BM;  // the 256 x 256 kernel has 128-row tiles too
  IntegerEpi<DT> e;
  if (!integer_tile<DT>(g, bm, T::BN, T::BM == 256 && bm == 256, e)) return;
  const uint8_t* a = g.a + (int64_t)e.row * g.lda;
  const uint8_t* b = g.b + e.e * g.stride_b + (TB == 1 ? (int64_t)e.n0 * g.ldb : (int64_t)e.n0);
  T::run(tile_args<DT, 0, TB>(g, a, b, e.m, e.n, g.k), (lds_u8*)smem, e);
}

// At most 16 rows a tile, K over a workgroup's waves; B stored N x K.
template <int DT>
__global__ void __launch_bounds__(512) integer_few(KInteger q) {
  typedef Skinny<DT, 1> T;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[T::LDS];
  const KGroup& g = q.g;
  IntegerEpi<DT> e;
  if (!integer_tile<DT>(g, T::BM, T::BN, false, e)) return;
  T::tile(g.a + (int64_t)e.row * g.lda, g.b + e.e * g.stride_b + (int64_t)e.n0 * g.ldb, g.lda, g.ldb, e.m, e.n, g.k, e, 0,
          0, (lds_u8*)smem);
}

#define GDY_INTEGER(DT, TB, ...) \
  group_kernel<__VA_ARGS__>(reinterpret_cast<const void*>(&integer_rows<DT, TB, __VA_ARGS__>))
template <int DT, int TB> GroupKernel integer_kernel(int tile) {
  switch (tile) {
    case 0: return GDY_INTEGER(DT, TB, TileP<DT, 0, TB>);
    case 1: return GDY_INTEGER(DT, TB, TileU<DT, 0, TB, 128, 128, 2, 2, 2>);
    case 2: return GDY_INTEGER(DT, TB, TileU<DT, 0, TB, 64, 128, 2, 2, 3>);
    case 3: return GDY_INTEGER(DT, TB, TileU<DT, 0, TB, 32, 128, 1, 4, 4>);
    case 4: return GDY_INTEGER(DT, TB, TileU<DT, 0, TB, 32, 64, 1, 4, 4>);
    default: return GroupKernel{nullptr, 0, 0, 0};
  }
}
template <int DT> GroupKernel integer_kernels(int tb, int tile, bool few) {
  if (few) {
    if (!tb) return GroupKernel{nullptr, 0, 0, 0};
    return GroupKernel{reinterpret_cast<const void*>(&integer_few<DT>), kSkinnyRows, Skinny<DT, 1>::BN, 512};
  }
  return tb ? integer_kernel<DT, 1>(tile) : integer_kernel<DT, 0>(tile);
}

}  // namespace gdy
