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
  __device__ __forceinline__ EpiOut operator()(int item, int tile_row) const {
    EpiOut o = GroupEpi::operator()(item, tile_row);
    typedef const __attribute__((address_space(4))) KInteger* Ptr;
    Ptr g = (Ptr)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(g));
    o.row_scales = g->row_scales ? g->row_scales + row : nullptr;
    o.col_scales = g->col_scales ? g->col_scales + e * g->stride_col_scales + n0 : nullptr;
    return o;
  }

  // The end of a 256 x 256 tile (p_tiles): acc[half of A][half of B][16-column block][16-row block].  The sums pass
  // through LDS, so that a lane has eight consecutive columns of a row.  All that the arithmetic reads (scales,
  // bias, the first residual rows) is on its way before the sums are laid down: with loads in front of each group of
  // rows the end of a tile took 14 us of the 44 that a tile of 8192 rows in 16 groups x 4096, K = 2048, with silu
  // takes in all, now 8.  Tiles without a residual leave by quadrants (28.5 us for (4096, 8192, 128) with silu, by rows
  // 30.5), those with one by rows, whose loads and stores are of 256 bytes (45.7 us, by quadrants 49.1).
  __device__ __forceinline__ void finish(const f32x4 (&acc)[2][2][2][4], bool half, lds_u8* smem) const {
    const EpiOut o = (*this)(0, 0);
    if (o.res) by_rows(o, acc, half, smem);
    else by_quadrants(o, acc, half, smem);
  }

  // 128 columns at a time, 16 lanes a row, a wave 32 rows, four of them a pass.
  __device__ __forceinline__ void by_rows(const EpiOut& o, const f32x4 (&acc)[2][2][2][4], bool half, lds_u8* smem) const {
    constexpr int OS = OutSize<DT>::v, PITCH = 128 * 4 + 16, PASSES = 8;
    constexpr int AHEAD = OS == 4 ? 1 : 4;  // passes with their residuals on the way: as registers allow
    static_assert(256 * PITCH <= kPLds, "half the columns fit in the ring");
    const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6), wm = wave >> 2, wn = wave & 3;
    const Rsrc rc = make_rsrc(o.c, o.c_bytes), rr = make_rsrc(o.res, ((o.m - 1) * o.ldr + o.n) * OS);
    const int r0 = wave * 32 + (lane >> 4), c0 = (lane & 15) * 8;
    float rs[PASSES];
    Columns<DT> of[2];
#pragma unroll
    for (int p = 0; p < PASSES; ++p) rs[p] = row_scale(o, r0 + 4 * p);
#pragma unroll
    for (int hb = 0; hb < 2; ++hb) of[hb].load(o, hb * 128 + c0);
    const bool live = wave * 32 < o.m;  // some of the wave's rows lie inside C
#pragma unroll
    for (int hb = 0; hb < 2; ++hb) {
      const int left = o.n - hb * 128 - c0;
      const bool whole = __ballot(left > 0 && left < 8) == 0;  // every lane has all its columns inside C, or none
      const bool c_vec = whole && (OS == 4 || o.c_vec), r_vec = whole && (OS == 4 || o.res_vec);
      auto at = [&](int p, int ld) {
        return r0 + 4 * p < o.m && left > 0 ? ((r0 + 4 * p) * ld + hb * 128 + c0) * OS : kOutOfRange;
      };
      auto inside = [&](int p) { return r0 + 4 * p < o.m ? left : 0; };
      Row8<DT> res[AHEAD];
      auto load = [&](int p0) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) res[u].load(rr, at(p0 + u, o.ldr), r_vec, inside(p0 + u));
      };
      if (live) load(0);
      if (hb) __syncthreads();  // the half before is read
#pragma unroll
      for (int ha = 0; ha < 2; ++ha) {
        if (ha && half) break;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j)
            *(__attribute__((address_space(3))) f32x4*)(smem + (ha * 128 + wm * 64 + i * 16 + (lane & 15)) * PITCH +
                                                        (wn * 32 + j * 16 + 4 * (lane >> 4)) * 4) = acc[ha][hb][j][i];
      }
      __syncthreads();
      if (!live) continue;
#pragma unroll
      for (int p0 = 0; p0 < PASSES; p0 += AHEAD) {
        if (p0) load(p0);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
          put_ints<DT>(smem + (r0 + 4 * (p0 + u)) * PITCH + c0 * 4, rs[p0 + u], of[hb], o.act, res[u], true, rc,
               at(p0 + u, o.ldc), c_vec, inside(p0 + u));
      }
    }
  }

  // The wave's quadrants of 64 x 32 through LDS of its own, in two places: no wave waits for another.  Four lanes a
  // row, 16 rows a pass.
  __device__ __forceinline__ void by_quadrants(const EpiOut& o, const f32x4 (&acc)[2][2][2][4], bool half,
                                               lds_u8* smem) const {
    constexpr int OS = OutSize<DT>::v, PITCH = 32 * 4 + 16, BLOCK = 64 * PITCH, PASSES = 4;
    static_assert(2 * 8 * BLOCK <= kPLds, "two blocks a wave fit in the ring");
    const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6), wm = wave >> 2, wn = wave & 3;
    const Rsrc rc = make_rsrc(o.c, o.c_bytes);
    const int r0 = wm * 64 + (lane >> 2), c0 = wn * 32 + (lane & 3) * 8;  // of quadrant 0
    float rs[2][PASSES];
    Columns<DT> of[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int p = 0; p < PASSES; ++p) rs[h][p] = row_scale(o, r0 + h * 128 + 16 * p);
      of[h].load(o, c0 + h * 128);
    }
    auto place = [&](int q) { return smem + (q & 1) * (8 * BLOCK) + wave * BLOCK; };
    // quadrant q: columns q / 2, rows q % 2
    auto dump = [&](int q) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          *(__attribute__((address_space(3))) f32x4*)(place(q) + (i * 16 + (lane & 15)) * PITCH +
                                                      (j * 16 + 4 * (lane >> 4)) * 4) = acc[q & 1][q >> 1][j][i];
    };
    auto done = [&](int q) { return half && (q & 1); };  // no such rows
    dump(0);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (q < 3 && !done(q + 1)) dump(q + 1);
      if (done(q)) continue;
      const int left = o.n - c0 - (q >> 1) * 128;  // columns of C from this lane's on
      const bool vec = __ballot(left > 0 && left < 8) == 0 && (OS == 4 || o.c_vec);
      // the wave's own sums, in LDS in the order of its instructions
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int p = 0; p < PASSES; ++p) {
        const int row = r0 + (q & 1) * 128 + 16 * p;
        const int at = row < o.m && left > 0 ? (row * o.ldc + c0 + (q >> 1) * 128) * OS : kOutOfRange;
        put_ints<DT>(place(q) + ((lane >> 2) + 16 * p) * PITCH + (lane & 3) * 32, rs[q & 1][p], of[q >> 1], o.act,
                     Row8<DT>(), false, rc, at, vec, row < o.m ? left : 0);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // before the next sums in this place
      __builtin_amdgcn_wave_barrier();
    }
  }
};

// The tile's place and extent.
template <int DT> __device__ __forceinline__ bool place_tile(const KGroup& g, int e, int lo, int m0, int m, int n0, int bn,
                                                             IntegerEpi<DT>& ep) {
  ep.e = uniform(e), ep.row = uniform(lo + m0), ep.n0 = uniform(n0);
  ep.m = uniform(m), ep.n = uniform(min(bn, g.n - n0));
  ep.slot = 0, ep.os = OutSize<DT>::v, ep.over_k = false;
  return ep.m > 0;
}

// The group that holds row tile `slot`, each lane's group having tiles(rows) of them; `here`: the lane's of the first 64,
// which are read once for a tile (64 rows in 16 groups x 2048, K = 2048: 13.5 -> 13.2 us; 400 in 100 x 512, 512: 11.5 -> 11.1).
template <class F>
__device__ __forceinline__ bool find_group(const KGroup& g, const GroupRows& here, int slot, F tiles, GroupSlot& out) {
  const int lane = threadIdx.x & 63;
  GroupRows r = here;
  int before = 0;
  for (int e0 = 0; e0 < g.groups; e0 += 64) {
    if (e0) r = group_rows(g.offsets, g.groups, g.rows, e0 + lane);
    const int t = tiles(r.count), s = before + wave_scan(t);
    const uint64_t past = __ballot(s > slot);
    if (past) {
      const int l = (int)__builtin_ctzll(past);
      out.e = e0 + l;
      out.lo = __builtin_amdgcn_readlane(r.lo, l), out.count = __builtin_amdgcn_readlane(r.count, l);
      out.first = __builtin_amdgcn_readlane(s - t, l);
      return true;
    }
    before = __builtin_amdgcn_readlane(s, 63);
  }
  return false;
}

// The tile of C that this workgroup computes, in tiles of bm x bn rows; false: none.  Each XCD takes a contiguous
// run of them (grouped_rows).
template <int DT> __device__ __forceinline__ bool integer_tile(const KGroup& g, int bm, int bn, IntegerEpi<DT>& ep) {
  const int tn = (g.n + bn - 1) / bn, lane = threadIdx.x & 63;
  auto tiles = [&](int rows) { return (rows + bm - 1) / bm; };
  GroupRows here = {0, 0};
  int total = 0;
  if (g.offsets) {
    GroupRows r = here = group_rows(g.offsets, g.groups, g.rows, lane);
    for (int e0 = 0; e0 < g.groups; e0 += 64) {
      if (e0) r = group_rows(g.offsets, g.groups, g.rows, e0 + lane);
      total += __builtin_amdgcn_readlane(wave_scan(tiles(r.count)), 63);
    }
    total = min(total, g.max_slots);
  } else {
    total = tiles(g.rows);
  }
  total *= tn;
  const int per = (total + kXcds - 1) / kXcds, j = (int)blockIdx.x / kXcds;
  const int id = ((int)blockIdx.x & (kXcds - 1)) * per + j;
  if (j >= per || id >= total) return false;
  GroupSlot s = {0, 0, g.rows, 0};
  if (g.offsets && !find_group(g, here, id / tn, tiles, s)) return false;
  int ti, tj;
  group_tile(id - s.first * tn, tiles(s.count), tn, ti, tj);
  return place_tile(g, s.e, s.lo, ti * bm, min(bm, s.count - ti * bm), tj * bn, bn, ep);
}

// The same in 256 x 256 tiles, of which a CU holds one.  What is left of a group behind its 256-row tiles runs as a tile
// of 128 rows where that holds it (a "short" one, 0.65 of a whole one's time); every XCD runs those behind its whole
// ones, so that they fill the CUs which the last of these leave (8192 rows in 16 groups of 206 to 1901 x 4096, K = 2048:
// 104 us with each group's tiles next to each other, 97.6 this way).  Where all of them find a CU the last whole tiles run
// as halves of 128 rows too.
__device__ __forceinline__ int whole_tiles(int rows) { return (rows + 127) / 256; }
__device__ __forceinline__ int short_tiles(int rows) { return (rows + 255) / 256 - (rows + 127) / 256; }

template <int DT> __device__ __forceinline__ bool integer_tile_256(const KGroup& g, IntegerEpi<DT>& ep) {
  const int tn = (g.n + 255) / 256, lane = threadIdx.x & 63;
  GroupRows here = {0, 0};
  int whole = 0, rest = 0;  // row tiles
  if (g.offsets) {
    GroupRows r = here = group_rows(g.offsets, g.groups, g.rows, lane);
    for (int e0 = 0; e0 < g.groups; e0 += 64) {
      if (e0) r = group_rows(g.offsets, g.groups, g.rows, e0 + lane);
      whole += __builtin_amdgcn_readlane(wave_scan(whole_tiles(r.count)), 63);
      rest += __builtin_popcountll(__ballot(short_tiles(r.count) != 0));
    }
    whole = min(whole, g.max_slots);
    rest = min(rest, g.max_slots - whole);
  } else {
    whole = whole_tiles(g.rows), rest = short_tiles(g.rows);
  }
  whole *= tn, rest *= tn;
  const int xcd = (int)blockIdx.x & (kXcds - 1);
  const int per = (whole + kXcds - 1) / kXcds, per_short = (rest + kXcds - 1) / kXcds;
  const int last = per % g.xcd_cus, halved = 2 * last + per_short <= g.xcd_cus ? last : 0;
  int j = (int)blockIdx.x / kXcds, half = -1;
  bool is_short = false;
  if (j >= per + halved) {
    is_short = true;
    j -= per + halved;
    if (j >= per_short) return false;
  } else if (j >= per - halved) {
    half = (j - (per - halved)) & 1;
    j = per - halved + (j - (per - halved)) / 2;
  }
  const int id = xcd * (is_short ? per_short : per) + j;
  if (id >= (is_short ? rest : whole)) return false;
  GroupSlot s = {0, 0, g.rows, 0};
  if (g.offsets &&
      !find_group(g, here, id / tn, [&](int rows) { return is_short ? short_tiles(rows) : whole_tiles(rows); }, s))
    return false;
  int ti, tj;
  if (is_short) {
    ti = whole_tiles(s.count), tj = id - s.first * tn;
  } else {
    group_tile(id - s.first * tn, whole_tiles(s.count), tn, ti, tj);
  }
  const int m0 = ti * 256 + (half > 0 ? 128 : 0);
  return place_tile(g, s.e, s.lo, m0, min(half >= 0 ? 128 : 256, s.count - m0), tj * 256, 256, ep);
}

template <int DT, int TB, class T>
__global__ void __launch_bounds__(T::NT, T::NT == 512 ? 2 : T::LDS > 80 * 1024 ? 1 : 2) integer_rows(KInteger q) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[T::LDS];
  const KGroup& g = q.g;
  IntegerEpi<DT> e;
  if (!(T::BM == 256 ? integer_tile_256<DT>(g, e) : integer_tile<DT>(g, T::BM, T::BN, e))) return;
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
  if (!integer_tile<DT>(g, T::BM, T::BN, e)) return;
  T::tile(g.a + (int64_t)e.row * g.lda, g.b + e.e * g.stride_b + (int64_t)e.n0 * g.ldb, g.lda, g.ldb, e.m, e.n, g.k, e, 0,
          0, (lds_u8*)smem);
}

// Tiles of go_kernel_u.h for operands that both take copies, with a ring of STAGES and the fragments of a K tile read
// in front of its MFMAs (TileU's loop takes any operands and reads them step by step: 244 products of 16 to 4096 rows
// ran 2% slower on its 64 x 128 tiles, (512, 4096, 4096) 21.3 us and 20.3).
template <int DT, int TB, int BM_, int BN_, int WM, int WN, int STAGES> struct TileD {
  static constexpr int BM = BM_, BN = BN_, NT = WM * WN * 64, LDS = UCfg<DT, BM, BN, WM, WN, STAGES>::LDS;
  template <class E> static __device__ __forceinline__ void run(const KArgs& p, lds_u8* smem, const E& e) {
    u_tiles<DT, 0, TB, BM, BN, WM, WN, STAGES, false, false, true, E>(p, 0, 1, smem, e);
  }
};

#define GDY_INTEGER(DT, TB, ...) \
  group_kernel<__VA_ARGS__>(reinterpret_cast<const void*>(&integer_rows<DT, TB, __VA_ARGS__>))
// The tiles of INT_* (gdy_internal.h).
template <int DT, int TB> GroupKernel integer_kernel(int tile) {
  switch (tile) {
    case INT_256: return GDY_INTEGER(DT, TB, TileP<DT, 0, TB>);
    case INT_64x128: return GDY_INTEGER(DT, TB, TileD<DT, TB, 64, 128, 2, 2, 3>);
    case INT_64: return GDY_INTEGER(DT, TB, TileD<DT, TB, 64, 64, 2, 2, 4>);
    case INT_32x64: return GDY_INTEGER(DT, TB, TileD<DT, TB, 32, 64, 1, 4, 4>);
    case INT_ANY_128: return GDY_INTEGER(DT, TB, TileU<DT, 0, TB, 128, 128, 2, 2, 2>);
    case INT_ANY_64x128: return GDY_INTEGER(DT, TB, TileU<DT, 0, TB, 64, 128, 2, 2, 3>);
    case INT_ANY_32x128: return GDY_INTEGER(DT, TB, TileU<DT, 0, TB, 32, 128, 1, 4, 4>);
    case INT_ANY_32x64: return GDY_INTEGER(DT, TB, TileU<DT, 0, TB, 32, 64, 1, 4, 4>);
    case INT_FEW:
      if constexpr (TB == 1)
        return GroupKernel{reinterpret_cast<const void*>(&integer_few<DT>), kSkinnyRows, Skinny<DT, 1>::BN, 512};
    default: return GroupKernel{nullptr, 0, 0, 0};
  }
}
template <int DT> GroupKernel integer_kernels(int tb, int tile) {
  return tb ? integer_kernel<DT, 1>(tile) : integer_kernel<DT, 0>(tile);
}

}  // namespace gdy
