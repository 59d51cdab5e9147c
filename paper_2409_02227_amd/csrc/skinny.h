// skinny.h -- GEMMs of at most 16 rows with epilogues (single tokens, small decode
// batches): the weight is read once and bounds the time, so the kernel is made for
// its stream.
//
// A workgroup of eight waves owns 16 columns (B stored N x K) or 64 (K x N), the
// waves an eighth of K each.  Both operands go from global memory straight into MFMA
// fragments: nothing is shared between waves, so there is no LDS stage, no barrier
// and no tile loop to fill.  The waves' sums meet in LDS, are added in wave order and
// leave through the epilogue, so a K needs no second kernel: (1, 2048, 2048) bf16 11.6 us on
// the tile kernels (two runs and their reduction), 7.2 here; K x N 9.0.
//
// A wave takes K in rounds of AHEAD steps: loads of 8 KiB of B (K x N: 16), then their
// MFMAs.  The source orders no more than that, and the compiler moves loads behind MFMAs: of
// a round's 16 loads of N x K, 16- and 8-bit types have 9 to 12 under way before the first
// wait, fp32 4; of K x N's 20 or 36, 4 to 10, and some waits are for all of them.  A round is so a
// chain of two to ten trips to HBM and not one, and what bounds this kernel where K is long.
// The times here and the rules that choose this kernel are of the code as it is.  It holds
// while K takes a wave at most two rounds (M = 1 and 16, N =
// 256 to 8192, weights from HBM, tile kernels against this one: bf16 N x K, K = 2048, one
// round, 14-16 and 9-15 us; K = 8192, four, 14-37 and 14-42; K x N, K = 2048, two, 14-17 and 9-14;
// K = 8192, eight, 16-38 and 26-47; fp8 N x K, K = 8192, two, 14-25 and 9-22).
//
// Grouped products over rows take the same loop (grouped_few), for any K and row count
// where 32 x 64 tiles would wait for one K tile after another: their sums have no split
// otherwise.
//
// Fragments (lane l, i = l % 16, g = l / 16; A's and B's K agree):
//  * N x K: lane l holds 16 bytes of K of column i, as A's of row i: K bytes 64 step +
//    16 g (8-bit types: 32 bytes, 128 step + 32 g).
//  * K x N: lane l loads the columns 4i .. 4i + 3 of the rows that its K bytes of A name
//    (16-bit types: eight rows of 8 bytes, transposed by byte permutes; fp32: four
//    rows of 16 bytes, no transpose); MFMA j takes column 4i + j of every lane.
#pragma once
#include "go_kernel_ep.h"
#include "grouped.h"

namespace gdy {

template <int DT, int TB> struct Skinny {
  static constexpr int ES = ElemSize<DT>::v;
  static constexpr int NW = 8, NT = NW * 64;
  static constexpr int BM = kSkinnyRows, BN = skinny_cols(TB), NJ = BN / 16;
  static constexpr int KB = skinny_kstep(ES);     // K bytes of a step
  static constexpr int AV = KB / 64;              // 16-byte loads of a lane's K bytes
  static constexpr int KROWS = 16 / ES;           // K x N: rows of a lane's K bytes
  static constexpr int AHEAD = skinny_ahead(ES, TB);  // steps of a round
  static constexpr int PITCH = BN * 4 + 16;
  static constexpr int TABLE = NW * BM * PITCH;   // column sums behind the waves' blocks
  static constexpr int LDS = TABLE + BM * BN * 4;
  static_assert(TB == 1 || ES != 1, "8-bit K x N operands take the tile kernels");
  typedef Mma<DT, 16> M;

  struct Step {
    u32x4 a[AV];
    u32x4 b[TB == 1 ? AV : (ES == 4 ? 4 : 1)];
    u32x2 r[TB == 0 && ES == 2 ? 8 : 1];
  };

  // m x n outputs (n <= BN) of A (m x k) and this tile's columns of B.
  template <class EP>
  static __device__ __forceinline__ void tile(const uint8_t* a, const uint8_t* b, int lda_b, int ldb_b, int m, int n,
                                              int k, const EP& ep, int item, int n0, lds_u8* smem) {
    const int tid = threadIdx.x, lane = tid & 63, i = lane & 15, g = lane >> 4;
    const int wave = uniform(tid >> 6);
    const int kbytes = k * ES;
    // whole dwords: the last element may share one with bytes past the operand
    const Rsrc ra = make_rsrc(a, ((m - 1) * lda_b + kbytes + 3) & ~3);
    const Rsrc rb = make_rsrc(b, (TB == 1 ? (n - 1) * ldb_b + kbytes + 3 : (k - 1) * ldb_b + n * ES + 3) & ~3);
    const int steps = (kbytes + KB - 1) / KB, per = (steps + NW - 1) / NW;
    const int s0 = wave * per, s1 = min(steps, s0 + per);
    const int a0 = i * lda_b + g * (16 * AV);
    const int b0 = TB == 1 ? i * ldb_b + g * (16 * AV) : g * KROWS * ldb_b + i * 4 * ES;

    // 8-bit integers have scales to wait for: (1, 2048, 2048) 4.5 us, with these loads behind the loop 5.1
    Columns<DT> columns;
    float rs = 1.0f;
    if constexpr (IsInt8<DT>::v) {
      if (wave == 0) {
        const EpiOut o = ep(item, 0);
        columns.load(o, n0 + (tid % (BN / 8)) * 8);
        rs = row_scale(o, tid / (BN / 8));
      }
    }

    f32x4 acc[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    auto load = [&](Step& x, int s) {
#pragma unroll
      for (int v = 0; v < AV; ++v) {
        // K bytes past K, and steps of the next wave, are sent out of range
        const bool in = s < s1 && s * KB + g * (16 * AV) + v * 16 < kbytes;
        const int ka = s * KB + v * 16;
        x.a[v] = __builtin_amdgcn_raw_buffer_load_b128(ra, in ? a0 + ka : kOutOfRange, 0, 0);
        if constexpr (TB == 1) x.b[v] = __builtin_amdgcn_raw_buffer_load_b128(rb, in ? b0 + ka : kOutOfRange, 0, 0);
      }
      if constexpr (TB == 0) {
        const int at = s < s1 ? b0 + s * (KB / ES) * ldb_b : kOutOfRange;
#pragma unroll
        for (int r = 0; r < KROWS; ++r) {
          if constexpr (ES == 4) x.b[r] = __builtin_amdgcn_raw_buffer_load_b128(rb, at + (s < s1 ? r * ldb_b : 0), 0, 0);
          else x.r[r] = __builtin_amdgcn_raw_buffer_load_b64(rb, at + (s < s1 ? r * ldb_b : 0), 0, 0);
        }
      }
    };
    auto mma = [&](const Step& x) {
      if constexpr (ES == 1) {
        i32x8 fa, fb;
#pragma unroll
        for (int q = 0; q < 8; ++q) fa[q] = x.a[q / 4][q & 3], fb[q] = x.b[q / 4][q & 3];
        acc[0] = M::run(fb, fa, acc[0]);
      } else if constexpr (ES == 4) {
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
          for (int j = 0; j < NJ; ++j) {
            const unsigned fb = TB == 1 ? x.b[0][s] : x.b[TB == 1 ? 0 : s][j], fa = x.a[0][s];
            acc[j] = M::run(__builtin_bit_cast(float, fb), __builtin_bit_cast(float, fa), acc[j]);
          }
      } else if constexpr (TB == 1) {
        acc[0] = M::run(x.b[0], x.a[0], acc[0]);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          u32x4 f;
#pragma unroll
          for (int q = 0; q < 4; ++q)  // column j of rows 2q and 2q + 1
            f[q] = __builtin_amdgcn_perm(x.r[2 * q + 1][j / 2], x.r[2 * q][j / 2], j & 1 ? 0x07060302u : 0x05040100u);
          acc[j] = M::run(f, x.a[0], acc[j]);
        }
      }
    };
    for (int s = s0; s < s1; s += AHEAD) {
      Step x[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) load(x[u], s + u);
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) mma(x[u]);
    }

    // accumulator r of MFMA j: row i of A; column 4 g + r of its 16 (N x K: j = 0), K x N: 16 g + 4 r + j
    typedef __attribute__((address_space(3))) f32x4 lds_f32x4;
    lds_u8* block = smem + wave * (BM * PITCH) + i * PITCH;
    if (i < m) {
      if constexpr (TB == 1) {
        *(lds_f32x4*)(block + g * 16) = acc[0];
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
          *(lds_f32x4*)(block + g * 64 + r * 16) = f32x4{acc[0][r], acc[1][r], acc[2][r], acc[3][r]};
      }
    }
    __syncthreads();
    if constexpr (IsInt8<DT>::v) {
      constexpr int LPR = BN / 8;  // lanes a row
      static_assert(BM * LPR <= 64, "the first wave finishes the rows");
      const int row = tid / LPR, c = n0 + (tid % LPR) * 8;
      if (wave == 0 && row < m) {
        const EpiOut o = ep(item, 0);
        const int left = o.n - c;
        const bool whole = __ballot(left > 0 && left < 8) == 0;
        if (left <= 0) return;
        constexpr int OS = OutSize<DT>::v;
        Row8<DT> res;
        if (o.res)
          res.load(make_rsrc(o.res, ((o.m - 1) * o.ldr + o.n) * OS), (row * o.ldr + c) * OS, whole && (OS == 4 || o.res_vec),
                   left);
        const lds_u8* at = smem + row * PITCH + (tid % LPR) * 32;
        i32x4 lo = {0, 0, 0, 0}, hi = lo;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
          lo += *(const __attribute__((address_space(3))) i32x4*)(at + w * (BM * PITCH));
          hi += *(const __attribute__((address_space(3))) i32x4*)(at + w * (BM * PITCH) + 16);
        }
        put_ints<DT>(__builtin_bit_cast(f32x4, lo), __builtin_bit_cast(f32x4, hi), rs, columns, o.act, res, o.res != nullptr,
                     make_rsrc(o.c, o.c_bytes), (row * o.ldc + c) * OS, whole && (OS == 4 || o.c_vec), left);
      }
      return;
    }
    typedef EpiWave<DT, BM, BN, 1> Epi;
    constexpr int USED = BM * Epi::LPR;  // threads that finish rows: 32 or 128
    const int row = tid / Epi::LPR;
    float* part = nullptr;
    if (tid < USED) {
      Epi x(ep(item, 0), lane);
      x.columns(n0);
      part = x.o.part;
      if (row < m && x.left > 0) {
        Row8<DT> res, aux;
        x.load_inputs(true, row, res, aux);
        const lds_u8* at = smem + row * PITCH + (tid % Epi::LPR) * 32;
        f32x4 lo = {0.0f, 0.0f, 0.0f, 0.0f}, hi = lo;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
          lo += *(const lds_f32x4*)(at + w * (BM * PITCH));
          hi += *(const lds_f32x4*)(at + w * (BM * PITCH) + 16);
        }
        float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        x.finish(true, row, v, res, aux);
      }
      if (part) x.put_sums(smem + TABLE, row, BN, (tid % Epi::LPR) * 8);
    }
    __syncthreads();
    if (part) add_sums<BM>(smem + TABLE, BN, part + n0, min(BN, n), tid);
  }

  // Work item tb of a member (ep_member): column tile tb % tiles_n of batch item tb / tiles_n.
  static __device__ __forceinline__ void run(const KArgs& p, int tb, int gi, lds_u8* smem) {
    const int item = tb / p.tiles_n, n0 = (tb - item * p.tiles_n) * BN;
    const int lda_b = (int)p.lda * ES, ldb_b = (int)p.ldb * ES;
    const uint8_t* b = p.b + item * p.stride_b + (TB == 1 ? (int64_t)n0 * ldb_b : (int64_t)n0 * ES);
    tile(p.a + item * p.stride_a, b, lda_b, ldb_b, (int)p.m, min(BN, (int)p.n - n0), (int)p.k, MemberEpi<1>{gi}, item,
         n0, smem);
  }
};

template <int DT, int TB>
__global__ void __launch_bounds__(512) go_skinny(KLaunch L, KEpis) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[Skinny<DT, TB>::LDS];
  ep_member<512, Skinny<DT, TB>>(L, (lds_u8*)smem);
}

// Products grouped by expert over rows, 16 rows a tile, K of any length: a round of loads
// after the other.
template <int DT, int TB>
__global__ void __launch_bounds__(512) grouped_few(KGroup g) {
  typedef Skinny<DT, TB> T;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[T::LDS];
  constexpr int ES = ElemSize<DT>::v;
  const int tn = (g.n + T::BN - 1) / T::BN;
  const int total = total_slots(g.offsets, g.groups, g.rows, T::BM, g.max_slots) * tn;
  const int per = (total + kXcds - 1) / kXcds;
  const int j = (int)blockIdx.x / kXcds, id = ((int)blockIdx.x & (kXcds - 1)) * per + j;
  if (j >= per || id >= total) return;
  GroupSlot s;
  if (!find_slot(g.offsets, g.groups, g.rows, T::BM, id / tn, s)) return;
  int ti, tj;
  group_tile(id - s.first * tn, (s.count + T::BM - 1) / T::BM, tn, ti, tj);
  GroupEpi e;
  e.e = uniform(s.e), e.row = uniform(s.lo + ti * T::BM), e.n0 = uniform(tj * T::BN);
  e.m = uniform(min(T::BM, s.count - ti * T::BM)), e.n = uniform(min(T::BN, g.n - tj * T::BN));
  e.slot = uniform(s.first + ti), e.os = OutSize<DT>::v, e.over_k = false;
  const uint8_t* a = g.a + (int64_t)e.row * g.lda * ES;
  const uint8_t* b = g.b + e.e * g.stride_b + (TB == 1 ? (int64_t)e.n0 * g.ldb : (int64_t)e.n0) * ES;
  T::tile(a, b, g.lda * ES, g.ldb * ES, e.m, e.n, g.k, e, 0, 0, (lds_u8*)smem);
}

template <int DT> GroupKernel few_kernel(int tb) {
  if (tb)
    return GroupKernel{reinterpret_cast<const void*>(&grouped_few<DT, 1>), kSkinnyRows, Skinny<DT, 1>::BN, 512};
  if constexpr (DT != DT_FP8)
    return GroupKernel{reinterpret_cast<const void*>(&grouped_few<DT, 0>), kSkinnyRows, Skinny<DT, 0>::BN, 512};
  else return GroupKernel{nullptr, 0, 0, 0};
}

template <int DT> const void* skinny_kernel(int tb) {
  if (tb) return reinterpret_cast<const void*>(&go_skinny<DT, 1>);
  if constexpr (DT != DT_FP8) return reinterpret_cast<const void*>(&go_skinny<DT, 0>);
  else return nullptr;
}

}  // namespace gdy
