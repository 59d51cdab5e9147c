// act_grad.h -- gradients around a linear layer that no product precedes: dz = dy *
// f'(z) and the column sums of dz (over all rows, or over the rows of each group),
// and the sums that finish every bias gradient of the library.
//
// Bound by memory: dy and z are read once and dz written once, 16 bytes a lane.  A
// workgroup of 512 threads takes 32 rows, four a thread, all loaded before the first
// is computed, and ends: workgroups that loop over 64 rows (256 threads) are all
// resident at once and load, compute and store in step ((8192, 4096) bf16 gelu 54 us, 41.8
// this way, 4.8 TB/s; 16 rows 40.7; with the column sums 55.6, 48.2 and 48.0; (16384, 8192)
// silu 154, 138 and 136, with sums 161, 151 and 156: 16 rows write twice the partial sums).
// Sums over many rows are split: each workgroup writes one row of partial sums,
// bias_sums or group_sums adds them in order (no atomics: the result does not
// depend on the run).
#pragma once
#include "grouped.h"

namespace gdy {

// Sums of COLS columns by LANES lanes of rows, added in order.  Many rows: 16 x 64, so
// that there are workgroups and rows in flight enough that each waits for memory
// about once (512 rows of 4096: with its launch 6.8 us, as on 64 x 16); few rows: 64 x 4
// (16 groups of about 6 rows of 1536: with the sums' kernel 16.4 us, on 16 x 64 22.6).
template <int COLS, int LANES>
__device__ __forceinline__ void column_sums(const float* part, float* out, int n, int rows, int col, float* lds) {
  const int lane = threadIdx.x % COLS, q = threadIdx.x / COLS;
  const bool live = col + lane < n;
  float x = 0.0f;
  if (live) {
    const float* p = part + col + lane;
#pragma unroll 8
    for (int r = q; r < rows; r += LANES) x += p[(int64_t)r * n];
  }
  lds[threadIdx.x] = x;
  __syncthreads();
  if (q == 0 && live) {
#pragma unroll
    for (int w = 1; w < LANES; ++w) x += lds[w * COLS + lane];
    out[col + lane] = x;
  }
}

// One work item a workgroup, more where a grid of one each would pass 2^32 threads.
template <int COLS, int LANES>
__global__ void __launch_bounds__(COLS * LANES) bias_sums(BiasSums s) {
  __shared__ float lds[COLS * LANES];
  for (int w = (int)blockIdx.x; w < s.first[s.count]; w += (int)gridDim.x) {
    if (w != (int)blockIdx.x) __syncthreads();  // the item before has read the sums
    int u = 0;
    while (u + 1 < s.count && w >= s.first[u + 1]) ++u;
    const int blocks = (s.n[u] + COLS - 1) / COLS, b = w - s.first[u];
    const int item = b / blocks;
    column_sums<COLS, LANES>(s.part[u] + (int64_t)item * s.rows[u] * s.n[u], s.out[u] + item * s.stride[u], s.n[u],
                             s.rows[u], (b - item * blocks) * COLS, lds);
  }
}

// The sums of group e, or of all groups (GroupSums::shared).
template <int COLS, int LANES>
__global__ void __launch_bounds__(COLS * LANES) group_sums(GroupSums s) {
  __shared__ float lds[COLS * LANES];
  const int blocks = (s.n + COLS - 1) / COLS, e = (int)blockIdx.x / blocks;
  const int col = ((int)blockIdx.x - e * blocks) * COLS;
  int first = 0, count;
  if (s.shared) {
    count = total_slots(s.offsets, s.groups, s.rows, s.bm, s.max_slots);
  } else {
    first = first_slot(s.offsets, s.groups, s.rows, s.bm, e);
    const GroupRows g = group_rows(s.offsets, s.groups, s.rows, e);
    count = min((g.count + s.bm - 1) / s.bm, max(s.max_slots - first, 0));
  }
  column_sums<COLS, LANES>(s.part + (int64_t)first * s.per * s.n, s.out + e * s.stride, s.n, count * s.per, col, lds);
}

// A workgroup: bm rows of a group x kActCols columns, a lane eight consecutive ones.
template <int DT>
__global__ void __launch_bounds__(kActThreads) act_grad(KActGrad g) {
  constexpr int OS = OutSize<DT>::v, LPR = kActCols / 8, RP = kActThreads / LPR, AHEAD = kActRows / RP;
  __shared__ __attribute__((aligned(16))) float lds[kActThreads * 8];
  const int tn = (g.n + kActCols - 1) / kActCols;
  const int slot = (int)blockIdx.x / tn, n0 = ((int)blockIdx.x - slot * tn) * kActCols;
  GroupSlot s = {0, 0, g.rows, 0};
  if (g.offsets && !find_slot(g.offsets, g.groups, g.rows, g.bm, slot, s)) return;
  const int r_lo = (slot - s.first) * g.bm;
  const int m = uniform(min(g.bm, s.count - r_lo)), row = uniform(s.lo + r_lo);
  const int cols = min(kActCols, g.n - n0);
  // this tile of each matrix
  auto tile = [&](const uint8_t* p, int ld) {
    return make_rsrc(p ? p + ((int64_t)row * ld + n0) * OS : nullptr, p ? ((m - 1) * ld + cols) * OS : 0);
  };
  const Rsrc ry = tile(g.dy, g.lddy), rz = tile(g.z, g.ldz), rd = tile(g.dz, g.lddz);
  const int tid = threadIdx.x, c8 = (tid % LPR) * 8, left = cols - c8;
  const bool whole = left >= 8, y_vec = whole && (OS == 4 || g.dy_vec), z_vec = whole && (OS == 4 || g.z_vec),
             d_vec = whole && (OS == 4 || g.dz_vec);
  float sum[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
  if (left > 0) {
    for (int r0 = tid / LPR; r0 < m; r0 += RP * AHEAD) {
      Row8<DT> y[AHEAD], z[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int r = r0 + u * RP;
        if (r >= m) break;
        y[u].load(ry, (r * g.lddy + c8) * OS, y_vec, left);
        if (g.z) z[u].load(rz, (r * g.ldz + c8) * OS, z_vec, left);
      }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int r = r0 + u * RP;
        if (r >= m) break;
        float x[8];
        y[u].get(x);
        if (g.z) {
          float v[8];
          z[u].get(v);
          apply_slopes(x, v, g.act);
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) sum[q] += x[q];
        if (g.dz) {
          Row8<DT> w;
          w.set(x);
          w.store(rd, (r * g.lddz + c8) * OS, d_vec, left);
        }
      }
    }
  }
  if (!g.part) return;
#pragma unroll
  for (int q = 0; q < 8; ++q) lds[(tid / LPR) * kActCols + c8 + q] = sum[q];
  __syncthreads();
  for (int c = tid; c < cols; c += kActThreads) {
    float x = lds[c];
#pragma unroll
    for (int r = 1; r < RP; ++r) x += lds[r * kActCols + c];
    g.part[(int64_t)slot * g.n + n0 + c] = x;
  }
}

}  // namespace gdy
