// experts.h -- what a mixture of experts does around its grouped products: the rows of
// each expert (route), tokens' rows to them (scatter) and back (combine), with the
// gradients of both.
//
// Scatter and combine are bound by memory.  Both go by tokens: a token's row is written once
// (combine), or read once for every four of its pairs (scatter), and its top_k rows of the other
// side next to it, so that nothing but the slots says where rows lie, no atomics are needed
// and every sum has a fixed order.  Scatter's later reads come out of the caches: 4096 rows of
// 4096 bf16 to eight experts each take 60.7 us, 8192 rows to two 40.4, both 5.0 TB/s counting one
// read of each row.
#pragma once
#include "grouped.h"
#include "rows.h"

namespace gdy {

// The weight of a pair.
template <int DT> __device__ __forceinline__ float pair_weight(const void* weights, bool f32, int64_t pair) {
  if (f32) return ((const float*)weights)[pair];
  if constexpr (ElemSize<DT>::v == 2) return ew_decode<DT>(((const uint16_t*)weights)[pair]);
  else return ((const float*)weights)[pair];
}

// ---- rows to the experts ---------------------------------------------------------
// MODE 0: copies, 1: weighted, 2: weighted, with the gradient of the weights.
template <int DT, int MODE>
__global__ void __launch_bounds__(kRowThreads) scatter_rows(KScatter g) {
  typedef RowChunk<DT> C;
  constexpr int JU = 4;  // pairs of a token that are under way together
  __shared__ float lds[MODE == 2 ? kRowThreads / 64 * JU : 1];
  const RowPlace at(g.tpr_log);
  const int step = 1 << g.tpr_log, n = g.n;
  for (int64_t t0 = (int64_t)blockIdx.x * at.rows; t0 < g.tokens; t0 += (int64_t)gridDim.x * at.rows) {
    const int64_t t = t0 + at.sub;
    const bool live = t < g.tokens;
    const uint8_t* x = g.x + (live ? t : 0) * g.ldx;
    for (int j0 = 0; j0 < g.top_k; j0 += JU) {
      int slot[JU];
      float w[JU], dot[JU];
#pragma unroll
      for (int u = 0; u < JU; ++u) {
        const int64_t pair = t * g.top_k + j0 + u;
        const bool in = live && j0 + u < g.top_k;
        slot[u] = in ? g.slots[pair] : -1;
        if ((unsigned)slot[u] >= (unsigned)g.rows) slot[u] = -1;
        w[u] = MODE && in ? pair_weight<DT>(g.weights, g.weights_f32, pair) : 1.0f;
        dot[u] = 0.0f;
      }
      for (int c = at.lane * C::VN; c < n; c += step * C::VN) {
        if (!live) break;
        const int left = n - c;
        C v, z[JU];
        v.load(x + (int64_t)c * C::ES, left);
        if (MODE == 2 && g.rows > 0) {
#pragma unroll
          for (int u = 0; u < JU; ++u)  // pairs without a row read one that is there
            z[u].load(g.z + max(slot[u], 0) * g.ldz + (int64_t)c * C::ES, left);
        }
#pragma unroll
        for (int u = 0; u < JU; ++u) {
          if (slot[u] < 0) continue;
          C o = v;
          if constexpr (MODE != 0) {
            float y[C::VN];
#pragma unroll
            for (int e = 0; e < C::VN; ++e) {
              y[e] = v.get(e) * w[u];
              if (MODE == 2) dot[u] = __builtin_fmaf(v.get(e), z[u].get(e), dot[u]);
            }
            o.set(y);
          }
          o.store(g.out + slot[u] * g.ldo + (int64_t)c * C::ES, left);
        }
      }
      if constexpr (MODE == 2) {
        // the row's threads in a fixed order: halves of a wave's lanes, then its waves
#pragma unroll
        for (int u = 0; u < JU; ++u)
          for (int d = 1; d < min(step, 64); d <<= 1) dot[u] += __shfl_xor(dot[u], d);
        const int wave = (int)threadIdx.x >> 6;
        if (step > 64) {
          if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int u = 0; u < JU; ++u) lds[wave * JU + u] = dot[u];
          __syncthreads();
          if (at.lane == 0)
#pragma unroll
            for (int u = 0; u < JU; ++u)
              for (int q = 1; q < step / 64; ++q) dot[u] += lds[(wave + q) * JU + u];
          __syncthreads();
        }
        if (live && at.lane == 0)
#pragma unroll
          for (int u = 0; u < JU; ++u)
            if (j0 + u < g.top_k) g.weight_grad[t * g.top_k + j0 + u] = slot[u] < 0 ? 0.0f : dot[u];
      }
    }
  }
}

// ---- rows back from them ------------------------------------------------------------
template <int DT>
__global__ void __launch_bounds__(kRowThreads) combine_rows(KCombine g) {
  typedef RowChunk<DT> C;
  constexpr int JU = 4;
  const RowPlace at(g.tpr_log);
  const int step = 1 << g.tpr_log, n = g.n;
  for (int64_t t = (int64_t)blockIdx.x * at.rows + at.sub; t < g.tokens; t += (int64_t)gridDim.x * at.rows) {
    for (int c = at.lane * C::VN; c < n; c += step * C::VN) {
      const int left = n - c;
      float acc[C::VN];
#pragma unroll
      for (int e = 0; e < C::VN; ++e) acc[e] = 0.0f;
      C r;
      if (g.res) r.load(g.res + t * g.ldr + (int64_t)c * C::ES, left);
      for (int j0 = 0; g.rows > 0 && j0 < g.top_k; j0 += JU) {
        int slot[JU];
        float w[JU];
        C z[JU];
#pragma unroll
        for (int u = 0; u < JU; ++u) {
          const int64_t pair = t * g.top_k + min(j0 + u, g.top_k - 1);
          slot[u] = j0 + u < g.top_k ? g.slots[pair] : -1;
          if ((unsigned)slot[u] >= (unsigned)g.rows) slot[u] = -1;
          w[u] = g.weights ? pair_weight<DT>(g.weights, g.weights_f32, pair) : 1.0f;
        }
#pragma unroll
        for (int u = 0; u < JU; ++u)  // pairs without a row read one that is there
          z[u].load(g.z + max(slot[u], 0) * g.ldz + (int64_t)c * C::ES, left);
#pragma unroll
        for (int u = 0; u < JU; ++u) {
          if (slot[u] < 0) continue;
#pragma unroll
          for (int e = 0; e < C::VN; ++e) acc[e] = __builtin_fmaf(w[u], z[u].get(e), acc[e]);
        }
      }
      if (g.res) {
#pragma unroll
        for (int e = 0; e < C::VN; ++e) acc[e] += r.get(e);
      }
      C o;
      o.set(acc);
      o.store(g.y + t * g.ldy + (int64_t)c * C::ES, left);
    }
  }
}

// ---- the rows of each expert -----------------------------------------------------------
// A stable sort by counting.  Its parts are kRoutePart * `steps` consecutive pairs each, a
// workgroup's; a wave takes consecutive pairs, 64 a step, so that the pairs before one are those
// of the parts before, of the waves before, and of the wave's own steps and lanes before.
// Within a step the lanes of one expert find each other by a ballot for each bit of the id.
// All counts are integers: no order of additions matters.
constexpr int kRouteWaves = kRoutePart / 64;

// The expert of pair p (`experts`: none).  Ids are read as dwords; pairs past the last read it.
__device__ __forceinline__ int pair_expert(const KRoute& g, int p) {
  if (g.pairs == 0) return g.experts;  // no last pair to read
  const int q = min(p, g.pairs - 1);
  int64_t at = q;
  if (!g.dense) {
    const int t = q / g.top_k;
    at = t * g.ld_ids + (q - t * g.top_k);
  }
  const int32_t* id = (const int32_t*)g.ids + (at << g.wide);
  const int lo = id[0], hi = id[g.wide];
  const bool in = p < g.pairs && (!g.wide || hi == 0) && (unsigned)lo < (unsigned)g.experts;
  return in ? lo : g.experts;
}

// The lanes of the wave whose expert is this lane's (in: it has one); bits: of the experts' numbers.
__device__ __forceinline__ uint64_t same_expert(int e, bool in, int bits) {
  uint64_t m = __ballot(in);
#pragma unroll 1
  for (int b0 = 0; b0 < bits; b0 += 4) {
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const unsigned bit = ((unsigned)e >> b) & 1;
      const uint64_t has = __ballot(bit);
      const unsigned off = bit - 1;  // all ones where the bit is 0
      m &= has ^ ((uint64_t)off << 32 | off);
    }
    e >>= 4;
  }
  return m;
}

// Pairs of each expert in every part: counts[part][expert].
template <int EXPERTS>
__global__ void __launch_bounds__(kRoutePart) route_count(KRoute g) {
  __shared__ int hist[EXPERTS];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int p = ((int)blockIdx.x * kRouteWaves + wave) * g.steps * 64 + lane;
  int e = pair_expert(g, p);
  for (int i = tid; i < g.experts; i += kRoutePart) hist[i] = 0;
  __syncthreads();
#pragma unroll 1
  for (int s = 0; s < g.steps; ++s) {
    p += 64;
    const int next = s + 1 < g.steps ? pair_expert(g, p) : 0;  // a step ahead
    const uint64_t m = same_expert(e, e < g.experts, g.bits);
    if (e < g.experts && lane == (int)__builtin_ctzll(m)) atomicAdd(&hist[e], (int)__builtin_popcountll(m));
    e = next;
  }
  __syncthreads();
  for (int i = tid; i < g.experts; i += kRoutePart) g.counts[(int64_t)blockIdx.x * g.experts + i] = hist[i];
}

// The parts' counts to those of the parts before, and the totals of every expert.  A workgroup has 64
// experts, a wave consecutive parts.
__global__ void __launch_bounds__(kRoutePart) route_sums(KRoute g) {
  __shared__ int sums[kRouteWaves][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, e = (int)blockIdx.x * 64 + lane;
  const int per = (g.parts + kRouteWaves - 1) / kRouteWaves, q0 = wave * per, q1 = min(q0 + per, g.parts);
  int32_t* c = g.counts + e;
  int x = 0;
  if (e < g.experts) {
#pragma unroll 8
    for (int q = q0; q < q1; ++q) x += c[(int64_t)q * g.experts];
  }
  sums[wave][lane] = x;
  __syncthreads();
  x = 0;
  int total = 0;
  for (int w = 0; w < kRouteWaves; ++w) {
    if (w < wave) x += sums[w][lane];
    total += sums[w][lane];
  }
  if (e >= g.experts) return;
  if (wave == 0) g.totals[e] = total;
#pragma unroll 8
  for (int q = q0; q < q1; ++q) {
    const int here = c[(int64_t)q * g.experts];
    c[(int64_t)q * g.experts] = x;
    x += here;
  }
}

// A wave's LDS accesses are done in the order of its instructions, which this keeps.  (A fence would
// also wait for the loads of the next step.)
__device__ __forceinline__ void lds_in_order() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_wave_barrier();
}

// Slots of a part's pairs, and (the first part) the offsets.  parts == 1: this kernel alone.
// Counts of a wave and expert are 16 bits: a part has fewer than 2^16 pairs.  The only step of
// a wave is ranked once; several are counted, then read and ranked again.  Without totals (route_sums) the
// parts' counts are summed by all threads, `wide` experts next to each other.
// The code is kept short: a call this small waits for its instructions as for its data.
template <int EXPERTS, int WAVES>
__global__ void __launch_bounds__(WAVES * 64) route_slots(KRoute g) {
  constexpr int PART = WAVES * 64;
  __shared__ int base[EXPERTS];
  __shared__ uint16_t count[WAVES][EXPERTS];
  __shared__ int sums[WAVES];
  __shared__ int part_total[PART], part_before[PART];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int E = g.experts;
  const int p0 = ((int)blockIdx.x * WAVES + wave) * g.steps * 64 + lane;
  int e = pair_expert(g, p0);
  for (int i = tid; i < E; i += PART)
#pragma unroll
    for (int w = 0; w < WAVES; ++w) count[w][i] = 0;
  __syncthreads();
  // the rank of a step's pair among the wave's pairs of its expert, on top of `count`
  auto rank = [&](int e) {
    const uint64_t m = same_expert(e, e < E, g.bits);
    int r = 0;
    if (e < E) {
      const int before = count[wave][e];  // read by all lanes of the expert, then written by the first
      r = before + (int)__builtin_popcountll(m & ((1ull << lane) - 1));
      lds_in_order();
      if (lane == (int)__builtin_ctzll(m)) count[wave][e] = (uint16_t)(before + (int)__builtin_popcountll(m));
    }
    lds_in_order();  // before the next step's reads
    return r;
  };
  int first_rank = 0;
  {
    int at = e;
#pragma unroll 1
    for (int s = 0; s < g.steps; ++s) {
      const int next = s + 1 < g.steps ? pair_expert(g, p0 + (s + 1) * 64) : 0;
      const int r = rank(at);
      if (s == 0) first_rank = r;
      at = next;
    }
  }
  // experts, `wide` at a time: counts of the waves before, of the parts before, of the experts before
  const int wide = min(PART, g.expert_threads), rows = PART / wide;
  const int column = tid & (wide - 1), row = tid / wide;
  int below = 0;
#pragma unroll 1
  for (int e0 = 0; e0 < E; e0 += wide) {
    const int x = e0 + column;
    int total = 0, before = 0;
    if (g.parts > 1) {
      if (x < E && g.totals) {
        if (row == 0) before = g.counts[(int64_t)blockIdx.x * E + x], total = g.totals[x];
      } else if (x < E) {
        const int32_t* c = g.counts + (int64_t)row * E + x;
        const int64_t stride = (int64_t)rows * E;
#pragma unroll 16
        for (int q = row; q < g.parts; q += rows, c += stride) {
          before += q < (int)blockIdx.x ? *c : 0;
          total += *c;
        }
      }
      part_total[tid] = total;
      part_before[tid] = before;
    }
    __syncthreads();  // also behind the waves' counts
    total = before = 0;
    const bool mine = row == 0 && x < E;
    if (mine) {
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        const int c = count[w][x];
        count[w][x] = (uint16_t)total;
        total += c;
      }
      if (g.parts > 1) {
        total = 0;
        for (int r = 0; r < rows; ++r) {
          total += part_total[r * wide + tid];
          before += part_before[r * wide + tid];
        }
      }
    }
    const int upto = wave_scan(total);  // of the wave's experts, this one among them
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    int first = below + upto - total;
    for (int w = 0; w < WAVES; ++w) {
      if (w < wave) first += sums[w];
      below += sums[w];
    }
    if (mine) {
      base[x] = first + before;
      if (blockIdx.x == 0) g.offsets[x] = first;
    }
    __syncthreads();
  }
  if (blockIdx.x == 0 && tid == 0) g.offsets[E] = below;
  if (g.steps == 1) {
    if (p0 < g.pairs) g.slots[p0] = e < E ? base[e] + count[wave][e] + first_rank : -1;
    return;
  }
#pragma unroll 1
  for (int s = 0; s < g.steps; ++s) {
    const int p = p0 + s * 64, next = s + 1 < g.steps ? pair_expert(g, p + 64) : 0;
    const int r = rank(e);
    if (p < g.pairs) g.slots[p] = e < E ? base[e] + r : -1;
    e = next;
  }
}

}  // namespace gdy
