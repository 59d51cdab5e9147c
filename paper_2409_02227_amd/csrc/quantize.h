// quantize.h -- rows to 8-bit integers with a scale for each: scale = max |x| / 127, q =
// 127 x / max |x| rounded to the nearest integer.
//
// Bound by memory: a row is read once, kept in registers between its maximum and its codes
// (up to 16384 elements, in launches of at most four rows a CU up to 32768; of longer rows the rest
// is read again), 16 elements a thread and step, and written 16 bytes a lane.  (4096, 8192) 22.7 to 24.6 us in bf16, 4.1
// to 4.4 TB/s, and 32.4 in fp32, 5.2 TB/s: the 16-bit types still show their arithmetic (with the exact rounding of
// fp32 28.8, by three operations a code more 30.4).  The next row's loads in front of a row's arithmetic: 34, for the
// waves that their registers cost.
//
// The quotient is rounded exactly.  x times the fp32 of 127 / max is off by at most 127 * 2^-24 <
// 1e-5, so only values that close to a half can fall on its wrong side.  Those of fp32 rows compare 127 x -
// q max with max / 2: the two products are sums of two floats each, the difference of the
// leading ones is exact (they lie within a factor of two of each other, or q is 0), as is
// its difference from max / 2, which it is close to, and the trailing ones are few bits.
#pragma once
#include "rows.h"

namespace gdy {

// A power of two that keeps every product with rows of this maximum in range.
__device__ __forceinline__ float quant_range(float most) {
  return most < 0x1p-100f ? 0x1p100f : most > 0x1p100f ? 0x1p-100f : 1.0f;
}

// 127 x / most to the nearest integer, halves to even; q: the nearest one to about 1e-4.
__device__ __forceinline__ float quant_exact(float x, float most, float q) {
#pragma clang fp contract(off)
  const float u = 127.0f * x, v = __builtin_fmaf(127.0f, x, -u);
  const float p = q * most, e = __builtin_fmaf(q, most, -p);
  const float lead = u - p, half = 0.5f * most;
  const float above = (lead - half) + (v - e), below = (lead + half) + (v - e);  // signs of (127 x / most - q) -+ 1/2
  const bool odd = 2.0f * __builtin_rintf(0.5f * q) != q;
  q += (above > 0.0f) | ((above == 0.0f) & odd) ? 1.0f : 0.0f;
  q -= (below < 0.0f) | ((below == 0.0f) & odd) ? 1.0f : 0.0f;
  return q;
}
// The same for 16-bit values.  x = X 2^s and most = M of at most 11 bits: 127 X 2^s / M is a half or at least
// 2^s / M, 2^-18 of itself, away from one, and x * r is off by 2^-23 of itself, so q is right but for halves; 127 x -
// q most is exact.  Half of the largest value is a half: of 1024 normal bf16 values one is, more often than not.
__device__ __forceinline__ float quant_even(float x, float most, float q) {
  const float rest = __builtin_fmaf(-q, most, 127.0f * x);
  const bool half = __builtin_fabsf(rest) * 2.0f == most, odd = ((int)q & 1) != 0;
  return (half & odd) ? q + __builtin_copysignf(1.0f, rest) : q;
}

// 16 elements of a row.  WHOLE: rows are whole units.
template <int DT, bool WHOLE> struct QuantUnit {
  typedef RowChunk<DT> C;
  static constexpr int N = 16, NC = N / C::VN;
  C c[NC];
  __device__ __forceinline__ void load(const uint8_t* x, int first, int n) {
    const uint8_t* p = x + (int64_t)first * C::ES;
    const int bytes = (n - first) * C::ES;  // of the row, from here on
#pragma unroll
    for (int q = 0; q < NC; ++q) {
      if (WHOLE || bytes >= 16 * (q + 1)) c[q].w = *(const u32x4_any*)(p + 16 * q);
      else c[q].w = load_part(p + 16 * q, max(bytes - 16 * q, 0));
    }
  }
  __device__ __forceinline__ float get(int e) const { return c[e / C::VN].get(e % C::VN); }
  // the largest |x|, as bits of a float: NaN above infinity above every number
  __device__ __forceinline__ unsigned most() const {
    if constexpr (C::ES == 4) {
      unsigned m = 0;
#pragma unroll
      for (int e = 0; e < N; ++e) m = max(m, c[e / 4].w[e & 3] & 0x7fffffffu);
      return m;
    } else {  // two at a time
      typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
      u16x2 m = {0, 0};
#pragma unroll
      for (int d = 0; d < N / 2; ++d)
        m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, c[d / 4].w[d & 3] & 0x7fff7fffu));
      return __builtin_bit_cast(unsigned, ew_decode<DT>(max(m[0], m[1])));
    }
  }
  // The codes, r = 127 / (most * by) rounded.  A product on top of 3 * 2^22 is rounded to a whole
  // number, whose last byte is the code; a row that needs `by` takes the exact way.
  __device__ __forceinline__ u32x4 codes(float most, float by, float r) const {
    constexpr float kWhole = 12582912.0f;
    u32x4 w;
    float far = by == 1.0f ? 0.0f : 1.0f;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      float y[4];
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const float x = get(4 * d + b);
        y[b] = __builtin_fmaf(x, r, kWhole);
        far = __builtin_fmaxf(far, __builtin_fabsf(__builtin_fmaf(x, r, kWhole - y[b])));
      }
      w[d] = bytes(__builtin_bit_cast(int, y[0]), __builtin_bit_cast(int, y[1]), __builtin_bit_cast(int, y[2]),
                   __builtin_bit_cast(int, y[3]));
    }
    if (far > 0.49999f) {
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        int q[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const float x = get(4 * d + b) * by;
          const float near = __builtin_rintf(x * r);
          q[b] = (int)(C::ES == 2 ? quant_even(x, most * by, near) : quant_exact(x, most * by, near));
          if (C::ES == 4) __builtin_amdgcn_sched_barrier(0);  // one value's registers at a time
        }
        w[d] = bytes(q[0], q[1], q[2], q[3]);
      }
    }
    return w;
  }
  static __device__ __forceinline__ unsigned bytes(int a, int b, int c, int d) {  // the last ones
    return __builtin_amdgcn_perm((unsigned)b, (unsigned)a, 0x0c0c0400u) |
           __builtin_amdgcn_perm((unsigned)d, (unsigned)c, 0x04000c0cu);
  }
};

// A row: 1 << tpr_log threads, 16 elements a thread and step; HELD steps are kept, and are all
// but for kQuantMost.
template <int DT, int HELD, bool WHOLE>
__global__ void __launch_bounds__(HELD == kQuantMost ? kRowThreads : 1024, HELD == 1 && (WHOLE || DT != DT_F32) ? 8 : 1)
quantize_rows(KQuantize g) {
  typedef QuantUnit<DT, WHOLE> Unit;
  constexpr int SLOTS = 2;  // rows of q that are known before the maximum is
  __shared__ unsigned lds[16];
  const int step = 1 << g.tpr_log, n = g.n;
  const int lane = (int)threadIdx.x & (step - 1), sub = (int)threadIdx.x >> g.tpr_log, rows = (int)blockDim.x >> g.tpr_log;
  const int first = lane * Unit::N, pitch = step * Unit::N;
  for (int64_t t0 = (int64_t)blockIdx.x * rows; t0 < g.rows; t0 += (int64_t)gridDim.x * rows) {
    const int64_t t = t0 + sub;
    const bool live = t < g.rows;
    const int end = live ? n : 0;
    const uint8_t* x = g.x + t * g.ldx;
    Unit held[HELD];
#pragma unroll
    for (int h = 0; h < HELD; ++h)
      if (first + h * pitch < end) held[h].load(x, first + h * pitch, n);
    int slot[SLOTS];
#pragma unroll
    for (int j = 0; j < SLOTS; ++j) slot[j] = g.slots && live && j < g.top_k ? g.slots[t * g.top_k + j] : -1;
    unsigned m = 0;
#pragma unroll
    for (int h = 0; h < HELD; ++h)
      if (first + h * pitch < end) m = max(m, held[h].most());
    for (int c = first + HELD * pitch; HELD == kQuantMost && c < end; c += pitch) {
      Unit u;
      u.load(x, c, n);
      m = max(m, u.most());
    }
    for (int d = 1; d < min(step, 64); d <<= 1) m = max(m, (unsigned)__shfl_xor((int)m, d));
    if (step > 64) {
      const int wave = (int)threadIdx.x >> 6, w0 = wave & ~(step / 64 - 1);
      __syncthreads();  // the maxima of the rows before are read
      if ((threadIdx.x & 63) == 0) lds[wave] = m;
      __syncthreads();
      for (int q = 0; q < step / 64; ++q) m = max(m, lds[w0 + q]);
    }
    const float most = __builtin_bit_cast(float, m);
    const bool finite = m < 0x7f800000u;
    const float by = quant_range(most), scale = most / 127.0f;
    const float r = finite && m ? 127.0f / (most * by) : 0.0f;
    // f(a row of q): each one that this row goes to
    auto each = [&](auto f) {
      if (!g.slots) {
        f(t);
        return;
      }
#pragma unroll
      for (int j = 0; j < SLOTS; ++j)
        if ((unsigned)slot[j] < (unsigned)g.out_rows) f((int64_t)slot[j]);
      for (int j = SLOTS; j < g.top_k; ++j) {
        const int s = g.slots[t * g.top_k + j];
        if ((unsigned)s < (unsigned)g.out_rows) f((int64_t)s);
      }
    };
    auto write = [&](const Unit& u, int c) {
      RowChunk<DT_FP8> o;  // bytes
      o.w = u.codes(most, by, r);
      if (!finite) o.w = u32x4{0u, 0u, 0u, 0u};
      each([&](int64_t to) { o.store((uint8_t*)g.q + to * g.ldq + c, WHOLE ? 16 : n - c); });
    };
    if (live && lane == 0) each([&](int64_t to) { g.scales[to] = scale; });
#pragma unroll
    for (int h = 0; h < HELD; ++h)
      if (first + h * pitch < end) write(held[h], first + h * pitch);
    for (int c = first + HELD * pitch; HELD == kQuantMost && c < end; c += pitch) {
      Unit u;
      u.load(x, c, n);
      write(u, c);
    }
  }
}

}  // namespace gdy
