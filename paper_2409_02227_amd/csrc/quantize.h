// quantize.h -- rows to 8-bit integers with a scale for each: scale = max |x| / 127, q =
// 127 x / max |x| rounded to the nearest integer.
//
// The quotient is rounded exactly: x * (127 / max) in fp32 is off by at most 127 * 2^-23 < 2e-5,
// so only values that close to a half can fall on its wrong side, and those compare
// 127 x with half * max, each product exact as a sum of two floats.
#pragma once
#include "rows.h"

namespace gdy {

constexpr int kQuantHeld = 4;  // units of 16 elements that a thread keeps between the maximum and the codes

// `x` times a power of two that keeps every product below in range (rows whose largest value
// is far from 1).
__device__ __forceinline__ float quant_range(float most) {
  return most < 0x1p-100f ? 0x1p100f : most > 0x1p100f ? 0x1p-100f : 1.0f;
}

// 127 x / most to the nearest integer: the nearest one to x * r (r = 127 / most rounded), unless
// that lies close to a half (`near`).
__device__ __forceinline__ float quant_near(float x, float r, bool& near) {
  const float t = x * r, q = __builtin_rintf(t);
  near |= __builtin_fabsf(t - q) > 0.49998f;
  return q;
}
// The same next to a half as elsewhere.
__device__ __forceinline__ float quant_exact(float x, float most, float r) {
#pragma clang fp contract(off)
  const float t = x * r, q = __builtin_rintf(t);
  const float half = q + (t > q ? 0.5f : -0.5f);  // the nearest half
  const float p = half * most, e = __builtin_fmaf(half, most, -p);
  const float u = 127.0f * x, v = __builtin_fmaf(127.0f, x, -u);
  const float over = (u - p) + (v - e);  // 127 x - half * most: every step is exact where it counts
  const float lo = half - 0.5f, hi = half + 0.5f;
  const float even = 2.0f * __builtin_rintf(0.5f * lo) == lo ? lo : hi;
  const float by = over < 0.0f ? lo : over > 0.0f ? hi : even;
  return __builtin_fabsf(t - q) > 0.49998f ? by : q;
}

// A row: 1 << tpr_log threads, 16 elements a thread and step.
template <int DT>
__global__ void __launch_bounds__(kRowThreads) quantize_rows(KQuantize g) {
  typedef RowChunk<DT> C;
  constexpr int UNIT = 16, NC = UNIT / C::VN;  // chunks of a unit
  __shared__ unsigned lds[kRowThreads / 64];
  const RowPlace at(g.tpr_log);
  const int step = 1 << g.tpr_log, n = g.n;
  struct Unit {
    C c[NC];
    __device__ __forceinline__ void load(const uint8_t* x, int first, int n) {
#pragma unroll
      for (int q = 0; q < NC; ++q) c[q].load(x + (int64_t)(first + q * C::VN) * C::ES, n - first - q * C::VN);
    }
    __device__ __forceinline__ float get(int e) const { return c[e / C::VN].get(e % C::VN); }
    // the largest |x| as bits: NaN above infinity above every number
    __device__ __forceinline__ unsigned most() const {
      unsigned m = 0;
#pragma unroll
      for (int e = 0; e < UNIT; ++e) m = max(m, __builtin_bit_cast(unsigned, get(e)) & 0x7fffffffu);
      return m;
    }
  };
  for (int64_t t0 = (int64_t)blockIdx.x * at.rows; t0 < g.rows; t0 += (int64_t)gridDim.x * at.rows) {
    const int64_t t = t0 + at.sub;
    const bool live = t < g.rows;
    const uint8_t* x = g.x + (live ? t : 0) * g.ldx;
    const int first = at.lane * UNIT, pitch = step * UNIT, end = live ? n : 0;
    Unit held[kQuantHeld];
    unsigned m = 0;
#pragma unroll
    for (int h = 0; h < kQuantHeld; ++h)
      if (first + h * pitch < end) held[h].load(x, first + h * pitch, n);
#pragma unroll
    for (int h = 0; h < kQuantHeld; ++h)
      if (first + h * pitch < end) m = max(m, held[h].most());
    for (int c = first + kQuantHeld * pitch; c < end; c += pitch) {
      Unit u;
      u.load(x, c, n);
      m = max(m, u.most());
    }
    for (int d = 1; d < min(step, 64); d <<= 1) m = max(m, (unsigned)__shfl_xor((int)m, d));
    if (step > 64) {
      const int wave = (int)threadIdx.x >> 6, w0 = wave & ~(step / 64 - 1);
      if ((threadIdx.x & 63) == 0) lds[wave] = m;
      __syncthreads();
      for (int q = 0; q < step / 64; ++q) m = max(m, lds[w0 + q]);
      __syncthreads();
    }
    const float top = __builtin_bit_cast(float, m);
    const bool finite = m < 0x7f800000u;
    const float by = quant_range(top), most = top * by;
    const float r = finite && m ? 127.0f / most : 0.0f;
    const float scale = top / 127.0f;
    auto write = [&](const Unit& u, int c) {
      float code[UNIT];
      bool near = false;
#pragma unroll
      for (int e = 0; e < UNIT; ++e) code[e] = quant_near(finite ? u.get(e) * by : 0.0f, r, near);
      if (near) {  // one wave in 25 takes this, of 1024 values spread evenly
#pragma unroll
        for (int e = 0; e < UNIT; ++e) code[e] = quant_exact(finite ? u.get(e) * by : 0.0f, most, r);
      }
      u32x4 codes;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        unsigned v = 0;
#pragma unroll
        for (int b = 0; b < 4; ++b) v |= (unsigned)((int)code[4 * w + b] & 255) << (8 * b);
        codes[w] = v;
      }
      RowChunk<DT_FP8> o;
      o.w = codes;
      if (!g.slots) {
        o.store((uint8_t*)g.q + t * g.ldq + c, n - c);
      } else {
        for (int j = 0; j < g.top_k; ++j) {
          const int s = g.slots[t * g.top_k + j];
          if ((unsigned)s < (unsigned)g.out_rows) o.store((uint8_t*)g.q + s * g.ldq + c, n - c);
        }
      }
    };
    if (live && at.lane == 0) {
      if (!g.slots) {
        g.scales[t] = scale;
      } else {
        for (int j = 0; j < g.top_k; ++j) {
          const int s = g.slots[t * g.top_k + j];
          if ((unsigned)s < (unsigned)g.out_rows) g.scales[s] = scale;
        }
      }
    }
#pragma unroll
    for (int h = 0; h < kQuantHeld; ++h)
      if (first + h * pitch < end) write(held[h], first + h * pitch);
    for (int c = first + kQuantHeld * pitch; c < end; c += pitch) {
      Unit u;
      u.load(x, c, n);
      write(u, c);
    }
  }
}

}  // namespace gdy
