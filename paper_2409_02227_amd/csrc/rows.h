// rows.h -- what the operators by token share: 16 bytes of a row at any alignment, and
// how a workgroup's threads share rows.
#pragma once
#include "go_kernel.h"

namespace gdy {

// Rows may start at any element: loads and stores of 16 bytes need no alignment.
typedef u32x4 u32x4_any __attribute__((aligned(1)));

// VN elements of a row; ES 1 stands for bytes that are copied.
template <int DT> struct RowChunk {
  static constexpr int ES = ElemSize<DT>::v, VN = 16 / ES;
  u32x4 w;
  __device__ __forceinline__ void load(const uint8_t* p, int left) {
    if (left >= VN) {
      w = *(const u32x4_any*)p;
    } else {
      w = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
      for (int e = 0; e < VN; ++e)
        if (e < left) {
          unsigned x;
          if constexpr (ES == 4) x = ((const unsigned*)p)[e];
          else if constexpr (ES == 2) x = ((const uint16_t*)p)[e];
          else x = p[e];
          w[e * ES / 4] |= x << ((e * ES * 8) & 31);
        }
    }
  }
  __device__ __forceinline__ void store(uint8_t* p, int left) const {
    if (left >= VN) {
      *(u32x4_any*)p = w;
    } else {
#pragma unroll
      for (int e = 0; e < VN; ++e)
        if (e < left) {
          const unsigned x = w[e * ES / 4] >> ((e * ES * 8) & 31);
          if constexpr (ES == 4) ((unsigned*)p)[e] = x;
          else if constexpr (ES == 2) ((uint16_t*)p)[e] = (uint16_t)x;
          else p[e] = (uint8_t)x;
        }
    }
  }
  __device__ __forceinline__ float get(int e) const {
    const unsigned x = w[e * ES / 4];
    return ew_decode<DT>(ES == 4 ? x : (x >> ((e * ES * 8) & 31)) & 0xffffu);
  }
  __device__ __forceinline__ void set(const float (&x)[VN]) {
    if constexpr (ES == 4) {
#pragma unroll
      for (int e = 0; e < VN; ++e) w[e] = __builtin_bit_cast(unsigned, x[e]);
    } else {
#pragma unroll
      for (int e = 0; e < VN; e += 2) w[e / 2] = to_out2<DT>(x[e], x[e + 1]);
    }
  }
};

// Threads of a workgroup of kRowThreads share rows: 1 << log2 of them a row.
struct RowPlace {
  int lane, sub, rows;  // this thread's place in its row, its row in the workgroup, rows of a workgroup
  __device__ __forceinline__ RowPlace(int tpr_log)
      : lane((int)threadIdx.x & ((1 << tpr_log) - 1)), sub((int)threadIdx.x >> tpr_log), rows(kRowThreads >> tpr_log) {}
};

}  // namespace gdy
