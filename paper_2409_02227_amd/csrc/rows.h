// rows.h -- what the operators by token share: 16 bytes of a row at any alignment, and
// how a workgroup's threads share rows.
#pragma once
#include "go_kernel.h"

namespace gdy {

// Rows may start at any element: loads and stores of several bytes need no alignment.
typedef u32x4 u32x4_any __attribute__((aligned(1)));
typedef u32x2 u32x2_any __attribute__((aligned(1)));
typedef unsigned u32_any __attribute__((aligned(1)));
typedef uint16_t u16_any __attribute__((aligned(1)));

// The first `bytes` of 16 bytes, by one access for each bit of the number.
__device__ __forceinline__ u32x4 load_part(const uint8_t* p, int bytes) {
  u32x4 w = {0u, 0u, 0u, 0u};
  if (bytes & 8) {
    const u32x2 x = *(const u32x2_any*)p;
    w[0] = x[0], w[1] = x[1];
  }
  unsigned y = 0;  // the dword that is not whole
  if (bytes & 4) {
    const unsigned x = *(const u32_any*)(p + (bytes & 8));
    w[0] = bytes & 8 ? w[0] : x;
    w[2] = bytes & 8 ? x : 0u;
  }
  if (bytes & 2) y = *(const u16_any*)(p + (bytes & 12));
  if (bytes & 1) y |= (unsigned)p[bytes & 14] << (8 * (bytes & 2));
  const int at = bytes >> 2;
  w[0] = at == 0 ? y : w[0], w[1] = at == 1 ? y : w[1], w[2] = at == 2 ? y : w[2], w[3] = at == 3 ? y : w[3];
  return w;
}
__device__ __forceinline__ void store_part(uint8_t* p, u32x4 w, int bytes) {
  const int at = bytes >> 2;
  const unsigned y = at == 0 ? w[0] : at == 1 ? w[1] : at == 2 ? w[2] : w[3];
  if (bytes & 8) *(u32x2_any*)p = u32x2{w[0], w[1]};
  if (bytes & 4) *(u32_any*)(p + (bytes & 8)) = bytes & 8 ? w[2] : w[0];
  if (bytes & 2) *(u16_any*)(p + (bytes & 12)) = (uint16_t)y;
  if (bytes & 1) p[bytes & 14] = (uint8_t)(y >> (8 * (bytes & 2)));
}

// 16 bytes of a row, VN elements; ES 1 stands for bytes that are copied.  left: the row's
// elements from these on.
template <int DT> struct RowChunk {
  static constexpr int ES = ElemSize<DT>::v, VN = 16 / ES;
  u32x4 w;
  __device__ __forceinline__ void load(const uint8_t* p, int left) {
    if (left >= VN) w = *(const u32x4_any*)p;
    else w = load_part(p, left * ES);
  }
  __device__ __forceinline__ void store(uint8_t* p, int left) const {
    if (left >= VN) *(u32x4_any*)p = w;
    else store_part(p, w, left * ES);
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
