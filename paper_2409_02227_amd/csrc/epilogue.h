// epilogue.h -- what a GEMM does with its fp32 sums before the one rounding:
//   z = scale * sum + bias(j);   aux(i,j) = round(z);   C = round(f(z) + R(i,j))
// or, backward (grad), with the saved pre-activation aux read:
//   g = (scale * sum + bias(j)) * f'(aux(i,j));   C = round(g + R(i,j))
// and the column sums of the unrounded C, from which bias gradients are made.
//
// Each wave passes its accumulators through LDS of its own as fp32 rows (32 or 64
// at a time, in the room of the operand stages), so that a lane owns eight
// consecutive columns: the residual and the saved pre-activation are read, and C
// written, with 16 consecutive bytes a lane, the bias stays in registers, and one
// rolled loop holds the activations, where the accumulators' order would need them
// unrolled over every block.  Nothing is rounded between the sum and C.  No barrier
// separates the waves, so that one's arithmetic runs beside another's stores.
#pragma once
#include <stddef.h>

#include <type_traits>

#include "lds_copy.h"

namespace gdy {

// Where a tile's results go: the matrix (an item of a batch, or a group's rows) and
// its epilogue, pointers at its first element.
struct EpiOut {
  uint8_t* c;
  int c_bytes, ldc, m, n;  // m, n: rows and columns of the matrix
  bool c_vec;
  float scale;
  const uint8_t *bias, *res;
  uint8_t* aux;
  float* part;  // the tile's row of column sums (null: none)
  int ldr, ldaux, act;
  bool bias_f32, grad, res_vec, aux_vec;
  // C = round(scale * sum + bias) alone: the rounded tile goes through LDS as the plain
  // kernels', two bytes an element and whole rows a store ((4813, 8064, 320) bf16 on
  // 128 x 128 tiles: 56.6 us by EpiWave, 46.3 this way, 41.9 without a bias; over K, 64
  // groups of 1024 rows in all, 2048 x 1024 each: 100 and 77).
  __device__ __forceinline__ bool linear() const { return act == ACT_NONE && !res && !aux && !part; }
};

// Kernels without epilogues.
struct NoEpi {
  static constexpr bool on = false;
};

// The member gi of a kernel whose arguments are (KLaunch, KEpis).  Read when a
// tile's sums are done: the empty asm hides the pointer's origin from the compiler
// there, which would otherwise load the fields before the tile loop and keep them
// in registers through it (scalars then spill to scratch memory).
// AHEAD: the rows whose residual and saved pre-activation a wave loads together.
// LINEAR: whether linear epilogues have a path of their own (not in the kernels of mixed
// 256 x 256 or fp8 members, whose registers it would pass).
template <int AHEAD, bool LINEAR = true> struct MemberEpi {
  static constexpr bool on = true, linear = LINEAR;
  static constexpr int ahead = AHEAD;
  static constexpr int kAt = (sizeof(KLaunch) + alignof(KEpis) - 1) / alignof(KEpis) * alignof(KEpis);
  typedef const __attribute__((address_space(4))) uint8_t* Ptr;
  int gi;
  __device__ __forceinline__ EpiOut operator()(int item, int tile_row) const {
    Ptr args = (Ptr)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(args));
    const auto* a = (const __attribute__((address_space(4))) KArgs*)(args + offsetof(KLaunch, g)) + gi;
    const auto* e = (const __attribute__((address_space(4))) KEpi*)(args + kAt) + gi;
    EpiOut o;
    o.c = a->c + item * a->stride_c;
    o.c_bytes = a->c_bytes, o.ldc = (int)a->ldc, o.m = (int)a->m, o.n = (int)a->n;
    o.c_vec = a->c_vec != 0, o.scale = a->scale;
    o.bias = e->bias ? e->bias + item * e->stride_bias : nullptr;
    o.res = e->res ? e->res + item * e->stride_res : nullptr;
    o.aux = e->aux ? e->aux + item * e->stride_aux : nullptr;
    o.part = e->part ? e->part + ((int64_t)item * e->part_rows + tile_row) * o.n : nullptr;
    o.ldr = e->ldr, o.ldaux = e->ldaux, o.act = e->act;
    o.bias_f32 = e->bias_f32 != 0, o.grad = e->grad != 0, o.res_vec = e->res_vec != 0, o.aux_vec = e->aux_vec != 0;
    return o;
  }
};

// ---- activations --------------------------------------------------------------
constexpr float kLog2e = 1.4426950408889634f;

// 1 / (1 + 2^y): the logistic function of -y / log2(e); 0 where 2^y overflows.
__device__ __forceinline__ float logistic2(float y) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(y));
}

// exp(-a^2 / 2) and Q(a) = erfcx(a / sqrt 2) / 2 for a >= 0: the normal distribution
// function is Phi(-a) = exp(-a^2 / 2) Q(a).  Q is a polynomial in t = 1 / (1 + 0.3 a),
// fitted to the least largest relative error on [0, 14] (4.6e-7 evaluated in fp32):
// small Phi keep their relative precision, which 1 + erf loses.
__device__ __forceinline__ float mills(float a, float& bell) {
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3f, a, 1.0f));
  float q = 0.03567638332048663f;
  q = __builtin_fmaf(q, t, -0.15720967723673793f);
  q = __builtin_fmaf(q, t, 0.20636469940526767f);
  q = __builtin_fmaf(q, t, -0.053693808301125495f);
  q = __builtin_fmaf(q, t, 0.12856693977021838f);
  q = __builtin_fmaf(q, t, 0.0999118991526421f);
  q = __builtin_fmaf(q, t, 0.12075420880971754f);
  q = __builtin_fmaf(q, t, 0.11962928249451463f);
  bell = __builtin_amdgcn_exp2f(a * a * (-0.5f * kLog2e));
  return q * t;
}

// (1 + tanh u) / 2 = logistic(2u), 2u = x (A + B x^2)
constexpr float kTanhA = 1.5957691216057308f;  // 2 sqrt(2 / pi)
constexpr float kTanhB = 1.5957691216057308f * 0.044715f;

template <int ACT> __device__ __forceinline__ float act_value(float x) {
  if constexpr (ACT == ACT_RELU) return x < 0.0f ? 0.0f : x;  // NaN stays NaN
  if constexpr (ACT == ACT_GELU) {
    float bell;
    const float q = mills(__builtin_fabsf(x), bell) * bell;
    return x * (x < 0.0f ? q : 1.0f - q);
  }
  if constexpr (ACT == ACT_GELU_TANH) return x * logistic2(x * __builtin_fmaf(-kLog2e * kTanhB, x * x, -kLog2e * kTanhA));
  if constexpr (ACT == ACT_SILU) return x * logistic2(-kLog2e * x);
  return x;
}

// f'(x).  At and beyond +-128 every slope is 0 or 1 in fp32 (silu's is x exp(x) far below 0, which
// leaves fp32 at -104; the logistic function's exponential passes its range at -89); the saved
// value may be infinite where it passed its type's range, and inf * 0 must not enter (NaN does).
template <int ACT> __device__ __forceinline__ float act_slope(float x) {
  if constexpr (ACT == ACT_RELU) return x <= 0.0f ? 0.0f : 1.0f;
  if constexpr (ACT == ACT_GELU) {
    // Phi(x) + x phi(x) is w = phi's factor exp(-a^2 / 2) times (Q(a) - a / sqrt(2 pi))
    // for x < 0, a = |x|, and 1 - w above
    float a = __builtin_fabsf(x);
    a = a > 128.0f ? 128.0f : a;
    float bell;
    const float q = mills(a, bell);
    const float w = bell * __builtin_fmaf(a, -0.3989422804014327f, q);
    return x < 0.0f ? w : 1.0f - w;
  }
  x = x > 128.0f ? 128.0f : x < -128.0f ? -128.0f : x;
  if constexpr (ACT == ACT_GELU_TANH) {
    const float x2 = x * x, p = logistic2(x * __builtin_fmaf(-kLog2e * kTanhB, x2, -kLog2e * kTanhA));
    return __builtin_fmaf(x * p * (1.0f - p), __builtin_fmaf(3.0f * kTanhB, x2, kTanhA), p);
  }
  if constexpr (ACT == ACT_SILU) {
    const float p = logistic2(-kLog2e * x);
    return __builtin_fmaf(x * p, 1.0f - p, p);
  }
  return 1.0f;
}

// Eight values by the activation that the call names: one branch for all of them
// (one for each cost more than the arithmetic: a 256 x 256 tile's bias alone 10 us).
template <class F> __device__ __forceinline__ void by_act(int act, F f) {
  switch (act) {
    case ACT_RELU: f(std::integral_constant<int, ACT_RELU>()); break;
    case ACT_GELU: f(std::integral_constant<int, ACT_GELU>()); break;
    case ACT_GELU_TANH: f(std::integral_constant<int, ACT_GELU_TANH>()); break;
    case ACT_SILU: f(std::integral_constant<int, ACT_SILU>()); break;
  }
}
// x = f(x)
__device__ __forceinline__ void apply_values(float (&x)[8], int act) {
  by_act(act, [&](auto a) {
#pragma unroll
    for (int q = 0; q < 8; ++q) x[q] = act_value<decltype(a)::value>(x[q]);
  });
}
// x *= f'(z)
__device__ __forceinline__ void apply_slopes(float (&x)[8], const float (&z)[8], int act) {
  by_act(act, [&](auto a) {
#pragma unroll
    for (int q = 0; q < 8; ++q) x[q] *= act_slope<decltype(a)::value>(z[q]);
  });
}

// ---- eight consecutive columns of a row of C's type -----------------------------
template <int DT> struct Row8 {
  static constexpr int OS = OutSize<DT>::v, W = OS / 2;
  static constexpr int OT = DT == DT_FP8 ? DT_BF16 : DT;  // type of C
  u32x4 w[W];
  // byte offset `off`; the first `left` columns lie inside the matrix (vec: all eight, or
  // `off` is out of range)
  __device__ __forceinline__ void load(Rsrc r, int off, bool vec, int left) {
    if (vec) {
#pragma unroll
      for (int q = 0; q < W; ++q) w[q] = __builtin_amdgcn_raw_buffer_load_b128(r, off + 16 * q, 0, 0);
    } else {
#pragma unroll
      for (int q = 0; q < W; ++q) w[q] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < left) w[e * OS / 16][(e * OS / 4) & 3] |= load_elem<OS>(r, off + e * OS) << ((e * OS * 8) & 31);
    }
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = get(e);
  }
  __device__ __forceinline__ float get(int e) const {
    const unsigned x = w[e * OS / 16][(e * OS / 4) & 3];
    return ew_decode<OT>(OS == 4 ? x : (x >> ((e * 16) & 31)) & 0xffffu);
  }
  __device__ __forceinline__ void set(const float (&x)[8]) {
    if constexpr (OS == 4) {
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e / 4][e & 3] = __builtin_bit_cast(unsigned, x[e]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; e += 2) w[0][e / 2] = to_out2<OT>(x[e], x[e + 1]);
    }
  }
  __device__ __forceinline__ void store(Rsrc r, int off, bool vec, int left) const {
    if (vec) {
#pragma unroll
      for (int q = 0; q < W; ++q) __builtin_amdgcn_raw_buffer_store_b128(w[q], r, off + 16 * q, 0, 0);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < left) {
          const unsigned x = w[e * OS / 16][(e * OS / 4) & 3];
          if constexpr (OS == 4) __builtin_amdgcn_raw_buffer_store_b32(x, r, off + e * OS, 0, 0);
          else __builtin_amdgcn_raw_buffer_store_b16((uint16_t)(x >> ((e * 16) & 31)), r, off + e * OS, 0, 0);
        }
    }
  }
};

// The bias of columns j .. j + 7 (reads past N return 0).
template <int DT>
__device__ __forceinline__ void load_bias(const EpiOut& o, int j, float (&b)[8]) {
#pragma unroll
  for (int q = 0; q < 8; ++q) b[q] = 0.0f;
  if (!o.bias) return;
  if (o.bias_f32) {
    Row8<DT_F32> w;
    w.load(make_rsrc(o.bias, o.n * 4), j * 4, true, 8);
#pragma unroll
    for (int q = 0; q < 8; ++q) b[q] = w.get(q);
  } else {
    constexpr int OS = OutSize<DT>::v;
    Row8<DT> w;
    // whole dwords: the last element may share one with bytes past the bias
    const bool dwords = ((uintptr_t)o.bias & 3) == 0;
    w.load(make_rsrc(o.bias, dwords ? (o.n * OS + 3) & ~3 : o.n * OS), j * OS, dwords, 8);
#pragma unroll
    for (int q = 0; q < 8; ++q) b[q] = w.get(q);
  }
}

// The bias of columns j .. j + 3, and four of a linear epilogue's sums, rounded (two bytes
// an element).
template <int DT> __device__ __forceinline__ f32x4 load_bias4(const EpiOut& o, int j) {
  constexpr int OS = OutSize<DT>::v;
  f32x4 b = {0.0f, 0.0f, 0.0f, 0.0f};
  if (!o.bias) return b;
  if (o.bias_f32) {
    return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(make_rsrc(o.bias, o.n * 4), j * 4, 0, 0));
  } else {
    const Rsrc r = make_rsrc(o.bias, o.n * OS);
#pragma unroll
    for (int q = 0; q < 4; ++q) b[q] = ew_decode<Row8<DT>::OT>(load_elem<OS>(r, (j + q) * OS));
    return b;
  }
}
template <int DT> __device__ __forceinline__ f32x4 linear_sums(f32x4 x, float scale, f32x4 b) {
#pragma unroll
  for (int q = 0; q < 4; ++q) x[q] = DT == DT_FP8 ? __builtin_fmaf(x[q], scale, b[q]) : x[q] + b[q];
  return x;
}
template <int DT> __device__ __forceinline__ u32x2 linear4(f32x4 x, float scale, f32x4 b) {
  x = linear_sums<DT>(x, scale, b);
  return u32x2{to_out2<Row8<DT>::OT>(x[0], x[1]), to_out2<Row8<DT>::OT>(x[2], x[3])};
}

// What a wave does with blocks of R rows x WC columns of a tile's sums, one after
// another: the caller lays a block's sums into the wave's LDS, PITCH bytes a row, and
// calls rows().  Lane l owns the columns 8 * (l % LPR) .. + 7.
template <int DT, int R, int WC, int ROWS_AHEAD> struct EpiWave {
  static constexpr int OS = OutSize<DT>::v;
  static constexpr int LPR = WC / 8;             // lanes per row
  static constexpr int RP = 64 / LPR;            // rows per pass
  static constexpr int PASSES = (R + RP - 1) / RP;
  static constexpr int AHEAD = PASSES < ROWS_AHEAD ? PASSES : ROWS_AHEAD;
  static_assert(PASSES % AHEAD == 0, "whole steps");
  static constexpr int PITCH = WC * 4 + 16;      // writes of 16 rows of 16 bytes hit distinct banks
  static constexpr int BYTES = R * PITCH;        // LDS of a wave
  const EpiOut o;
  Rsrc rc, rr, ra;
  int lane;
  int col, left;  // this lane's first column, and how many of its eight lie inside C
  bool grad;
  bool whole;     // every lane of the wave has all its columns inside C, or none
  float b[8], sum[8];

  __device__ __forceinline__ EpiWave(const EpiOut& out, int lane_) : o(out), lane(lane_) {
    rc = make_rsrc(o.c, o.c_bytes);
    rr = make_rsrc(o.res, o.res ? ((o.m - 1) * o.ldr + o.n) * OS : 0);
    ra = make_rsrc(o.aux, o.aux ? ((o.m - 1) * o.ldaux + o.n) * OS : 0);
    grad = o.grad && o.act != ACT_NONE;
  }
  // the blocks from here on start at column `first` of C
  __device__ __forceinline__ void columns(int first) {
    col = first + (lane % LPR) * 8;
    left = o.n - col;
    whole = __ballot(left > 0 && left < 8) == 0;
    load_bias<DT>(o, col, b);
#pragma unroll
    for (int q = 0; q < 8; ++q) sum[q] = 0.0f;
  }

  // Byte offset of this lane's columns in a row; out of every range where `in` is false.
  __device__ __forceinline__ int at(bool in, int row, int ld) const { return in ? (row * ld + col) * OS : kOutOfRange; }

  __device__ __forceinline__ void load_inputs(bool in, int row, Row8<DT>& res, Row8<DT>& aux) {
    if (o.res) res.load(rr, at(in, row, o.ldr), whole && (OS == 4 || o.res_vec), left);
    if (grad) aux.load(ra, at(in, row, o.ldaux), whole && (OS == 4 || o.aux_vec), left);
  }

  // Eight sums of a row to C.
  __device__ __forceinline__ void finish(bool in, int row, float (&x)[8], const Row8<DT>& res, const Row8<DT>& aux) {
    Row8<DT> w;
#pragma unroll
    for (int q = 0; q < 8; ++q) x[q] = DT == DT_FP8 ? __builtin_fmaf(x[q], o.scale, b[q]) : x[q] + b[q];
    if (grad) {
      float z[8];
      aux.get(z);
      apply_slopes(x, z, o.act);
    } else if (!o.grad) {
      if (o.aux) {
        w.set(x);
        w.store(ra, at(in, row, o.ldaux), whole && (OS == 4 || o.aux_vec), left);
      }
      apply_values(x, o.act);
    }
    if (o.res) {
#pragma unroll
      for (int q = 0; q < 8; ++q) x[q] += res.get(q);
    }
    if (o.part) {
#pragma unroll
      for (int q = 0; q < 8; ++q) sum[q] += in ? x[q] : 0.0f;
    }
    w.set(x);
    w.store(rc, at(in, row, o.ldc), whole && (OS == 4 || o.c_vec), left);
  }

  // The block at `block`: rows m0, m0 + 1, ... of C, which has `inside` from m0 on.  No
  // branch depends on a lane: rows and columns outside C go out of range.
  __device__ __forceinline__ void rows(const lds_u8* block, int m0, int inside) {
    const int count = min(R, inside);  // a pass may reach past a block of 16 rows
    if (count <= 0) return;
    // the wave's own sums, in LDS in the order of its instructions
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll 1
    for (int u0 = 0; u0 < PASSES; u0 += AHEAD) {
      Row8<DT> res[AHEAD], aux[AHEAD];
      const int r0 = lane / LPR + u0 * RP;
#pragma unroll
      for (int u = 0; u < AHEAD; ++u)
        load_inputs(r0 + u * RP < count && left > 0, m0 + r0 + u * RP, res[u], aux[u]);
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int r = r0 + u * RP;
        const lds_u8* p = block + (PASSES * RP > R ? min(r, R - 1) : r) * PITCH + (lane % LPR) * 32;
        const f32x4 lo = *(const __attribute__((address_space(3))) f32x4*)p;
        const f32x4 hi = *(const __attribute__((address_space(3))) f32x4*)(p + 16);
        float x[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        finish(r < count && left > 0, m0 + r, x, res[u], aux[u]);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // before the next block's sums
    __builtin_amdgcn_wave_barrier();
  }

  // This lane's sums of its eight columns to LDS: row `r0` (of its RP) of a table of
  // `width` columns, the lane's at `c`.
  __device__ __forceinline__ void put_sums(lds_u8* table, int row, int width, int c) const {
    typedef __attribute__((address_space(3))) f32x4 lds_f32x4;
    lds_u8* at = table + (row * width + c) * 4;
    *(lds_f32x4*)at = f32x4{sum[0], sum[1], sum[2], sum[3]};
    *(lds_f32x4*)(at + 16) = f32x4{sum[4], sum[5], sum[6], sum[7]};
  }
};

// The table of column sums that the waves have laid down (`rows` rows of `width`) to
// part: lanes added their rows in ascending order, the table's rows are added in
// order, so the result does not depend on the run.
template <int ROWS>
__device__ __forceinline__ void add_sums(const lds_u8* table, int width, float* part, int cols, int tid) {
  if (tid < cols) {
    float x = 0.0f;
#pragma unroll 8
    for (int r = 0; r < ROWS; ++r)
      x += *(const __attribute__((address_space(3))) float*)(table + (r * width + tid) * 4);
    part[tid] = x;
  }
}

// ---- split-K reduction with an epilogue -------------------------------------------
// As split_reduce, kEpiReduceRows rows x 128 columns a tile: 256 threads of eight
// columns, a wave four rows.
template <int DT>
__global__ void __launch_bounds__(256) split_reduce_ep(KLaunch L, KEpis E) {
  (void)E;  // read by MemberEpi
  constexpr int BN = 128;
  __shared__ __attribute__((aligned(16))) uint8_t smem[256 * 8 * 4];
  const int gi = owner_of(L);
  const KArgs& p = L.g[gi];
  const int wg0 = L.first[gi];
  const int nwg = L.first[gi + 1] - wg0;
  typedef EpiWave<DT, 4, BN, 1> Wave;
  const int tid = threadIdx.x;
  const int M = (int)p.m, N = (int)p.n, S = p.split;
  const int tn = (N + BN - 1) / BN, tm = (M + kEpiReduceRows - 1) / kEpiReduceRows;
  const int ntiles = tm * tn, total = ntiles * p.batch;
  const size_t plane = (size_t)M * (size_t)N;
  for (int tb = (int)blockIdx.x - wg0; tb < total; tb += nwg) {
    const int item = tb / ntiles, t = tb - item * ntiles;
    const int row = (t / tn) * kEpiReduceRows + tid / Wave::LPR, n0 = (t % tn) * BN;
    Wave x(MemberEpi<1>{gi}(item, t / tn), tid & 63);
    x.columns(n0);
    if (row < M && x.left > 0) {
      Row8<DT> res, aux;
      x.load_inputs(true, row, res, aux);
      const float* P = p.ws + (size_t)item * S * plane + (size_t)row * N + x.col;
      float v[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
      if ((N & 3) == 0 && x.left >= 8) {  // 16-byte aligned rows of the planes
        for (int s = 0; s < S; ++s) {
          const float4 lo = *reinterpret_cast<const float4*>(P + s * plane);
          const float4 hi = *reinterpret_cast<const float4*>(P + s * plane + 4);
          v[0] += lo.x, v[1] += lo.y, v[2] += lo.z, v[3] += lo.w;
          v[4] += hi.x, v[5] += hi.y, v[6] += hi.z, v[7] += hi.w;
        }
      } else {
#pragma unroll
        for (int q = 0; q < 8; ++q)
          if (q < x.left)
            for (int s = 0; s < S; ++s) v[q] += P[s * plane + q];
      }
      x.finish(true, row, v, res, aux);
    }
    if (x.o.part) {
      x.put_sums((lds_u8*)smem, tid / Wave::LPR, BN, (tid % Wave::LPR) * 8);
      __syncthreads();
      add_sums<kEpiReduceRows>((lds_u8*)smem, BN, x.o.part + n0, min(BN, N - n0), tid);
      __syncthreads();  // the next tile's sums overwrite these
    }
  }
}

}  // namespace gdy
