// epilogue.h -- what a GEMM does with its fp32 sums before the one rounding:
//   z = scale * sum + bias(j);   aux(i,j) = round(z);   C = round(f(z) + R(i,j))
// or, backward (grad), with the saved pre-activation aux read:
//   g = (scale * sum + bias(j)) * f'(aux(i,j));   C = round(g + R(i,j))
// and the column sums of the unrounded C, from which bias gradients are made.
//
// The accumulators of a tile go through LDS as fp32 rows (64 or 128 at a time,
// which the operand stages they replace have room for), so that a lane owns
// eight consecutive columns of whole rows: the residual and the saved
// pre-activation are read, and C written, with 16 consecutive bytes a lane, the
// bias stays in registers, and one rolled loop holds the activations, where the
// accumulators' order would need them unrolled over every block.  Nothing is
// rounded between the sum and C.
#pragma once
#include <stddef.h>

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
};

// Kernels without epilogues.
struct NoEpi {
  static constexpr bool on = false;
};

// The member gi of a kernel whose arguments are (KLaunch, KEpis).  Read when a
// tile's sums are done: the empty asm hides the pointer's origin from the compiler
// there, which would otherwise load the fields before the tile loop and keep them
// in registers through it (scalars then spill to scratch memory).
struct MemberEpi {
  static constexpr bool on = true;
  typedef const __attribute__((address_space(4))) uint8_t* Ptr;
  int gi;
  __device__ __forceinline__ EpiOut operator()(int item, int tile_row) const {
    constexpr int at = (sizeof(KLaunch) + alignof(KEpis) - 1) / alignof(KEpis) * alignof(KEpis);
    Ptr args = (Ptr)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(args));
    const auto* a = (const __attribute__((address_space(4))) KArgs*)(args + offsetof(KLaunch, g)) + gi;
    const auto* e = (const __attribute__((address_space(4))) KEpi*)(args + at) + gi;
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

__device__ __forceinline__ float logistic(float x) {  // 1 / (1 + e^-x); 0 where e^-x overflows
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * x));
}

// exp(-x^2 / 2) and Phi(x), the normal distribution function.  With a = |x|,
// Phi(-a) = exp(-a^2 / 2) Q(a), Q(a) = erfcx(a / sqrt 2) / 2, and Q as a polynomial
// in t = 1 / (1 + 0.3 a), fitted to the least largest relative error on [0, 14]
// (4.6e-7 evaluated in fp32): small Phi keep their relative precision, which 1 +
// erf loses.
__device__ __forceinline__ float normal_cdf(float x, float& bell) {
  const float a = __builtin_fabsf(x);
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
  q = q * t * bell;
  return x < 0.0f ? q : 1.0f - q;
}

constexpr float kTanhA = 1.5957691216057308f;              // 2 sqrt(2 / pi)
constexpr float kTanhB = 1.5957691216057308f * 0.044715f;  // (1 + tanh u) / 2 = logistic(2u)

__device__ __forceinline__ float act_value(float x, int act) {
  switch (act) {
    case ACT_RELU: return x < 0.0f ? 0.0f : x;  // NaN stays NaN
    case ACT_GELU: {
      float bell;
      return x * normal_cdf(x, bell);
    }
    case ACT_GELU_TANH: return x * logistic(x * __builtin_fmaf(kTanhB, x * x, kTanhA));
    case ACT_SILU: return x * logistic(x);
    default: return x;
  }
}

// f'(x).  Beyond +-64 every slope is 0 or 1 in fp32; the saved value may be
// infinite where it passed its type's range, and inf * 0 must not enter.
__device__ __forceinline__ float act_slope(float x, int act) {
  x = x > 64.0f ? 64.0f : x < -64.0f ? -64.0f : x;
  switch (act) {
    case ACT_RELU: return x <= 0.0f ? 0.0f : 1.0f;
    case ACT_GELU: {
      float bell;
      const float cdf = normal_cdf(x, bell);
      return __builtin_fmaf(x * bell, 0.3989422804014327f, cdf);
    }
    case ACT_GELU_TANH: {
      const float x2 = x * x, p = logistic(x * __builtin_fmaf(kTanhB, x2, kTanhA));
      return __builtin_fmaf(x * p * (1.0f - p), __builtin_fmaf(3.0f * kTanhB, x2, kTanhA), p);
    }
    case ACT_SILU: {
      const float p = logistic(x);
      return __builtin_fmaf(x * p, 1.0f - p, p);
    }
    default: return 1.0f;
  }
}

// ---- eight consecutive columns of a row of C's type -----------------------------
template <int DT> struct Row8 {
  static constexpr int OS = OutSize<DT>::v, W = OS / 2;
  static constexpr int OT = DT == DT_FP8 ? DT_BF16 : DT;  // type of C
  u32x4 w[W];
  // byte offset `off`; the first `left` columns lie inside the matrix
  __device__ __forceinline__ void load(Rsrc r, int off, bool vec, int left) {
    if (vec && left >= 8) {
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
    if (vec && left >= 8) {
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
    const Rsrc r = make_rsrc(o.bias, o.n * 4);
#pragma unroll
    for (int q = 0; q < 8; ++q) b[q] = ew_decode<DT_F32>(load_elem<4>(r, (j + q) * 4));
  } else {
    constexpr int OS = OutSize<DT>::v;
    const Rsrc r = make_rsrc(o.bias, o.n * OS);
#pragma unroll
    for (int q = 0; q < 8; ++q) b[q] = ew_decode<Row8<DT>::OT>(load_elem<OS>(r, (j + q) * OS));
  }
}

// One tile's epilogue, by the NT threads of a workgroup: the caller lays some of its
// rows into LDS, PITCH bytes apart, and calls rows() between two barriers, until
// all rows are done, then sums().
template <int DT, int BN, int NT> struct EpiTile {
  static constexpr int OS = OutSize<DT>::v;
  static constexpr int LPR = BN / 8;       // lanes per row
  static constexpr int RP = NT / LPR;      // rows per pass
  static constexpr int PITCH = BN * 4 + 16;  // a half wave's 16 rows of 16 bytes on distinct banks
  static constexpr int AHEAD = NT == 512 ? 2 : 4;  // rows whose residual and aux are loaded together
  const EpiOut o;
  Rsrc rc, rr, ra;
  int c8, left;  // first column of this lane within the tile, and how many of its eight lie inside C
  int n0, cols;  // the tile's first column, and how many of its columns lie inside C
  int tid;
  bool grad;
  float b[8], sum[8];

  __device__ __forceinline__ EpiTile(const EpiOut& out, int n0_, int tid_) : o(out), n0(n0_), tid(tid_) {
    cols = min(BN, o.n - n0);
    rc = make_rsrc(o.c, o.c_bytes);
    rr = make_rsrc(o.res, o.res ? ((o.m - 1) * o.ldr + o.n) * OS : 0);
    ra = make_rsrc(o.aux, o.aux ? ((o.m - 1) * o.ldaux + o.n) * OS : 0);
    c8 = (tid % LPR) * 8;
    left = cols - c8;
    grad = o.grad && o.act != ACT_NONE;
    load_bias<DT>(o, n0 + c8, b);
#pragma unroll
    for (int q = 0; q < 8; ++q) sum[q] = 0.0f;
  }

  __device__ __forceinline__ void load_inputs(int row, Row8<DT>& res, Row8<DT>& aux) {
    const int col = (n0 + c8) * OS;
    if (o.res) res.load(rr, row * o.ldr * OS + col, OS == 4 || o.res_vec, left);
    if (grad) aux.load(ra, row * o.ldaux * OS + col, OS == 4 || o.aux_vec, left);
  }

  // Eight sums of a row to C.
  __device__ __forceinline__ void finish(int row, float (&x)[8], const Row8<DT>& res, const Row8<DT>& aux) {
    const int col = (n0 + c8) * OS;
    Row8<DT> w;
#pragma unroll
    for (int q = 0; q < 8; ++q) x[q] = x[q] * o.scale + b[q];
    if (grad) {
#pragma unroll
      for (int q = 0; q < 8; ++q) x[q] *= act_slope(aux.get(q), o.act);
    } else if (!o.grad) {
      if (o.aux) {
        w.set(x);
        w.store(ra, row * o.ldaux * OS + col, OS == 4 || o.aux_vec, left);
      }
#pragma unroll
      for (int q = 0; q < 8; ++q) x[q] = act_value(x[q], o.act);
    }
    if (o.res) {
#pragma unroll
      for (int q = 0; q < 8; ++q) x[q] += res.get(q);
    }
#pragma unroll
    for (int q = 0; q < 8; ++q) sum[q] += x[q];
    w.set(x);
    w.store(rc, row * o.ldc * OS + col, OS == 4 || o.c_vec, left);
  }

  // The rows 0 .. count - 1 at `rows_lds`: rows m0, m0 + 1, ... of C.
  __device__ __forceinline__ void rows(const lds_u8* rows_lds, int m0, int count) {
    if (left <= 0) return;
    for (int r0 = tid / LPR; r0 < count; r0 += RP * AHEAD) {
      Row8<DT> res[AHEAD], aux[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u)
        if (r0 + u * RP < count) load_inputs(m0 + r0 + u * RP, res[u], aux[u]);
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int r = r0 + u * RP;
        if (r >= count) break;
        const lds_u8* at = rows_lds + r * PITCH + c8 * 4;
        const f32x4 lo = *(const __attribute__((address_space(3))) f32x4*)at;
        const f32x4 hi = *(const __attribute__((address_space(3))) f32x4*)(at + 16);
        float x[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        finish(m0 + r, x, res[u], aux[u]);
      }
    }
  }

  // The tile's column sums to its row of part.  Lanes add their rows in ascending
  // order, then the row groups are added in order: the result does not depend on
  // the run.  `lds` holds NT * 8 floats and no rows that are still read.
  __device__ __forceinline__ void sums(lds_u8* lds) {
    typedef __attribute__((address_space(3))) f32x4 lds_f32x4;
    lds_u8* at = lds + (tid / LPR) * (BN * 4) + c8 * 4;
    *(lds_f32x4*)at = f32x4{sum[0], sum[1], sum[2], sum[3]};
    *(lds_f32x4*)(at + 16) = f32x4{sum[4], sum[5], sum[6], sum[7]};
    __syncthreads();
    if (tid < cols) {
      float x = 0.0f;
#pragma unroll 4
      for (int r = 0; r < RP; ++r) x += *(const __attribute__((address_space(3))) float*)(lds + r * (BN * 4) + tid * 4);
      o.part[n0 + tid] = x;
    }
  }
};

// ---- split-K reduction with an epilogue -------------------------------------------
// As split_reduce, kEpiReduceRows rows x 128 columns a tile: 256 threads of eight columns.
template <int DT>
__global__ void __launch_bounds__(256) split_reduce_ep(KLaunch L, KEpis E) {
  (void)E;  // read by MemberEpi
  constexpr int BN = 128;
  __shared__ __attribute__((aligned(16))) uint8_t smem[256 * 8 * 4];
  const int gi = owner_of(L);
  const KArgs& p = L.g[gi];
  const int wg0 = L.first[gi];
  const int nwg = L.first[gi + 1] - wg0;
  typedef EpiTile<DT, BN, 256> Tile;
  const int tid = threadIdx.x;
  const int M = (int)p.m, N = (int)p.n, S = p.split;
  const int tn = (N + BN - 1) / BN, tm = (M + kEpiReduceRows - 1) / kEpiReduceRows;
  const int ntiles = tm * tn, total = ntiles * p.batch;
  const size_t plane = (size_t)M * (size_t)N;
  for (int tb = (int)blockIdx.x - wg0; tb < total; tb += nwg) {
    const int item = tb / ntiles, t = tb - item * ntiles;
    const int row = (t / tn) * kEpiReduceRows + tid / Tile::LPR;
    Tile x(MemberEpi{gi}(item, t / tn), (t % tn) * BN, tid);
    if (row < M && x.left > 0) {
      Row8<DT> res, aux;
      x.load_inputs(row, res, aux);
      const float* P = p.ws + (size_t)item * S * plane + (size_t)row * N + x.n0 + x.c8;
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
      x.finish(row, v, res, aux);
    }
    if (x.o.part) {
      x.sums((lds_u8*)smem);
      __syncthreads();  // the next tile's sums overwrite these
    }
  }
}

}  // namespace gdy
