// gdy_internal.h -- structures shared by the GO-Kernel instantiation units
// and the host runtime of libgdy (not part of the public C-ABI).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace gdy {

// Element types, numerically equal to the public gdy_dtype values.
enum : int { DT_F16 = 1, DT_BF16 = 2, DT_FP8 = 3, DT_F32 = 4 };
// Products of 8-bit integers (integer.h), by the type of C; inside the library only.
enum : int { DT_I8_F16 = 5, DT_I8_BF16 = 6, DT_I8_F32 = 7 };

// Kernel arguments, passed by value.  Sizes and leading dimensions are in
// elements; the storage reading is row-major with op(A)(i,k) = A[i*lda+k]
// (or A[k*lda+i] when A is used transposed) and op(B)(k,j) = B[k*ldb+j]
// (or B[j*ldb+k] when transposed).
struct KArgs {
  const uint8_t* a;
  const uint8_t* b;
  uint8_t* c;
  int64_t m, n, k;
  int64_t lda, ldb, ldc;
  float scale;        // sa*sb rounded once in fp32 (1 for 16-bit inputs)
  int32_t a_bytes;    // extent of each operand in bytes (< 2^31): reads and
  int32_t b_bytes;    // writes outside it are dropped by the buffer unit
  int32_t c_bytes;
  int32_t tiles_m;    // ceil(m / BM)
  int32_t tiles_n;    // ceil(n / BN)
  int32_t a_vec;      // adds, 1: A base and rows are aligned for vector loads
  int32_t b_vec;      // 1: same for B
  int32_t c_vec;      // 1: C base and rows allow 8-byte stores
  int32_t a_dma;      // 1: A takes direct 16-byte copies to LDS (base, pitch and item stride
  int32_t b_dma;      //    aligned; K-contiguous: K whole chunks); b_dma: same for B
  int32_t group_m;    // tile-order swizzle: tile rows per group
  int32_t xcd_remap;  // 1: keep consecutive tiles on one XCD
  int32_t batch;      // items of a strided batch (>= 1); the extents above are per item
  int32_t code;       // joint launches: the member's tile and layout
  int32_t rows128;    // 256 x 256 kernels: 1: tiles of 128 rows (tiles_m counts them)
  int32_t ew;         // 0: a GEMM; else the DT_* of an element-wise add (C = A + B)
  int32_t split;      // split-K: K tiles are cut into `split` runs of `split_kt` tiles;
  int32_t split_kt;   //   each run writes an fp32 M x N plane, a reduction kernel sums them
  float* ws;          // split > 1: the planes, batch x split of them, leading dimension N
  int64_t stride_a;   // bytes between consecutive items of A, B and C
  int64_t stride_b;
  int64_t stride_c;
};

// One kernel dispatch: up to kMaxFused GEMMs that use the same kernel share
// one grid.  GEMM i owns workgroups [first[i], first[i+1]) and walks its own
// tiles with that range's length as the stride, so a tile is computed by
// exactly the same code (and gives the same bits) whether the GEMM runs
// alone or fused with others.  first[i] is a multiple of 8 for i > 0 so a
// GEMM's local workgroup index keeps the hardware's XCD round-robin phase.
//
// XCD placement (placed != 0; GEMM members that neither split nor cap their
// grid): the hardware deals workgroup b to XCD b % 8, so b runs as slot
// b / 8 of XCD x = b % 8.  The slots of XCD x walk its pieces
// [xcd_first[x], xcd_first[x+1]): piece q covers that XCD's slots up to
// piece_end[q] (exclusive, counted from the XCD's first slot) with the
// consecutive work items piece_tile[q], piece_tile[q] + 1, ... of member
// piece_gemm[q].  Slots past the XCD's last piece are idle.  The host gives
// each XCD an even share of the dispatch's work built from few members, so
// each member's A is fetched by few XCDs' L2s.  A work item is computed by
// the same code wherever it runs: the bits do not change.
constexpr int kMaxFused = 16;
constexpr int kXcds = 8;
constexpr int kMaxPieces = 48;
struct KLaunch {
  int32_t count;                  // GEMMs in this dispatch, 1..kMaxFused
  int32_t first[kMaxFused + 1];   // workgroup ranges; first[count] = grid size
  KArgs g[kMaxFused];
  int32_t placed;                 // 1: the piece table below maps workgroups to work
  int32_t xcd_first[kXcds + 1];
  int32_t piece_end[kMaxPieces];
  int32_t piece_tile[kMaxPieces];
  int8_t piece_gemm[kMaxPieces];
};

// The member of a range dispatch that owns workgroup b (uniform per
// workgroup: a short scalar scan of the workgroup ranges).
__host__ __device__ inline int owner_of(const KLaunch& L, int b) {
  int i = 0;
  while (i + 1 < L.count && b >= L.first[i + 1]) ++i;
  return i;
}

// Workgroup b's member gi, its first work item lwg and its stride nwg (work
// items lwg, lwg + nwg, ... of that member).  Range dispatches: the member's
// workgroup range.  Placed dispatches: one work item from the XCD's piece
// table (nwg past any item count), or gi = -1 for an idle slot.  The kernels
// and the host's dispatch map (gdy_dispatch_map) run this same code.
__host__ __device__ inline void locate(const KLaunch& L, int b, int& gi, int& lwg, int& nwg) {
  if (L.placed) {
    const int x = b & (kXcds - 1), j = b / kXcds;
    const int q0 = L.xcd_first[x], q1 = L.xcd_first[x + 1];
    int q = q0;
    while (q < q1 && j >= L.piece_end[q]) ++q;
    if (q == q1) {
      gi = -1;
      return;
    }
    gi = L.piece_gemm[q];
    lwg = L.piece_tile[q] + j - (q == q0 ? 0 : L.piece_end[q - 1]);
    nwg = 1 << 30;
    return;
  }
  gi = owner_of(L, b);
  lwg = b - L.first[gi];
  nwg = L.first[gi + 1] - L.first[gi];
}

// Activations, numerically equal to the public gdy_act values.
enum : int { ACT_NONE = 0, ACT_RELU = 1, ACT_GELU = 2, ACT_GELU_TANH = 3, ACT_SILU = 4 };

// The epilogue of one member.  Strides are bytes between items of a batch.
struct KEpi {
  const uint8_t* bias;   // N values (null: none)
  const uint8_t* res;    // M x N of C's type (null: none); may be C itself
  uint8_t* aux;          // M x N of C's type: written (grad: read)
  float* part;           // column sums of C by tile row: part_rows rows of N per item (null: none)
  int64_t stride_bias, stride_res, stride_aux;
  int32_t ldr, ldaux;    // elements
  int32_t part_rows;
  int32_t bias_f32;      // 1: bias is fp32, else of C's type
  int32_t act, grad;
  int32_t res_vec, aux_vec;  // 1: rows allow 16-byte accesses (KArgs::c_vec's rule)
};
struct KEpis {
  KEpi e[kMaxFused];
};

// The split reduction with epilogues takes this many rows a tile.
constexpr int kEpiReduceRows = 16;

// A product grouped by expert (grouped.h).
struct KGroup {
  const uint8_t* a;
  const uint8_t* b;
  uint8_t* c;
  const int32_t* offsets;  // groups + 1
  const float* scales;     // one per group (null: 1)
  int64_t stride_b;        // bytes between groups of B
  int64_t stride_c;        // over K: bytes between groups of C
  int32_t rows, groups;
  int32_t m, n, k;         // over rows: C is rows x n, K = k; over K: C_e is m x n
  int32_t lda, ldb, ldc;   // elements
  float scale;
  int32_t a_dma, b_dma, c_vec;
  int32_t bm;              // over rows: rows of a tile
  int32_t max_slots;       // over rows: the most row tiles
  int32_t xcd_cus;         // CUs of an XCD
  KEpi epi;                // over K: the residual only; strides between groups
};

// A kernel of grouped products: its tile and threads.  Tiles by index: 256 x 256,
// 128 x 128, 64 x 128 (over K 64 x 64), and over rows 32 x 128 and 32 x 64.
struct GroupKernel {
  const void* func;
  int bm, bn, threads;
};

// The kernels that finish bias gradients: a workgroup's columns and threads, for sums of
// many rows and of fewer than kSumManyRows.
constexpr int kSumManyRows = 64;
constexpr int sum_cols(bool many) { return many ? 16 : 64; }
constexpr int sum_threads(bool many) { return many ? 1024 : 256; }

// Partial sums to a bias gradient: out[item][j] = sum over `rows` rows of part.
struct BiasSums {
  int32_t count;
  int32_t many;                  // 1: some member has many rows
  int32_t first[kMaxFused + 1];  // workgroup ranges: sum_cols() columns of an item each
  const float* part[kMaxFused];
  float* out[kMaxFused];
  int64_t stride[kMaxFused];     // between items of out
  int32_t n[kMaxFused], rows[kMaxFused];
};

// The partial sums of grouped rows: those of group e's row tiles of bm rows, `per` rows of
// sums a tile, to out[e]; shared: of all groups, to out[0].
struct GroupSums {
  const float* part;
  float* out;
  const int32_t* offsets;
  int64_t stride;
  int32_t n, rows, groups, bm, max_slots, shared, per;
};
// dz = dy * f'(z), and partial column sums by row tile.
struct KActGrad {
  const uint8_t* dy;
  const uint8_t* z;        // null where f is the identity
  uint8_t* dz;             // null: not written
  const int32_t* offsets;  // null: one group of all rows
  float* part;             // row tiles x n (null: no sums)
  int32_t rows, groups, n, bm, max_slots;
  int32_t lddy, ldz, lddz, act;
  int32_t dy_vec, z_vec, dz_vec;
};

constexpr int kActCols = 512, kActRows = 32, kActThreads = 512;  // of a workgroup

// Rows to the experts and back (experts.h).  Pitches are bytes.
constexpr int kRowThreads = 256;  // of a workgroup
struct KScatter {
  const uint8_t* x;
  uint8_t* out;
  const uint8_t* z;        // read for weight_grad
  const int32_t* slots;
  const void* weights;
  float* weight_grad;
  int64_t tokens, ldx, ldo, ldz;
  int32_t rows, n, top_k;
  int32_t weights_f32;     // 1: weights are fp32, else of the rows' type
  int32_t tpr_log;         // threads of a row: 1 << tpr_log
};
struct KCombine {
  const uint8_t* z;
  const uint8_t* res;      // null: none; may be y
  uint8_t* y;
  const int32_t* slots;
  const void* weights;     // null: 1
  int64_t tokens, ldz, ldr, ldy;
  int32_t rows, n, top_k, weights_f32, tpr_log;
};

// The rows of each expert: parts of kRoutePart * steps pairs, a workgroup of kRoutePart
// threads each.
constexpr int kRoutePart = 1024, kRouteFew = 256, kMaxExperts = 4096;
constexpr int kRouteMaxSteps = 63;  // parts of fewer than 2^16 pairs
constexpr int kRouteSmall = 4;      // waves of a workgroup that is enough for all pairs
struct KRoute {
  const void* ids;
  int32_t* slots;
  int32_t* offsets;
  int32_t* counts;         // parts x experts; with totals: of the parts before
  int32_t* totals;         // one an expert (null: the parts' counts are not summed yet)
  int64_t ld_ids;
  int32_t pairs, top_k, experts;
  int32_t bits;            // of the experts' numbers
  int32_t wide, dense;     // 64-bit ids; ld_ids == top_k
  int32_t steps, parts;
  int32_t expert_threads;  // a power of two >= experts, at least 64
};

// Rows to 8-bit integers (quantize.h).  Pitches are bytes.
struct KQuantize {
  const uint8_t* x;
  int8_t* q;
  float* scales;
  const int32_t* slots;    // null: row i to row i
  int64_t rows, ldx, ldq;
  int32_t n, top_k, out_rows, tpr_log;
};

// A product of 8-bit integers (integer.h): the grouped product (offsets null: one group of
// all rows) and its scales.
struct KInteger {
  KGroup g;
  const float* row_scales;    // null: 1
  const float* col_scales;    // null: 1
  int64_t stride_col_scales;  // elements between groups
};

// Compile-time description of one instantiated kernel.
struct KernelDesc {
  const char* name;   // e.g. "bf16_nn_256x256_w8_m32"
  int dtype;          // DT_*
  int ta, tb;         // transposed use of A / B
  int bm, bn, bk;     // macro tile (bk in elements)
  int waves;          // waves per workgroup
  int mfma;           // 32 -> 32x32 MFMA blocks, 16 -> 16x16 blocks
  int lds_bytes;      // static LDS per workgroup
  const void* func;   // __global__ entry, launched with hipExtLaunchKernel (null: another
                      // catalogue kernel runs its GEMMs, see exec_of)
  int direct;         // 1: global->LDS copies; needs K % bk == 0 and 16-byte alignment
  int ew;             // 1: the element-wise add (a non-GEMM op), not a GEMM kernel
  const void* func_split;  // GEMM kernels: the split-K twin (runs split = 1 GEMMs too)
  int joint;          // family whose joint kernel can run this kernel's GEMMs: 1 (256 threads),
                      // 2 (512 threads), 0 none
  int joint_code;     // KArgs::code there, and the tile it runs
  int joint_bm, joint_bn;
};

// Each instantiation unit exports its table.
int kernels_bf16(const KernelDesc** out);
int kernels_f16(const KernelDesc** out);
int kernels_fp8(const KernelDesc** out);
int kernels_f32(const KernelDesc** out);
int kernels_ew(const KernelDesc** out);
// Split-K reduction kernel for an output type (DT_BF16, DT_F16, DT_F32).
const void* split_reduce_kernel(int out_dt);
// Joint kernel of a family (1, 2) for an input type; null if it has none.
const void* joint_bf16(int family);
const void* joint_f16(int family);
const void* joint_fp8(int family);
const void* joint_f32(int family);
// Kernels of launches with epilogues: of a family (1, 2), or the split-K
// reduction (0); null if there is none.
const void* ep_bf16(int family);
const void* ep_f16(int family);
const void* ep_fp8(int family);
const void* ep_f32(int family);
// For launches whose members share a joint code; copies: all of them take copies.
const void* ep_lone_bf16(int family, int code, bool copies);
const void* ep_lone_f16(int family, int code, bool copies);
const void* ep_lone_fp8(int family, int code, bool copies);
const void* ep_lone_f32(int family, int code, bool copies);
// GEMMs of at most kSkinnyRows rows, by type and transposed B (null: none); the columns
// of a workgroup, the K bytes of a wave's step, and the steps of a round.
constexpr int kSkinnyRows = 16;
const void* skinny_ep(int dt, int tb);
constexpr int skinny_cols(int tb) { return tb ? 16 : 64; }
constexpr int skinny_kstep(int es) { return es == 1 ? 128 : 64; }
constexpr int skinny_ahead(int es, int tb) { return tb && es != 1 ? 8 : 4; }
// Grouped products over rows in tiles of kSkinnyRows rows (skinny.h).
GroupKernel group_few(int dt, int tb);
GroupKernel group_bf16(int over_k, int tb, int tile);
GroupKernel group_f16(int over_k, int tb, int tile);
GroupKernel group_fp8(int over_k, int tb, int tile);
GroupKernel group_f32(int over_k, int tb, int tile);
const void* act_grad_kernel(int dt);  // null: no such type
const void* scatter_kernel(int dt, int mode);  // mode 0: copies (dt names the size), 1: weighted, 2: with weight_grad
const void* combine_kernel(int dt);
const void* route_count_kernel(bool few);  // few: at most kRouteFew experts
const void* route_sums_kernel();
const void* route_slots_kernel(bool few, int waves);  // kRouteSmall waves (few alone) or those of kRoutePart
// held: steps that a thread keeps (1, 2, or kQuantMost and more); whole: rows of whole steps.
constexpr int kQuantMost = 4;
const void* quantize_kernel(int dt, int held, bool whole);
// Products of 8-bit integers by the type of C (null: no such tile).  For operands that both take copies: 256 x 256
// tiles, smaller ones, and kSkinnyRows rows with B stored N x K; for any operands INT_ANY_*.
enum : int {
  INT_256, INT_64x128, INT_64, INT_32x64, INT_FEW, INT_ANY_128, INT_ANY_64x128, INT_ANY_32x128, INT_ANY_32x64
};
GroupKernel integer_bf16(int tb, int tile);
GroupKernel integer_f16(int tb, int tile);
GroupKernel integer_f32(int tb, int tile);
const void* bias_sum_kernel(bool many);
const void* group_sum_kernel(bool many);
int kernels_d_bf16(const KernelDesc** out);
int kernels_d_f16(const KernelDesc** out);
int kernels_d_fp8(const KernelDesc** out);

}  // namespace gdy
