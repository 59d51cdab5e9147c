/*
 * gdy.h -- C-ABI of libgdy: many independent dense GEMMs on one MI355X,
 * run either one after another or concurrently under a dynamic selector.
 *
 * Method: GOLDYLOC (Pati, Aga, Jayasena, Sinclair), "Global Optimizations &
 * Lightweight Dynamic Logic for Concurrency", arXiv 2409.02227.
 *   - GEMM definition: Sec. 2.1.2 -- C (M x N) from A (M x K) and B, with
 *     2*M*N*K flops; T1/T2 say whether A and B are used transposed.
 *   - GO-Kernels: Sec. 4.2 -- per GEMM shape, one kernel tuned for
 *     isolated execution plus one per concurrency degree (CD), found by
 *     tuning under resource constraints (fewer CUs).
 *   - Dynamic logic: Sec. 4.3 -- given the pending independent GEMMs,
 *     predict a CD from per-GEMM features with a multi-class logistic
 *     regression (Eq. 1), run min(CD, available) of them together, and
 *     bind each to the GO-Kernel tuned for that CD.
 *   - Execution configurations: Sec. 5.5 -- sequential, default (all
 *     GEMMs at once with isolation-tuned kernels), GO-Kernels, GOLDYLOC.
 *   - Heterogeneous sets: Sec. 6.7 -- GEMMs run together only if all of
 *     them prefer that CD; otherwise they are split into smaller sets.
 *
 * Storage reading (the paper fixes no base layout): every matrix is
 * row-major with a leading dimension in elements.
 *   op(A)(i,k) = A[i*lda + k]  (trans_a = 0)   or A[k*lda + i] (trans_a = 1)
 *   op(B)(k,j) = B[k*ldb + j]  (trans_b = 0)   or B[j*ldb + k] (trans_b = 1)
 *   C[i*ldc + j] = round(scale_a * scale_b * sum_k op(A)(i,k) op(B)(k,j))
 * with fp32 accumulation, alpha = 1 apart from the fp8 scales, beta = 0
 * (C is overwritten) and round-to-nearest-even into the output type.
 *
 * Supported (a_type, b_type, c_type): (F16, F16, F16), (BF16, BF16, BF16),
 * (FP8_E4M3, FP8_E4M3, BF16), (F32, F32, F32).  FP8_E4M3 is the OCP "E4M3FN"
 * encoding (bias 7, largest finite 448, no infinities).  F32 runs on the
 * fp32 MFMAs (the full-precision GEMMs of Sec. 5.2 and 6.8) and stores C
 * unrounded.
 *
 * Ownership: all matrices are device buffers owned by the caller, who keeps
 * them alive until the origin stream passes the work.  The library owns its
 * stream pool, events, split-K workspace and plan state.  No call allocates
 * device memory after gdy_create.
 *
 * Errors: every call returns a gdy_status; nothing is thrown across the ABI.
 * gdy_execute validates all descriptors before launching anything (all or
 * nothing); gdy_last_error() gives a message for the most recent failure.
 * A context is not thread-safe: use one per host thread, or lock.
 *
 * Environment: HIP maps streams onto GPU_MAX_HW_QUEUES hardware queues per
 * process (4 by default); set it to cover the stream pool plus the caller's
 * streams (24 for the default 16-stream pool) before the process first
 * touches HIP, or concurrent GEMMs share queues and serialise.
 */
#ifndef GDY_H
#define GDY_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define GDY_MAX_GEMMS 256   /* most GEMMs in one submission                   */
#define GDY_N_CD 5          /* CD classes 1, 2, 4, 8, 16 (Sec. 4.3)           */
#define GDY_N_FEATURES 18   /* M, N, K, then (#WGs, occupancy, #waves) per CD */

typedef enum {
  GDY_OK = 0,
  GDY_ERR_INVALID_ARG = 1, /* null pointer, negative size, bad ld, bad mode, bad scale */
  GDY_ERR_UNSUPPORTED = 2, /* dtype triple, alignment or extent the kernels cannot take */
  GDY_ERR_ALIAS = 3,       /* a C range overlaps an A, B or C range of the submission */
  GDY_ERR_TOO_MANY = 4,    /* n > GDY_MAX_GEMMS                                      */
  GDY_ERR_TABLE = 5,       /* reserved: a bad GO table falls back instead (gdy_create)  */
  GDY_ERR_HIP = 6,         /* a HIP runtime call failed                              */
  GDY_ERR_NOMEM = 7        /* host allocation failed                                 */
} gdy_status;

typedef enum { GDY_F16 = 1, GDY_BF16 = 2, GDY_FP8_E4M3 = 3, GDY_F32 = 4 } gdy_dtype;

/* Execution configurations (Sec. 5.5). */
typedef enum {
  GDY_SEQUENTIAL = 0, /* isolation-tuned kernel per GEMM, one after another on the origin stream */
  GDY_DEFAULT = 1,    /* isolation-tuned kernels, all n GEMMs at once, one stream each           */
  GDY_GO = 2,         /* GO-Kernels for CD = n, all at once (forced_cd > 0: groups of forced_cd
                         in submission order, one after another)                          */
  GDY_SELECTOR = 3,   /* GOLDYLOC: predicted CD per GEMM, grouping, GO-Kernels per group        */
  GDY_FORCED = 4,     /* each GEMM's `variant`, round-robin over forced_cd streams (tuning)     */
  GDY_FORCED_GROUPED = 5, /* each GEMM's `variant`; consecutive runs of forced_cd GEMMs form
                             groups run one after another, dispatched as GO and SELECTOR
                             groups are (tuning)                                            */
  /* CU-Partition (Sec. 5.5, Sec. 6.9): P = forced_cd (2, 4 or 8; 0: the
     smallest of them >= the number of GEMMs, at most 8) streams on disjoint
     CU masks of CUs/P each; GEMM t of the submission runs on partition
     t mod P (plan.stream_of), one dispatch per GEMM.  Needs a context
     created with use_cu_masks & 2.  The three differ in the kernels:      */
  GDY_CU_PARTITION = 6,    /* isolation-tuned kernels (the paper's CU-Partition)             */
  GDY_CU_PARTITION_GO = 7, /* the GO-Kernels of CD class P, tuned for the unpartitioned GPU    */
  GDY_CU_PARTITION_RC = 8  /* the kernels tuned under CUs/P CUs (the GO table's partition
                              kernels; GO-Kernels of class P where the table has none)       */
} gdy_mode;

/*
 * Dispatch of a group (GO, SELECTOR, FORCED_GROUPED): the GEMMs of a group
 * that are bound to the same kernel share ONE kernel dispatch (up to 16 per
 * dispatch; each GEMM keeps its own grid cap as its share of the grid) in
 * launch order.  The first dispatch of a group runs on the origin stream,
 * further ones on pool streams forked from and joined back to it.  A
 * hardware queue switch costs tens of microseconds on MI355X, far more than
 * the small GEMMs of a group take, so the concurrency of a group lives in one
 * grid wherever its kernels allow.  Each tile is computed by the same code as
 * in an isolated launch, so results are bit-identical.  In GO and SELECTOR,
 * dispatches of a group whose kernels belong to one family (256 x 256 tiles;
 * smaller ones) and input type run jointly in one kernel launch, each GEMM on
 * tiles of its own kernel's size or, where that is estimated to be faster, of
 * the other family's, with the same bits: the plan still counts a
 * dispatch per kernel, and they share a stream slot and, in the timings, an
 * interval.  SEQUENTIAL, DEFAULT and FORCED launch one dispatch per GEMM.
 */
#define GDY_MAX_FUSED 16

/* What an entry of a submission computes.  GDY_OP_ADD is the non-GEMM
 * co-runner of Sec. 7.1: C[i][j] = A[i][j] + B[i][j] over an M x N region
 * (A and B M x N with lda, ldb >= N; k must be 0; trans flags 0; a_type ==
 * b_type == c_type in {F16, BF16, F32}; the sum is formed in fp32 and
 * rounded once).  The selector lets an add join any group (it restricts
 * no concurrency); the GEMMs' predicted degrees decide whether it co-runs. */
typedef enum { GDY_OP_GEMM = 0, GDY_OP_ADD = 1 } gdy_op;

/* One GEMM (or element-wise add) of a submission. */
typedef struct {
  int64_t m, n, k;                  /* sizes; m or n == 0 is a no-op, k == 0 writes zeros   */
  int32_t a_type, b_type, c_type;   /* gdy_dtype values                                     */
  int32_t trans_a, trans_b;         /* T1, T2: 0 or 1 (see storage reading above)          */
  const void* a; int64_t lda;       /* device pointers; leading dimensions in elements      */
  const void* b; int64_t ldb;
  void* c;       int64_t ldc;       /* ldc >= n                                             */
  float scale_a, scale_b;           /* fp8 per-tensor scales; must be 1.0f for other types  */
  int32_t tenant;                   /* caller's tag, reported back in per-kernel timings    */
  int32_t variant;                  /* GDY_FORCED: variant id to use; otherwise ignored     */
  /* Strided batch (B-GEMM, Sec. 6.7): `batch` independent GEMMs of this
   * shape; item b reads A + b*stride_a, B + b*stride_b and writes
   * C + b*stride_c (strides in elements).  batch 0 or 1: a single GEMM and
   * the strides are ignored.  C items must not overlap each other; A and B
   * items may (stride 0 broadcasts one operand).  Every item obeys the
   * single-GEMM extent limits; strides are at most 2^44. */
  int32_t batch;
  int32_t op;                       /* gdy_op: what this entry computes (0: a GEMM)         */
  int64_t stride_a, stride_b, stride_c;
} gdy_gemm;

/* A plan: how a submission is grouped, streamed and bound to variants. */
typedef struct {
  int32_t n;                            /* GEMMs planned                                   */
  int32_t cd;                           /* largest number of GEMMs launched together       */
  int32_t n_groups;                     /* groups run one after another                    */
  int32_t fallback;                     /* 1: no usable GO table (isolated heuristics), or a
                                           GEMM whose type and layout it holds no shape of
                                           (kernels of a sibling's shapes, see gdy_create)  */
  int32_t order[GDY_MAX_GEMMS];         /* launch order: order[t] is a GEMM index          */
  int32_t group_of[GDY_MAX_GEMMS];      /* group of GEMM i                                 */
  int32_t stream_of[GDY_MAX_GEMMS];     /* pool stream slot of GEMM i's dispatch (-1: origin) */
  int32_t variant_of[GDY_MAX_GEMMS];    /* variant id bound to GEMM i (-1: not launched)   */
  int32_t pred_cd[GDY_MAX_GEMMS];       /* selector: min(predicted CD, n) of GEMM i, else 0 */
  int32_t group_size[GDY_MAX_GEMMS];    /* size of group g (first n_groups entries)        */
  int32_t n_dispatches;                 /* kernel dispatches of the submission              */
  int32_t dispatch_of[GDY_MAX_GEMMS];   /* dispatch that runs GEMM i (-1: none); dispatches
                                           are numbered in launch order                    */
  int32_t split_of[GDY_MAX_GEMMS];      /* split-K runs of GEMM i (1: none; 0: not launched) */
} gdy_plan_t;

/*
 * Split-K (all modes; a property of the library's kernels, not of the
 * paper).  A GEMM whose tiles fill at most half of the CU slots its kernel
 * has (CUs x occupancy; a grid cap does not count) and whose K is long runs
 * each tile as S work items over consecutive runs of K tiles: S is the
 * largest power of two up to 16 with S x tiles within the slots, at least
 * 16 K tiles per run (32 in other types than fp32 where the tiles alone are
 * as many as the CUs) and at most 16 MiB of fp32 partial planes; kernels with
 * tiles above 128 x 128 do not split.  A GEMM that 16 K tiles a run would
 * split runs without its variant's grid cap.  S depends only on the GEMM and its
 * kernel -- never on what runs at the same time -- so a variant gives a GEMM
 * the same bits alone and concurrent.  Each run writes an fp32 M x N plane
 * into a workspace the context allocates at creation (256 MiB); a reduction
 * kernel on the dispatch's stream sums the planes in run order, scales,
 * rounds and stores C.  The split GEMMs of a group take consecutive regions
 * of the workspace and groups reuse it (in SEQUENTIAL each GEMM starts at
 * the beginning); a split GEMM that no longer fits in what its group has
 * left moves, with its split, to a group appended after the others (the plan
 * shows it).  Submissions of one context must be ordered (one origin stream
 * at a time): they share the workspace.
 */

/* Static description of one catalogue variant (a kernel plus its grid cap). */
typedef struct {
  char name[64];
  int32_t dtype, trans_a, trans_b;
  int32_t bm, bn, bk;       /* macro tile                                              */
  int32_t waves;            /* waves per workgroup                                     */
  int32_t mfma;             /* MFMA block edge (32 or 16)                              */
  int32_t lds_bytes;        /* LDS per workgroup                                       */
  int32_t vgprs;            /* registers per lane reported by the runtime              */
  int32_t occupancy;        /* workgroups resident per CU (runtime occupancy query)    */
  int32_t grid_cap_cus;     /* 0: one workgroup per tile; else grid = cap * occupancy  */
  int32_t direct;           /* 1: global->LDS copies; needs K % bk == 0 and 16-byte
                               aligned A/B bases and row pitches, else the staged
                               variant of the same tile and cap runs instead     */
  int32_t kind;             /* 0: a GEMM kernel; 1: the element-wise add (GDY_OP_ADD),
                               bm x bn is then its workgroup tile of elements    */
} gdy_variant_desc;

typedef struct gdy_ctx gdy_ctx;

/*
 * Create a context on HIP device `device` (the one-time set-up of Sec. 4.1:
 * the GO library tuned offline for this GPU, Sec. 4.2, and the concurrency
 * the runtime may use).  Loads the catalogue, queries each kernel's
 * occupancy, creates `max_streams` (1..64; 0 means 16) pool streams at
 * default priority and their events, and allocates the split-K workspace.
 * `table_path` names a GO table written by the offline tuner.  Without a
 * usable table -- NULL or "", missing, unreadable, built for another device
 * or naming a variant the library does not have -- the context still
 * returns GDY_OK: SELECTOR and GO modes fall back to isolated heuristics
 * (every GEMM at CD 1, i.e. isolated kernels one after another, Sec. 5.5's
 * sequential configuration) and every plan reports fallback = 1;
 * gdy_last_error() gives the reason until the next call.  A GEMM whose input
 * type and layout a usable table holds no shape of binds the kernels tuned for
 * a sibling (fp16 and bf16 for each other, else the type's untransposed
 * layout), on its own kernels of the closest tiles; its plans report fallback =
 * 1 too.  With nothing to borrow, and alone where it is a batch or fp32, it
 * runs its isolated heuristic.
 * `use_cu_masks` is a bit set: bit 0 creates one CU-masked stream for each
 * resource constraint GPU/2, GPU/4 and GPU/8 (isolated runs of the tuner);
 * bit 1 creates the CU-Partition streams (2 + 4 + 8 streams whose masks
 * split the CUs into 2, 4 or 8 disjoint parts).  Every stream needs its own
 * hardware queue (a CU mask is a queue property), so GPU_MAX_HW_QUEUES must
 * cover the pool, the masked streams and the caller's streams (24 for a
 * 16-stream pool alone; 32 for an 8-stream pool with partitions).  HIP
 * creates CU-masked streams as blocking streams, so work on the null stream
 * synchronises with all of them: give CU-Partition launches a created
 * origin stream (on the null stream a submission of 8 partitions measured
 * 2-3x slower).  On error *out is NULL.
 *
 * device < 0 creates a host-only context that plans without a GPU: its CU
 * count is GDY_HOST_CUS (default 256) or the loaded table's, kernel
 * occupancy comes from LDS size and wave count alone, the table's device
 * line is not checked, and gdy_execute returns GDY_ERR_UNSUPPORTED.
 */
gdy_status gdy_create(gdy_ctx** out, int device, const char* table_path, int32_t max_streams,
                      int32_t use_cu_masks);

/*
 * Resource constraint for subsequent launches (Sec. 4.2.1 "RC tuning"):
 * 0 = whole GPU; 128, 64 or 32 = launches that go to pool streams run on
 * the CU-masked streams restricted to that many CUs (needs use_cu_masks
 * bit 0 at create).  Pool streams carry every dispatch of GDY_DEFAULT and
 * GDY_FORCED (the tuner's isolated runs use GDY_FORCED with forced_cd 1)
 * and the further dispatches of a group (which therefore do not run jointly
 * with the first under a budget); what runs on the caller's origin
 * stream (GDY_SEQUENTIAL, a group's first dispatch) is not masked.  Other
 * values: GDY_ERR_INVALID_ARG.
 */
gdy_status gdy_set_rc(gdy_ctx* ctx, int32_t budget_cus);

/* Destroy a context: synchronises its streams, then frees streams and events. */
void gdy_destroy(gdy_ctx* ctx);

/*
 * Plan a submission without touching device memory (pointers are validated
 * for null/alias only and never dereferenced).  Sec. 4.3 dynamic logic for
 * SELECTOR; see gdy_mode for the others.  forced_cd: GO and FORCED modes
 * (0 = n); ignored otherwise.
 */
gdy_status gdy_plan(gdy_ctx* ctx, const gdy_gemm* gemms, int32_t n, int32_t mode,
                    int32_t forced_cd, gdy_plan_t* out);

/*
 * Plan and launch a submission: the problem statement of Sec. 4.1 -- given a
 * set of independent GEMMs, predict a performant CD and schedule that many
 * GEMMs at a time with the kernels tuned for it (SELECTOR, Sec. 4.3), or run
 * one of the other execution configurations of Sec. 5.5 (see gdy_mode).
 * `gemms` (host array of n descriptors, read during the call only) names
 * caller-owned device buffers.  Asynchronous to the host: the work is
 * ordered after what is already on `hip_stream` (a hipStream_t; NULL is the
 * null stream) and `hip_stream` is ordered after all of it when this
 * returns.  `out` (nullable) receives the plan.  Every descriptor is
 * validated before anything launches (all or nothing).  On GDY_ERR_HIP the
 * streams are still joined back to the origin stream.
 */
gdy_status gdy_execute(gdy_ctx* ctx, const gdy_gemm* gemms, int32_t n, int32_t mode,
                       int32_t forced_cd, void* hip_stream, gdy_plan_t* out);

/*
 * gdy_execute for callers that cannot allocate device memory (code under HIP
 * graph capture, tight serving loops, harnesses that forbid allocation):
 * the same plan and the same kernels as gdy_execute, with the split-K
 * planes in a static device array of GDY_STATIC_SCRATCH_BYTES that the
 * library holds on every device it runs on until the process ends, instead
 * of the context's workspace.  Allocates nothing, on the device or through
 * any allocating library routine.  A plan whose split GEMMs need more than
 * the array at once (one group's planes; one GEMM's in SEQUENTIAL) returns
 * GDY_ERR_UNSUPPORTED before anything launches.  Every call on a device
 * shares that device's array, which keeps the last call's partial planes
 * (each run overwrites its plane before the reduction reads it, so nothing
 * needs clearing): calls that overlap on one device, from any context or
 * thread, race and must be ordered by the caller.  Results are bit-identical
 * to gdy_execute's.
 */
#define GDY_STATIC_SCRATCH_BYTES (64ll * 1024 * 1024)
gdy_status gdy_execute_static(gdy_ctx* ctx, const gdy_gemm* gemms, int32_t n, int32_t mode,
                              int32_t forced_cd, void* hip_stream, gdy_plan_t* out);

/*
 * Epilogues: what a GEMM does with its fp32 sums before the one rounding into C.
 *   z(i,j) = scale_a * scale_b * sum_k op(A)(i,k) op(B)(k,j) + bias(j)
 *   forward  (grad = 0): C(i,j) = round(f(z) + R(i,j)); aux(i,j) = round(z) where
 *                        aux is given (a backward pass reads it)
 *   backward (grad = 1): C(i,j) = round(z * f'(aux(i,j)) + R(i,j)), aux the saved
 *                        pre-activation (not read for GDY_ACT_NONE)
 *   bias_grad(j) = the sum of column j of C before its rounding, in fp32 and in an
 *                  order that the plan fixes: the gradient of the bias that the
 *                  layer below added to aux.
 * f: the identity, max(z, 0), z Phi(z) (the normal distribution function), z (1 +
 * tanh(sqrt(2/pi) (z + 0.044715 z^3))) / 2, or z / (1 + exp(-z)).  The slope of
 * GDY_ACT_RELU at 0 is 0.  f of minus infinity is what the formula gives in floating
 * point (NaN but for GDY_ACT_RELU and GDY_ACT_NONE), slopes at infinities are the limits, 0
 * and 1.  A zeroed struct is no epilogue.
 */
typedef enum {
  GDY_ACT_NONE = 0,
  GDY_ACT_RELU = 1,
  GDY_ACT_GELU = 2,
  GDY_ACT_GELU_TANH = 3,
  GDY_ACT_SILU = 4
} gdy_act;

typedef struct {
  int32_t act;                      /* gdy_act                                              */
  int32_t grad;                     /* 0: forward, 1: backward                              */
  const void* bias;                 /* N values, or NULL                                    */
  int32_t bias_type;                /* of bias: C's type or GDY_F32 (ignored without bias)  */
  int32_t reserved;                 /* must be 0                                            */
  const void* residual; int64_t ldr;    /* R: M x N of C's type, or NULL; ldr >= n          */
  void* aux;            int64_t ldaux;  /* M x N of C's type, or NULL; ldaux >= n           */
  float* bias_grad;                 /* N values, or NULL; overwritten; at most 2^26 an entry  */
  /* between items of a strided batch (or groups, gdy_execute_grouped), in elements: bias 0
   * shares one bias, bias_grad 0 adds the items' sums up.  Ignored for a single GEMM. */
  int64_t stride_bias, stride_r, stride_aux, stride_bias_grad;
} gdy_epilogue;

/*
 * gdy_execute for GEMMs with epilogues: epilogues[i] belongs to gemms[i] (a
 * host array of n, read during the call only; NULL: no epilogues, exactly
 * gdy_execute).  The plan is gdy_execute's for the same GEMMs, and every mode takes
 * them; members with and without epilogues mix, and adds (GDY_OP_ADD) must have
 * none.  k = 0 gives z = bias; m = 0 writes nothing but a bias_grad of zeros.
 * A GEMM's fp32 sums are those of its plain launch, whatever runs beside it.  GEMMs
 * with an epilogue of at most 16 rows, an untransposed A, 16-byte aligned operands
 * and a short K (at most 8 KiB of a row of A, 4 KiB where B is not transposed) run
 * on a kernel of their own whatever kernel and split the plan names, which adds in
 * another order, alone and beside others alike.
 * R may be C itself (same pointer, ldr = ldc, stride_r = stride_c), as may a backward
 * pass's aux; otherwise no output (C, a written aux, bias_grad) may overlap anything
 * else that the submission reads or writes.
 * Every pointer is aligned to its elements.  The split-K workspace also holds the
 * partial column sums of a group's bias gradients: a group that needs more of both
 * than the workspace has is refused (GDY_ERR_UNSUPPORTED) before anything launches.
 * Replays of graphs captured from one context share its workspace too, and must be ordered.
 */
gdy_status gdy_execute_epilogue(gdy_ctx* ctx, const gdy_gemm* gemms, const gdy_epilogue* epilogues, int32_t n,
                                int32_t mode, int32_t forced_cd, void* hip_stream, gdy_plan_t* out);
/* The same as gdy_execute_static is to gdy_execute: the workspace is the library's static array. */
gdy_status gdy_execute_epilogue_static(gdy_ctx* ctx, const gdy_gemm* gemms, const gdy_epilogue* epilogues,
                                       int32_t n, int32_t mode, int32_t forced_cd, void* hip_stream,
                                       gdy_plan_t* out);

/*
 * Products grouped by expert (the GEMMs of a mixture-of-experts layer): independent
 * products whose row counts only the device knows.  The rows of A are sorted by
 * group; group e holds the rows [offsets[e], offsets[e+1]) (device array of groups
 * + 1 values, not decreasing, 0 <= offsets[0], offsets[groups] <= rows; values outside
 * 0 .. rows are clamped to it, so that no offset leads outside the operands).
 *   GDY_OVER_ROWS: C[i][:] = epilogue(scale * A[i][:] op(B_e)) for the rows i of e:
 *                  A rows x k, B_e k x n (trans_b: stored n x k), C rows x n.  The
 *                  forward product, and with the other trans_b its input gradient.
 *                  Rows of no group are left as they were.
 *   GDY_OVER_K:    C_e = scale * A_e^T B_e + R_e, A_e and B_e the rows of e of A (rows
 *                  x k) and B (rows x n), C_e k x n: the weight gradient.  A group
 *                  without rows gives R_e or zeros.
 * with scale = scale_a * scale_b * scales[e].  Types, storage, rounding and
 * alignment as for gdy_gemm; several groups may share a B (stride_b 0).
 */
#define GDY_MAX_GROUPS 4096
typedef enum { GDY_OVER_ROWS = 0, GDY_OVER_K = 1 } gdy_over;

typedef struct {
  int32_t over;                     /* gdy_over                                             */
  int32_t groups;                   /* 0 .. GDY_MAX_GROUPS                                  */
  int64_t rows, n, k;
  int32_t a_type, b_type, c_type;   /* as gdy_gemm                                          */
  int32_t trans_b;                  /* GDY_OVER_K: 0                                        */
  const int32_t* offsets;           /* device                                               */
  const void* a; int64_t lda;       /* device pointers; leading dimensions in elements      */
  const void* b; int64_t ldb;
  int64_t stride_b;                 /* GDY_OVER_ROWS: elements between the groups of B      */
  void* c; int64_t ldc;
  int64_t stride_c;                 /* GDY_OVER_K: elements between the groups of C         */
  float scale_a, scale_b;           /* fp8 per-tensor scales; 1.0f for other types          */
  const float* scales;              /* device, one fp32 scale a group (fp8 only), or NULL   */
} gdy_grouped;

/*
 * Launch a grouped product on `hip_stream`, asynchronously.  `epilogue` may be NULL.
 * Over rows it applies to the rows of C as to a GEMM's: residual and aux are rows x
 * n, bias_grad is groups x n (stride_bias_grad 0: n sums over all groups) and bias
 * groups x n (stride_bias 0: shared); stride_r and stride_aux are ignored.  Over K
 * it may hold a residual only (R_e at stride_r; C itself accumulates into it).
 * Aliasing rules as for gdy_execute_epilogue.  Allocates nothing; bias gradients use the
 * context's split-K workspace (calls of one context, and replays of graphs captured from
 * them, must be ordered) and are refused
 * (GDY_ERR_UNSUPPORTED) where a fp32 row of n for each tile of 16 to 256 rows does
 * not fit into it.  Over K, A and B must end within 2 GiB; over rows only a group's B,
 * and 512 rows of A and of C, have to.
 */
gdy_status gdy_execute_grouped(gdy_ctx* ctx, const gdy_grouped* product, const gdy_epilogue* epilogue,
                               void* hip_stream);

/*
 * The tile of C, rows x cols, that a workgroup of gdy_execute_grouped computes for this
 * product (its last tiles of 256 rows may run as halves); 0 x 0 where no workgroup
 * runs.  Checks the product as the call does; host only, also on host-only contexts.
 */
gdy_status gdy_grouped_tile(gdy_ctx* ctx, const gdy_grouped* product, int32_t* rows, int32_t* cols);

/*
 * Activation and bias gradients that no product precedes:
 *   dz(i,j) = round(dy(i,j) * f'(z(i,j)));  bias_grad_e(j) = the sum of dy * f'(z) over the rows of e,
 * before its rounding, in fp32 and in an order that the sizes and offsets fix.  All
 * matrices are rows x n of `type` (F16, BF16 or F32).  offsets as for gdy_grouped (rows
 * of no group are left as they were), or NULL: one group of all rows.  dz may be
 * dy or z itself (same pointer and leading dimension).  Asynchronous on `hip_stream`;
 * allocates nothing.  Bias gradients of more than 32 rows, or of groups, use the context's
 * split-K workspace, as gdy_execute_grouped's do (calls of one context, and replays of
 * graphs captured from them, must be ordered), and are refused (GDY_ERR_UNSUPPORTED) where
 * a fp32 row of n for each 32 rows of a group does not fit into it.  512 rows of each matrix
 * must end within 2 GiB.
 */
typedef struct {
  int64_t rows, n;
  int32_t type;                     /* gdy_dtype                                            */
  int32_t act;                      /* gdy_act; GDY_ACT_NONE: z is not read                 */
  int32_t groups;                   /* with offsets: 0 .. GDY_MAX_GROUPS                    */
  int32_t reserved;                 /* must be 0                                            */
  const int32_t* offsets;           /* device, or NULL                                      */
  const void* dy; int64_t lddy;
  const void* z;  int64_t ldz;
  void* dz;       int64_t lddz;     /* or NULL: bias_grad only                              */
  float* bias_grad;                 /* groups x n (without offsets n), or NULL: dz only     */
  int64_t stride_bias_grad;         /* elements between groups; 0: sums over all groups     */
} gdy_act_grad;
gdy_status gdy_execute_act_grad(gdy_ctx* ctx, const gdy_act_grad* op, void* hip_stream);

/*
 * Tokens and experts: what a mixture of experts does around its grouped products.  Token t
 * sends a row to each of its top_k experts; slots (device, tokens x top_k, contiguous) names
 * the row of every pair (t, j) among the rows sorted by expert, -1: none.  No two pairs of a
 * call may have the same row; slots outside 0 .. rows - 1 are none.  Rows that no slot names
 * are left as they were.  All calls are asynchronous on `hip_stream` and allocate nothing;
 * outputs may overlap nothing else but where it is said.  Leading dimensions are at most
 * 2^44, a matrix ends within 2^63 bytes, at any alignment of its elements.
 *
 * Routing: ids[t * ld_ids + j] is the expert of pair (t, j); ids outside 0 .. experts - 1 are none
 * (the share of another GPU, padding).  The pairs sorted by expert, those of one expert in
 * the order of t * top_k + j, are the rows:
 *   offsets[e] = the number of pairs of the experts below e (experts + 1 values: the
 *                bounds of gdy_execute_grouped)
 *   slots[t * top_k + j] = the row of the pair, -1 where it has none
 * All of both are written.  More than GDY_ROUTE_ALONE pairs may use the context's split-K workspace
 * (calls of one context, and replays of graphs captured from them, must be ordered).
 */
#define GDY_MAX_TOP_K 64
#define GDY_ROUTE_ALONE 2048
typedef struct {
  int64_t tokens;                   /* tokens x top_k at most 2^24                          */
  int32_t top_k;                    /* 1 .. GDY_MAX_TOP_K                                   */
  int32_t experts;                  /* 0 .. GDY_MAX_GROUPS                                  */
  const void* ids; int64_t ld_ids;  /* device, tokens x top_k                               */
  int32_t id_bytes;                 /* 4 or 8: int32_t or int64_t                           */
  int32_t reserved;                 /* must be 0                                            */
  int32_t* slots;                   /* device, tokens x top_k                               */
  int32_t* offsets;                 /* device, experts + 1                                  */
} gdy_route;
gdy_status gdy_execute_route(gdy_ctx* ctx, const gdy_route* op, void* hip_stream);

/*
 * Rows to the experts, and the gradient of the weighted sum that brings them back:
 *   out[slots(t,j)][:] = round(w(t,j) * x[t][:])           (without weights: x[t][:] itself)
 *   weight_grad(t,j) = sum_c x[t][c] * z[slots(t,j)][c]     (0 where the pair has no row)
 * With x the gradient of gdy_execute_combine's y, out is the gradient of its z and
 * weight_grad that of its weights.  The gradient of out with respect to x is
 * gdy_execute_combine without weights.
 */
typedef struct {
  int64_t tokens, rows, n;          /* x: tokens x n; out, z: rows x n                      */
  int32_t top_k;                    /* 1 .. GDY_MAX_TOP_K                                   */
  int32_t type;                     /* F16, BF16, F32; without weights FP8_E4M3 too         */
  const int32_t* slots;
  const void* x; int64_t ldx;
  const void* weights;              /* device, tokens x top_k, contiguous, or NULL: 1       */
  int32_t weights_type;             /* GDY_F32 or `type` (ignored without weights)          */
  int32_t reserved;                 /* must be 0                                            */
  void* out; int64_t ldo;
  const void* z; int64_t ldz;       /* read for weight_grad                                 */
  float* weight_grad;               /* device, tokens x top_k, or NULL; needs weights and z */
} gdy_scatter;
gdy_status gdy_execute_scatter(gdy_ctx* ctx, const gdy_scatter* op, void* hip_stream);

/*
 * Rows back from the experts: y[t][:] = round(sum_j w(t,j) * z[slots(t,j)][:] + R[t][:]), in fp32
 * in the order of j.  y may be R itself (same pointer and leading dimension).
 */
typedef struct {
  int64_t tokens, rows, n;          /* y, R: tokens x n; z: rows x n                        */
  int32_t top_k;                    /* 1 .. GDY_MAX_TOP_K                                   */
  int32_t type;                     /* F16, BF16 or F32                                     */
  const int32_t* slots;
  const void* z; int64_t ldz;
  const void* weights;              /* device, tokens x top_k, contiguous, or NULL: 1       */
  int32_t weights_type;             /* GDY_F32 or `type` (ignored without weights)          */
  int32_t reserved;                 /* must be 0                                            */
  const void* residual; int64_t ldr;  /* R, or NULL                                         */
  void* y; int64_t ldy;
} gdy_combine;
gdy_status gdy_execute_combine(gdy_ctx* ctx, const gdy_combine* op, void* hip_stream);

/*
 * Rows in 8-bit integers, a scale for each:
 *   scale_i = max_c |x[i][c]| / 127,  q[i][c] = 127 * x[i][c] / max_c |x[i][c]| rounded to
 * the nearest integer (the exact quotient, halves to even), so that scale_i * q[i][c] stands for
 * x[i][c].  A row of zeros has scale 0; a row that holds an infinity or a NaN has one of
 * them as its scale and codes of 0, so that its products are NaN.  With slots, row i of x goes
 * to the rows slots(i, 0 .. top_k - 1) of q and scales (as gdy_execute_scatter's); without, to row i.
 */
typedef struct {
  int64_t rows, n;                  /* of x                                                 */
  int32_t type;                     /* of x: F16, BF16 or F32                               */
  int32_t top_k;                    /* with slots: 1 .. GDY_MAX_TOP_K; otherwise 0          */
  const void* x; int64_t ldx;
  const int32_t* slots;             /* device, rows x top_k, or NULL                        */
  int64_t out_rows;                 /* with slots: rows of q and scales; otherwise 0        */
  int8_t* q; int64_t ldq;
  float* scales;                    /* device, a value a row of q                           */
} gdy_quantize;
gdy_status gdy_execute_quantize(gdy_ctx* ctx, const gdy_quantize* op, void* hip_stream);

/*
 * Products of 8-bit integers with a scale for each row of A (token) and each column of C
 * (channel):
 *   z(i,j) = row_scales[i] * col_scales[j] * sum_k A[i][k] op(B)(k,j) + bias(j)
 *   C(i,j) = round(f(z) + R(i,j))
 * The sums are exact (32-bit integers; k is at most 131071); each of the products with the
 * scales, and the rest, is fp32.  With offsets, a product grouped by expert over rows, as
 * gdy_execute_grouped: the rows offsets[e] .. offsets[e+1] - 1 of A and C belong to group e, with
 * its own B, column scales and bias; offsets do not decrease and are clamped to 0 .. rows; rows of no
 * group are left as they were.  Without, one product of all rows (groups and the strides are ignored).  The epilogue
 * may hold a bias, an activation and a residual (R may be C itself; stride_bias counts
 * between groups).  Allocates nothing and uses no workspace.  A group's B, and 512 rows of A and
 * of C, must end within 2 GiB.  Non-finite scales give what the formulas give.
 */
typedef struct {
  int64_t rows, n, k;               /* A rows x k, B k x n (trans_b: n x k), C rows x n     */
  int32_t c_type;                   /* F16, BF16 or F32                                     */
  int32_t trans_b;                  /* 0 or 1                                               */
  int32_t groups;                   /* with offsets: 0 .. GDY_MAX_GROUPS                    */
  int32_t reserved;                 /* must be 0                                            */
  const int32_t* offsets;           /* device, or NULL                                      */
  const int8_t* a; int64_t lda;
  const int8_t* b; int64_t ldb;
  int64_t stride_b;                 /* between groups of B                                  */
  const float* row_scales;          /* device, rows values, or NULL: 1                      */
  const float* col_scales;          /* device, n values a group, or NULL: 1                 */
  int64_t stride_col_scales;        /* between groups; 0: shared                            */
  void* c; int64_t ldc;
} gdy_integer;
gdy_status gdy_execute_integer(gdy_ctx* ctx, const gdy_integer* product, const gdy_epilogue* epilogue,
                               void* hip_stream);
/* The tile of C that a workgroup of gdy_execute_integer computes for this product, as
 * gdy_grouped_tile tells it. */
gdy_status gdy_integer_tile(gdy_ctx* ctx, const gdy_integer* product, int32_t* rows, int32_t* cols);

/*
 * Per-kernel timing (Sec. 5.3 measures each GEMM's kernel runtime, with the
 * GEMMs run back-to-back on their streams).  When enabled, every dispatch
 * of gdy_execute records a start and a stop event on the stream it runs on
 * (hipExtLaunchKernel), and a submission start event on the origin stream.
 * After the caller has synchronised, gdy_last_kernel_times fills
 * start_ms[i] / end_ms[i] (host arrays of n floats; milliseconds from the
 * submission start) for GEMM i of the last submission; GEMMs that launched
 * nothing get -1.  GEMMs that share a dispatch report that dispatch's
 * interval (a split GEMM's interval ends with its reduction).
 * GDY_ERR_INVALID_ARG when no timed submission exists or a pointer is NULL.
 */
gdy_status gdy_set_timing(gdy_ctx* ctx, int32_t enable);
gdy_status gdy_last_kernel_times(gdy_ctx* ctx, float* start_ms, float* end_ms, int32_t n);
/* Same for an earlier timed submission: back = 0 is the last one, up to 63
 * (the context keeps the events of the last 64 timed submissions). */
gdy_status gdy_kernel_times(gdy_ctx* ctx, int32_t back, float* start_ms, float* end_ms,
                            int32_t n);

/*
 * Dispatch map (host only; works on host-only contexts): plans the
 * submission as gdy_plan does, builds launch block `dispatch` of the plan
 * as gdy_execute would, and reports what each of its workgroups computes,
 * with the kernels' own mapping code (workgroups of other dispatches that run
 * jointly with it are reported idle).  *grid receives the launch's
 * workgroup count; for workgroup b < min(*grid, max_workgroups),
 * gemm_of_wg[b] is the submission index of the member it serves (-1: an
 * idle workgroup) and it runs that member's work items first_item[b],
 * first_item[b] + item_stride[b], ... below the member's item count.
 * items_of_gemm (n entries) receives each member's work items in this
 * dispatch (tiles x batch items x split runs; 0 for GEMMs of other
 * dispatches).  Lets a caller check on the CPU that every work item of a
 * dispatch is computed exactly once (XCD placement included).
 */
gdy_status gdy_dispatch_map(gdy_ctx* ctx, const gdy_gemm* gemms, int32_t n, int32_t mode, int32_t forced_cd,
                            int32_t dispatch, int32_t max_workgroups, int32_t* grid, int32_t* gemm_of_wg,
                            int32_t* first_item, int32_t* item_stride, int64_t* items_of_gemm);

/* Features of one GEMM (Sec. 4.3): M, N, K, then for each CD class
 * 1, 2, 4, 8, 16 the bound variant's #WGs, occupancy and #waves. */
gdy_status gdy_features(gdy_ctx* ctx, const gdy_gemm* gemm, double* out_features);

/* Catalogue queries.  Variant ids are 0 .. gdy_variant_count()-1. */
int32_t gdy_variant_count(gdy_ctx* ctx);
gdy_status gdy_variant_info(gdy_ctx* ctx, int32_t id, gdy_variant_desc* out);
int32_t gdy_variant_find(gdy_ctx* ctx, const char* name); /* -1 if absent */
/* Isolated (CD 1) variant the library binds to a GEMM, from the table or heuristics. */
int32_t gdy_isolated_variant(gdy_ctx* ctx, const gdy_gemm* gemm);
/* FNV-1a hash of the catalogue's variant names, as stored in GO tables. */
uint64_t gdy_catalogue_hash(gdy_ctx* ctx);
/* Number of compute units of the context's device. */
int32_t gdy_device_cus(gdy_ctx* ctx);

const char* gdy_status_string(gdy_status s);
const char* gdy_last_error(gdy_ctx* ctx); /* valid until the next call on ctx; "" if none */

#ifdef __cplusplus
}
#endif

#endif /* GDY_H */
