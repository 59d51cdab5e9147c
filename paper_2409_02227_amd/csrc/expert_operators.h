// expert_operators.h -- host side of routing, scatter, combine, quantisation and products
// of 8-bit integers: checks, tile choice, launches.  Part of gdy.cpp, behind operators.h.
#pragma once

namespace {

bool good_ld(int64_t ld, int64_t n) { return ld >= n && ld <= kMaxStride; }

// Whether 64-bit byte offsets reach the end of a matrix: 2^31 rows of 2^44 elements pass them.
bool good_extent(int64_t rows, int64_t n, int64_t ld, int es) {
  return rows <= 1 || ((__int128)(rows - 1) * ld + n) * es <= INT64_MAX;
}

bool row_type(int32_t t) { return t == GDY_F16 || t == GDY_BF16 || t == GDY_F32; }

// Sizes of the operators by token.
gdy_status check_tokens(gdy_ctx* ctx, const char* what, int64_t tokens, int64_t rows, int64_t n, int32_t top_k) {
  if (tokens < 0 || rows < 0 || n < 0) return fail(ctx, GDY_ERR_INVALID_ARG, "%s: negative size", what);
  if (top_k < 1 || top_k > GDY_MAX_TOP_K)
    return fail(ctx, GDY_ERR_INVALID_ARG, "%s: top_k %d is not 1 to %d", what, top_k, GDY_MAX_TOP_K);
  if (tokens > INT32_MAX - 4096 || rows > INT32_MAX - 4096 || n > INT32_MAX / 8)
    return fail(ctx, GDY_ERR_UNSUPPORTED, "%s: sizes too large", what);
  return GDY_OK;
}

// The weights of pairs: their type, place and range.
gdy_status check_weights(gdy_ctx* ctx, const char* what, const void* weights, int32_t weights_type, int32_t type,
                         int64_t pairs, std::vector<Range>* ranges) {
  if (!weights) return GDY_OK;
  if (weights_type != GDY_F32 && weights_type != type)
    return fail(ctx, GDY_ERR_UNSUPPORTED, "%s: weights of type %d, rows of %d", what, weights_type, type);
  const int ws = elem_size(weights_type);
  if ((uintptr_t)weights % ws) return fail(ctx, GDY_ERR_UNSUPPORTED, "%s: weights not element aligned", what);
  ranges->push_back({matrix_range(weights, 1, pairs, 0, 1, 0, ws), false, 0});
  return GDY_OK;
}

// Threads that share a row of `units` pieces of work, as a power of two of at most kRowThreads.
int row_threads_log(int64_t units) {
  int l = 0;
  while ((1 << l) < kRowThreads && (1 << l) < units) ++l;
  return l;
}

// Workgroups for `rows` rows; kernels loop where so many are not enough.
const int kMostRowGrid = 1 << 21;
unsigned row_grid(int64_t rows, int tpr_log) {
  const int64_t per = kRowThreads >> tpr_log;
  return (unsigned)std::min<int64_t>((rows + per - 1) / per, kMostRowGrid);
}

hipError_t launch_rows(const void* func, void* args, int64_t rows, int tpr_log, hipStream_t hs) {
  void* argv[] = {args};
  return hipExtLaunchKernel(func, dim3(row_grid(rows, tpr_log)), dim3(kRowThreads), argv, 0, hs, nullptr, nullptr, 0);
}

// ---------------------------------------------------------------------------
// Routing
// ---------------------------------------------------------------------------
gdy_status validate_route(gdy_ctx* ctx, const gdy_route& g) {
  if (g.tokens < 0 || g.experts < 0) return fail(ctx, GDY_ERR_INVALID_ARG, "route: negative size");
  if (g.top_k < 1 || g.top_k > GDY_MAX_TOP_K)
    return fail(ctx, GDY_ERR_INVALID_ARG, "route: top_k %d is not 1 to %d", g.top_k, GDY_MAX_TOP_K);
  if (g.experts > GDY_MAX_GROUPS)
    return fail(ctx, GDY_ERR_TOO_MANY, "route: %d experts > %d", g.experts, GDY_MAX_GROUPS);
  if ((g.id_bytes != 4 && g.id_bytes != 8) || g.reserved != 0)
    return fail(ctx, GDY_ERR_INVALID_ARG, "route: id_bytes must be 4 or 8, reserved 0");
  if (g.tokens > ((int64_t)1 << 24) / g.top_k)
    return fail(ctx, GDY_ERR_UNSUPPORTED, "route: more than 2^24 pairs");
  if (!g.offsets || (uintptr_t)g.offsets % 4) return fail(ctx, GDY_ERR_INVALID_ARG, "route: null or unaligned offsets");
  std::vector<Range> ranges;
  ranges.push_back({matrix_range(g.offsets, 1, (int64_t)g.experts + 1, 0, 1, 0, 4), true, 0});
  if (g.tokens > 0) {
    if (!g.ids || !g.slots || (uintptr_t)g.slots % 4 || (uintptr_t)g.ids % g.id_bytes)
      return fail(ctx, GDY_ERR_INVALID_ARG, "route: null or unaligned ids or slots");
    if (!good_ld(g.ld_ids, g.top_k)) return fail(ctx, GDY_ERR_INVALID_ARG, "route: bad ld_ids");
    if (!good_extent(g.tokens, g.top_k, g.ld_ids, g.id_bytes))
      return fail(ctx, GDY_ERR_UNSUPPORTED, "route: ids past 64-bit offsets");
    ranges.push_back({matrix_range(g.ids, g.tokens, g.top_k, g.ld_ids, 1, 0, g.id_bytes), false, 0});
    ranges.push_back({matrix_range(g.slots, 1, g.tokens * g.top_k, 0, 1, 0, 4), true, 0});
  }
  return check_ranges(ctx, ranges);
}

static_assert(GDY_MAX_GROUPS == kMaxExperts, "the kernels' tables hold every expert");

gdy_status launch_route(gdy_ctx* ctx, const gdy_route& g, hipStream_t hs) {
  KRoute a;
  std::memset(&a, 0, sizeof a);
  a.ids = g.ids;
  a.slots = g.slots;
  a.offsets = g.offsets;
  a.ld_ids = g.ld_ids;
  a.pairs = (int32_t)(g.tokens * g.top_k);
  a.top_k = g.top_k;
  a.experts = g.experts;
  a.bits = ceil_log2(g.experts);
  a.wide = g.id_bytes == 8;
  a.dense = g.ld_ids == g.top_k || g.tokens <= 1;
  a.expert_threads = 1 << std::max(ceil_log2(g.experts), 6);
  const bool few = g.experts <= kRouteFew;
  // A step costs a workgroup about 1 us, a second launch 3: 2048 pairs in one part 6.2 us, in two 6.8, 4096 9.2
  // and 7.1.  2^20 pairs of 64 experts in 256 parts 17.5 us, in 128 24.9, in 1024 31.
  const bool alone = a.pairs <= GDY_ROUTE_ALONE;
  const int part = kRoutePart * (alone ? 1 : 256);
  a.steps = std::max(std::min((a.pairs + part - 1) / part, kRouteMaxSteps), 1);
  a.parts = std::max((a.pairs + kRoutePart * a.steps - 1) / (kRoutePart * a.steps), 1);
  void* argv[] = {&a};
  auto launch = [&](const void* kernel, int grid) {
    return hipExtLaunchKernel(kernel, dim3(grid), dim3(kRoutePart), argv, 0, hs, nullptr, nullptr, 0);
  };
  if (!alone) {
    a.counts = (int32_t*)ctx->split_ws;  // at most 261 parts x 4096 experts and the totals: 4.1 MiB
    HIP_TRY(ctx, launch(route_count_kernel(few), a.parts));
    // Every workgroup of the last launch reads the counts, or a launch of its own sums them: 131072 pairs of 96 experts
    // (12288 counts) 9.8 and 10.7 us, of 128 (16384) 9.7 and 10.6, of 160 (20480) 12.2 and 10.9, of 256 12.1 and 10.8, of
    // 4096 83 and 20; 2^20 pairs of 64 (16384) 17.2 and 19.2, of 128 19.7 and 19.3; 16384 pairs of 1024 (16384) 11.3 and
    // 11.6, of 2048 15.9 and 13.6.
    if (a.parts * a.experts > 16384) {
      a.totals = a.counts + (int64_t)a.parts * a.experts;
      HIP_TRY(ctx, launch(route_sums_kernel(), (a.experts + 63) / 64));
    }
  }
  // Few pairs and experts take a workgroup of four waves in place of 16: 64 pairs of 16 experts 3.7 us and 3.9,
  // of 256 3.7 and 4.2.
  const bool small = few && a.pairs <= kRouteSmall * 64;
  const int waves = small ? kRouteSmall : kRoutePart / 64;
  HIP_TRY(ctx, hipExtLaunchKernel(route_slots_kernel(few, waves), dim3(a.parts), dim3(waves * 64), argv, 0, hs, nullptr,
                                  nullptr, 0));
  return GDY_OK;
}

// ---------------------------------------------------------------------------
// Rows to the experts and back
// ---------------------------------------------------------------------------
gdy_status validate_scatter(gdy_ctx* ctx, const gdy_scatter& g) {
  gdy_status s = check_tokens(ctx, "scatter", g.tokens, g.rows, g.n, g.top_k);
  if (s != GDY_OK) return s;
  if (!row_type(g.type) && !(g.type == GDY_FP8_E4M3 && !g.weights))
    return fail(ctx, GDY_ERR_UNSUPPORTED, "scatter: unsupported type %d", g.type);
  if (g.reserved != 0) return fail(ctx, GDY_ERR_INVALID_ARG, "scatter: reserved must be 0");
  if (g.weight_grad && !g.weights) return fail(ctx, GDY_ERR_INVALID_ARG, "scatter: weight_grad needs weights");
  if (g.tokens == 0) return GDY_OK;
  const int es = elem_size(g.type);
  const int64_t pairs = g.tokens * g.top_k;
  std::vector<Range> ranges;
  if (!g.slots || (uintptr_t)g.slots % 4) return fail(ctx, GDY_ERR_INVALID_ARG, "scatter: null or unaligned slots");
  ranges.push_back({matrix_range(g.slots, 1, pairs, 0, 1, 0, 4), false, 0});
  s = check_weights(ctx, "scatter", g.weights, g.weights_type, g.type, pairs, &ranges);
  if (s != GDY_OK) return s;
  if ((uintptr_t)g.weight_grad % 4) return fail(ctx, GDY_ERR_UNSUPPORTED, "scatter: weight_grad not element aligned");
  ranges.push_back({matrix_range(g.weight_grad, 1, pairs, 0, 1, 0, 4), true, 0});
  if (g.n > 0 && g.rows > 0) {
    if (!g.x || !g.out || (g.weight_grad && !g.z)) return fail(ctx, GDY_ERR_INVALID_ARG, "scatter: null x, out or z");
    if (!good_ld(g.ldx, g.n) || !good_ld(g.ldo, g.n) || (g.weight_grad && !good_ld(g.ldz, g.n)))
      return fail(ctx, GDY_ERR_INVALID_ARG, "scatter: a leading dimension < n or > 2^44");
    if (!good_extent(g.tokens, g.n, g.ldx, es) || !good_extent(g.rows, g.n, g.ldo, es) ||
        (g.weight_grad && !good_extent(g.rows, g.n, g.ldz, es)))
      return fail(ctx, GDY_ERR_UNSUPPORTED, "scatter: operands past 64-bit offsets");
    if (((uintptr_t)g.x | (uintptr_t)g.out | (g.weight_grad ? (uintptr_t)g.z : 0)) % es)
      return fail(ctx, GDY_ERR_UNSUPPORTED, "scatter: operands not element aligned");
    ranges.push_back({matrix_range(g.x, g.tokens, g.n, g.ldx, 1, 0, es), false, 0});
    ranges.push_back({matrix_range(g.out, g.rows, g.n, g.ldo, 1, 0, es), true, 0});
    if (g.weight_grad) ranges.push_back({matrix_range(g.z, g.rows, g.n, g.ldz, 1, 0, es), false, 0});
  }
  return check_ranges(ctx, ranges);
}

gdy_status launch_scatter(gdy_ctx* ctx, const gdy_scatter& g, hipStream_t hs) {
  // without rows or columns there is nothing to move; weight_grad is zeros
  const bool moves = g.n > 0 && g.rows > 0;
  if (g.tokens == 0 || (!moves && !g.weight_grad)) return GDY_OK;
  const int es = elem_size(g.type);
  KScatter a;
  std::memset(&a, 0, sizeof a);
  a.x = (const uint8_t*)g.x;
  a.out = (uint8_t*)g.out;
  a.z = (const uint8_t*)g.z;
  a.slots = g.slots;
  a.weights = g.weights;
  a.weight_grad = g.weight_grad;
  a.tokens = g.tokens;
  a.ldx = g.ldx * es;
  a.ldo = g.ldo * es;
  a.ldz = g.ldz * es;
  a.rows = moves ? (int32_t)g.rows : 0;
  a.n = moves ? (int32_t)g.n : 0;
  a.top_k = g.top_k;
  a.weights_f32 = g.weights_type == GDY_F32;
  a.tpr_log = row_threads_log(((int64_t)a.n * es + 15) / 16);
  HIP_TRY(ctx, launch_rows(scatter_kernel(g.type, g.weight_grad ? 2 : g.weights ? 1 : 0), &a, g.tokens, a.tpr_log, hs));
  return GDY_OK;
}

gdy_status validate_combine(gdy_ctx* ctx, const gdy_combine& g) {
  gdy_status s = check_tokens(ctx, "combine", g.tokens, g.rows, g.n, g.top_k);
  if (s != GDY_OK) return s;
  if (!row_type(g.type)) return fail(ctx, GDY_ERR_UNSUPPORTED, "combine: unsupported type %d", g.type);
  if (g.reserved != 0) return fail(ctx, GDY_ERR_INVALID_ARG, "combine: reserved must be 0");
  if (g.tokens == 0 || g.n == 0) return GDY_OK;
  const int es = elem_size(g.type);
  const int64_t pairs = g.tokens * g.top_k;
  std::vector<Range> ranges;
  if (!g.slots || (uintptr_t)g.slots % 4) return fail(ctx, GDY_ERR_INVALID_ARG, "combine: null or unaligned slots");
  ranges.push_back({matrix_range(g.slots, 1, pairs, 0, 1, 0, 4), false, 0});
  s = check_weights(ctx, "combine", g.weights, g.weights_type, g.type, pairs, &ranges);
  if (s != GDY_OK) return s;
  if (!g.y || (g.rows > 0 && !g.z)) return fail(ctx, GDY_ERR_INVALID_ARG, "combine: null y or z");
  if (!good_ld(g.ldy, g.n) || (g.rows > 0 && !good_ld(g.ldz, g.n)) || (g.residual && !good_ld(g.ldr, g.n)))
    return fail(ctx, GDY_ERR_INVALID_ARG, "combine: a leading dimension < n or > 2^44");
  if (!good_extent(g.tokens, g.n, g.ldy, es) || !good_extent(g.rows, g.n, g.ldz, es) ||
      (g.residual && !good_extent(g.tokens, g.n, g.ldr, es)))
    return fail(ctx, GDY_ERR_UNSUPPORTED, "combine: operands past 64-bit offsets");
  if (((uintptr_t)g.y | (uintptr_t)g.residual | (g.rows > 0 ? (uintptr_t)g.z : 0)) % es)
    return fail(ctx, GDY_ERR_UNSUPPORTED, "combine: operands not element aligned");
  ranges.push_back({matrix_range(g.y, g.tokens, g.n, g.ldy, 1, 0, es), true, 1});
  ranges.push_back({matrix_range(g.residual, g.tokens, g.n, g.ldr, 1, 0, es), false,
                    g.residual == g.y && g.ldr == g.ldy ? 1 : 0});
  if (g.rows > 0) ranges.push_back({matrix_range(g.z, g.rows, g.n, g.ldz, 1, 0, es), false, 0});
  return check_ranges(ctx, ranges);
}

gdy_status launch_combine(gdy_ctx* ctx, const gdy_combine& g, hipStream_t hs) {
  if (g.tokens == 0 || g.n == 0) return GDY_OK;
  const int es = elem_size(g.type);
  KCombine a;
  std::memset(&a, 0, sizeof a);
  a.z = (const uint8_t*)g.z;
  a.res = (const uint8_t*)g.residual;
  a.y = (uint8_t*)g.y;
  a.slots = g.slots;
  a.weights = g.weights;
  a.tokens = g.tokens;
  a.ldz = g.ldz * es;
  a.ldr = g.ldr * es;
  a.ldy = g.ldy * es;
  a.rows = (int32_t)g.rows;
  a.n = (int32_t)g.n;
  a.top_k = g.top_k;
  a.weights_f32 = g.weights_type == GDY_F32;
  a.tpr_log = row_threads_log((g.n * es + 15) / 16);
  HIP_TRY(ctx, launch_rows(combine_kernel(g.type), &a, g.tokens, a.tpr_log, hs));
  return GDY_OK;
}

// ---------------------------------------------------------------------------
// Rows to 8-bit integers
// ---------------------------------------------------------------------------
gdy_status validate_quantize(gdy_ctx* ctx, const gdy_quantize& g) {
  if (!g.slots && (g.top_k != 0 || g.out_rows != 0))
    return fail(ctx, GDY_ERR_INVALID_ARG, "quantize: top_k and out_rows belong to slots, 0 without them");
  const gdy_status s = check_tokens(ctx, "quantize", g.rows, g.out_rows, g.n, g.slots ? g.top_k : 1);
  if (s != GDY_OK) return s;
  if (!row_type(g.type)) return fail(ctx, GDY_ERR_UNSUPPORTED, "quantize: unsupported type %d", g.type);
  const int64_t out_rows = g.slots ? g.out_rows : g.rows;
  if (g.rows == 0 || out_rows == 0) return GDY_OK;
  const int es = elem_size(g.type);
  if ((uintptr_t)g.slots % 4 || !g.scales || (uintptr_t)g.scales % 4)
    return fail(ctx, GDY_ERR_INVALID_ARG, "quantize: unaligned slots, null or unaligned scales");
  std::vector<Range> ranges;
  ranges.push_back({matrix_range(g.slots, 1, g.rows * g.top_k, 0, 1, 0, 4), false, 0});
  ranges.push_back({matrix_range(g.scales, 1, out_rows, 0, 1, 0, 4), true, 0});
  if (g.n > 0) {
    if (!g.x || !g.q) return fail(ctx, GDY_ERR_INVALID_ARG, "quantize: null x or q");
    if (!good_ld(g.ldx, g.n) || !good_ld(g.ldq, g.n))
      return fail(ctx, GDY_ERR_INVALID_ARG, "quantize: a leading dimension < n or > 2^44");
    if (!good_extent(g.rows, g.n, g.ldx, es) || !good_extent(out_rows, g.n, g.ldq, 1))
      return fail(ctx, GDY_ERR_UNSUPPORTED, "quantize: operands past 64-bit offsets");
    if ((uintptr_t)g.x % es) return fail(ctx, GDY_ERR_UNSUPPORTED, "quantize: x not element aligned");
    ranges.push_back({matrix_range(g.x, g.rows, g.n, g.ldx, 1, 0, es), false, 0});
    ranges.push_back({matrix_range(g.q, out_rows, g.n, g.ldq, 1, 0, 1), true, 0});
  }
  return check_ranges(ctx, ranges);
}

gdy_status launch_quantize(gdy_ctx* ctx, const gdy_quantize& g, hipStream_t hs) {
  if (g.rows == 0 || (g.slots && g.out_rows == 0)) return GDY_OK;
  KQuantize a;
  std::memset(&a, 0, sizeof a);
  a.x = (const uint8_t*)g.x;
  a.q = g.q;
  a.scales = g.scales;
  a.slots = g.slots;
  a.rows = g.rows;
  a.ldx = g.ldx * elem_size(g.type);
  a.ldq = g.ldq;
  a.n = (int32_t)g.n;
  a.top_k = g.top_k;
  a.out_rows = (int32_t)g.out_rows;
  // Rows of more than 4096 elements take up to 1024 threads where there are few of them: (64, 16384) bf16 6.6 us on 256
  // and 4.8 on 1024, (512, 16384) 9.8 and 9.2, (1024, 8192) 9.2 and 8.8, (4096, 8192) 23.1 and 26.4.
  const int64_t units = (g.n + 15) / 16;
  const int threads = units > kRowThreads && units <= 2048 && g.rows <= 4 * ctx->cus ? 1024 : kRowThreads;
  while ((1 << a.tpr_log) < threads && (1 << a.tpr_log) < units) ++a.tpr_log;
  const int64_t steps = (units + (1 << a.tpr_log) - 1) >> a.tpr_log;
  const int64_t per = threads >> a.tpr_log;
  const int64_t grid = std::min<int64_t>((g.rows + per - 1) / per, kMostRowGrid);
  void* argv[] = {&a};
  HIP_TRY(ctx, hipExtLaunchKernel(quantize_kernel(g.type, steps <= 1 ? 1 : steps <= 2 ? 2 : kQuantMost, g.n % 16 == 0),
                                  dim3((unsigned)grid), dim3(threads), argv, 0, hs, nullptr, nullptr, 0));
  return GDY_OK;
}

// ---------------------------------------------------------------------------
// Products of 8-bit integers
// ---------------------------------------------------------------------------
const int64_t kMaxIntegerK = 131071;  // k * 128 * 128 < 2^31

gdy_status validate_integer(gdy_ctx* ctx, const gdy_integer& g, const gdy_epilogue* ep) {
  const bool grouped = g.offsets != nullptr;
  if (g.rows < 0 || g.n < 0 || g.k < 0 || (grouped && g.groups < 0))
    return fail(ctx, GDY_ERR_INVALID_ARG, "integer: negative size");
  if (grouped && g.groups > GDY_MAX_GROUPS)
    return fail(ctx, GDY_ERR_TOO_MANY, "integer: %d groups > %d", g.groups, GDY_MAX_GROUPS);
  if (!row_type(g.c_type)) return fail(ctx, GDY_ERR_UNSUPPORTED, "integer: unsupported type %d of C", g.c_type);
  if ((g.trans_b != 0 && g.trans_b != 1) || g.reserved != 0)
    return fail(ctx, GDY_ERR_INVALID_ARG, "integer: trans_b must be 0 or 1, reserved 0");
  if (g.k > kMaxIntegerK)
    return fail(ctx, GDY_ERR_UNSUPPORTED, "integer: k %lld > %lld, whose sums may pass 32 bits", (long long)g.k,
                (long long)kMaxIntegerK);
  if (ep && (ep->grad || ep->aux || ep->bias_grad))
    return fail(ctx, GDY_ERR_UNSUPPORTED, "integer: the epilogue may hold a bias, an activation and a residual only");
  const int64_t groups = grouped ? g.groups : 1;
  if (groups == 0 || g.rows == 0 || g.n == 0) return GDY_OK;
  // sizes are 32-bit on the device, row tiles and their columns one 31-bit count
  if (g.rows > INT32_MAX - 4096 || g.n > INT32_MAX - 4096 ||
      ((g.rows + 15) / 16 + groups) * ((g.n + 15) / 16) > INT32_MAX / 2)
    return fail(ctx, GDY_ERR_UNSUPPORTED, "integer: sizes too large");
  if ((uintptr_t)g.offsets % 4 || (uintptr_t)g.row_scales % 4 || (uintptr_t)g.col_scales % 4)
    return fail(ctx, GDY_ERR_INVALID_ARG, "integer: unaligned offsets or scales");
  const int os = g.c_type == GDY_F32 ? 4 : 2;
  if (!g.c) return fail(ctx, GDY_ERR_INVALID_ARG, "integer: null C");
  if (g.ldc < g.n) return fail(ctx, GDY_ERR_INVALID_ARG, "integer: ldc < n");
  if ((uintptr_t)g.c % os) return fail(ctx, GDY_ERR_UNSUPPORTED, "integer: C not element aligned");
  int64_t bytes;
  const int64_t tile_rows = std::min<int64_t>(g.rows, 256);
  if (!stored_extent(tile_rows, g.n, g.ldc, os, &bytes))
    return fail(ctx, GDY_ERR_UNSUPPORTED, "integer: rows of C too long");
  const bool many = groups > 1;
  if (many && g.col_scales && (g.stride_col_scales < 0 || (g.stride_col_scales > 0 && g.stride_col_scales < g.n)))
    return fail(ctx, GDY_ERR_INVALID_ARG, "integer: bad stride_col_scales");
  if (many && ((g.col_scales && g.stride_col_scales > kMaxStride) || g.stride_b > kMaxStride))
    return fail(ctx, GDY_ERR_UNSUPPORTED, "integer: stride too large");
  std::vector<Range> ranges;
  ranges.push_back({matrix_range(g.offsets, 1, groups + 1, 0, 1, 0, 4), false, 0});
  ranges.push_back({matrix_range(g.row_scales, 1, g.rows, 0, 1, 0, 4), false, 0});
  ranges.push_back({matrix_range(g.col_scales, 1, g.n, 0, groups, many ? g.stride_col_scales : 0, 4), false, 0});
  ranges.push_back({matrix_range(g.c, g.rows, g.n, g.ldc, 1, 0, os), true, 1});
  if (g.k > 0) {
    if (!g.a || !g.b) return fail(ctx, GDY_ERR_INVALID_ARG, "integer: null A or B");
    if (g.lda < g.k || g.ldb < (g.trans_b ? g.k : g.n))
      return fail(ctx, GDY_ERR_INVALID_ARG, "integer: lda or ldb too small");
    if (many && g.stride_b < 0) return fail(ctx, GDY_ERR_INVALID_ARG, "integer: negative stride_b");
    const int64_t br = g.trans_b ? g.n : g.k, bc = g.trans_b ? g.k : g.n;
    if (!stored_extent(tile_rows, g.k, g.lda, 1, &bytes) || !stored_extent(br, bc, g.ldb, 1, &bytes))
      return fail(ctx, GDY_ERR_UNSUPPORTED, "integer: A or B extent too large");
    ranges.push_back({matrix_range(g.a, g.rows, g.k, g.lda, 1, 0, 1), false, 0});
    ranges.push_back({matrix_range(g.b, br, bc, g.ldb, groups, many ? g.stride_b : 0, 1), false, 0});
  }
  if (ep) {
    const EpiTarget t = {"integer", 0, g.c, g.rows, g.n, g.ldc, -1, 1, groups, g.c_type, 1};
    const gdy_status s = validate_epilogue(ctx, *ep, t, &ranges);
    if (s != GDY_OK) return s;
  }
  return check_ranges(ctx, ranges);
}

// What a tile of such a product costs, in us: start + step for each 128 bytes of K where it has a CU to itself, share +
// share_step where tiles fill the CUs.  Fitted to 244 products of 16 to 4096 rows, N = 1024 to 8192, K = 512 to 8192 and 1,
// 8 and 32 groups (any: 132 of odd sizes), silu and a bias: their choices take 1.7% (any: 1.6%) more than the fastest
// tile of each on average, 34% (21%) at most; the fp8 products' rule took 7% and 38%.
struct IntegerTileCost {
  int tile, bm, bn;
  bool copies;  // both operands take copies
  double start, step, share, share_step;  // share 0: a CU holds one at a time
};
const IntegerTileCost kIntegerTiles[] = {
    {INT_256, 256, 256, true, 13.36, 1.169, 0, 0},
    {INT_64x128, 64, 128, true, 5.85, 0.430, 3.63, 0.319},
    {INT_64, 64, 64, true, 4.91, 0.303, 2.56, 0.219},
    {INT_32x64, 32, 64, true, 4.72, 0.230, 1.43, 0.163},
    {INT_FEW, 16, 16, true, 4.98, 0.096, 1.65, 0.096},
    {INT_ANY_128, 128, 128, false, 8.89, 1.161, 7.74, 0.810},
    {INT_ANY_64x128, 64, 128, false, 6.87, 0.797, 5.46, 0.587},
    {INT_ANY_32x128, 32, 128, false, 5.63, 0.601, 3.95, 0.452},
    {INT_ANY_32x64, 32, 64, false, 4.91, 0.439, 2.63, 0.325}};

// Groups' sizes are unknown here: their row tiles as group_rows_tile counts them.
const IntegerTileCost& integer_tile_of(const gdy_ctx* ctx, const gdy_integer& g, bool copies) {
  const double cus = ctx->cus, groups = g.offsets ? (double)std::min<int64_t>(g.groups, g.rows) : 1.0;
  const double avg = (double)g.rows / groups, steps = std::ceil((double)g.k / 128);
  const IntegerTileCost* best = nullptr;
  double best_t = 0;
  for (const IntegerTileCost& c : kIntegerTiles) {
    if (c.copies != copies || (c.tile == INT_FEW && !g.trans_b)) continue;
    auto tiles = [&](int bm) {  // a CU's
      const double rows = groups <= 1 ? std::ceil((double)g.rows / bm) : groups / (1.0 - std::exp(-bm / avg));
      return rows * (double)((g.n + c.bn - 1) / c.bn) / cus;
    };
    const double n = tiles(c.bm), alone = c.start + c.step * steps;
    double t;
    if (c.share > 0) {
      t = std::max(alone, std::ceil(n - 0.01) * (c.share + c.share_step * steps));
    } else {  // integer_tile_256's order: whole tiles, then those of 128 rows on the CUs that are free
      const double rest = 2 * n - tiles(128), whole = n - rest, full = std::floor(whole), last = whole - full;
      const double behind = rest - (1.0 - last);  // that start when the last whole ones end
      t = alone * (full + (last == 0                ? 0.65 * std::ceil(rest)
                           : 2 * last + rest <= 1.0 ? 0.65
                           : behind <= 0            ? 1.0
                           : behind <= 1.0 - last   ? 1.3
                                                    : 1.0 + 0.65 * std::ceil(behind)));
    }
    if (!best || t < best_t) best = &c, best_t = t;
  }
  return *best;
}

// Whether a valid product computes a tile at all, and which.
bool integer_has_tiles(const gdy_integer& g) { return (!g.offsets || g.groups > 0) && g.rows > 0 && g.n > 0; }
bool integer_a_copies(const gdy_integer& g) { return copies_ok(g.a, g.lda, g.k, 1, true, 0); }
bool integer_b_copies(const gdy_integer& g) {
  return copies_ok(g.b, g.ldb, g.k, 1, g.trans_b != 0, g.offsets && g.groups > 1 ? g.stride_b : 0);
}

gdy_status launch_integer(gdy_ctx* ctx, const gdy_integer& g, const gdy_epilogue* ep, hipStream_t hs) {
  if (!integer_has_tiles(g)) return GDY_OK;
  const bool grouped = g.offsets != nullptr;
  const int groups = grouped ? g.groups : 1;
  const int os = g.c_type == GDY_F32 ? 4 : 2;
  const bool many = groups > 1;
  KInteger q;
  std::memset(&q, 0, sizeof q);
  q.row_scales = g.row_scales;
  q.col_scales = g.col_scales;
  q.stride_col_scales = many ? g.stride_col_scales : 0;
  KGroup& a = q.g;
  a.a = (const uint8_t*)g.a;
  a.b = (const uint8_t*)g.b;
  a.c = (uint8_t*)g.c;
  a.offsets = g.offsets;
  a.stride_b = many ? g.stride_b : 0;
  a.rows = a.m = (int32_t)g.rows;
  a.groups = groups;
  a.n = (int32_t)g.n;
  a.k = (int32_t)g.k;
  a.lda = (int32_t)g.lda;
  a.ldb = (int32_t)g.ldb;
  a.ldc = (int32_t)g.ldc;
  a.scale = 1.0f;
  auto vec = [&](const void* p, int64_t ld) { return (uintptr_t)p % 8 == 0 && (ld * os) % 8 == 0; };
  a.c_vec = vec(g.c, g.ldc);
  a.a_dma = integer_a_copies(g);
  a.b_dma = integer_b_copies(g);
  a.xcd_cus = std::max(ctx->cus / kXcds, 1);
  if (ep) {
    a.epi.bias = (const uint8_t*)ep->bias;
    a.epi.bias_f32 = ep->bias && ep->bias_type == GDY_F32;
    a.epi.stride_bias = many ? ep->stride_bias * (a.epi.bias_f32 ? 4 : os) : 0;
    a.epi.res = (const uint8_t*)ep->residual;
    a.epi.ldr = (int32_t)ep->ldr;
    a.epi.res_vec = vec(ep->residual, ep->ldr);
    a.epi.act = ep->act;
  }
  const IntegerTileCost& tile = integer_tile_of(ctx, g, a.a_dma && a.b_dma);
  const GroupKernel kern = g.c_type == GDY_BF16  ? integer_bf16(g.trans_b, tile.tile)
                           : g.c_type == GDY_F16 ? integer_f16(g.trans_b, tile.tile)
                                                 : integer_f32(g.trans_b, tile.tile);
  a.bm = tile.bm;
  a.max_slots = (int32_t)(grouped ? max_row_tiles(g.rows, groups, a.bm) : (g.rows + a.bm - 1) / a.bm);
  const int64_t tn = (g.n + kern.bn - 1) / kern.bn;
  // of an XCD: the last tiles' other halves, and its short tiles are rounded up by themselves
  const int64_t halves = a.bm == 256 ? a.xcd_cus / 2 + 1 : 0;
  const int64_t grid = (((int64_t)a.max_slots * tn + kXcds - 1) / kXcds + halves) * kXcds;
  if (grid * kern.threads > UINT32_MAX)  // threads of a launch
    return fail(ctx, GDY_ERR_UNSUPPORTED, "integer: a grid of %lld workgroups", (long long)grid);
  void* argv[] = {&q};
  HIP_TRY(ctx, hipExtLaunchKernel(kern.func, dim3((unsigned)grid), dim3(kern.threads), argv, 0, hs, nullptr, nullptr, 0));
  return GDY_OK;
}

}  // namespace
