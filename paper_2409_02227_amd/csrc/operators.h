// operators.h -- host side of epilogues, grouped products and activation
// gradients: checks, tile choice, launches.  Part of gdy.cpp.
#pragma once

namespace {

// ---------------------------------------------------------------------------
// Checks
// ---------------------------------------------------------------------------
// A memory range of a call.  Outputs may overlap nothing but what they may be
// themselves (`twin` names it: the same tag).
struct Range {
  Extent x;
  bool out;
  int twin;  // ranges of one nonzero twin may coincide
};

// Values of a member's bias_grad, all items together: the work items of a launch of
// kMaxFused members' sums, at most one a value, are a 31-bit count.
const int64_t kMaxBiasGrad = (int64_t)1 << 26;

gdy_status check_ranges(gdy_ctx* ctx, const std::vector<Range>& r) {
  for (size_t i = 0; i < r.size(); ++i) {
    if (!r[i].out) continue;
    for (size_t j = 0; j < r.size(); ++j)
      if (i != j && overlap(r[i].x, r[j].x) && !(r[i].twin && r[i].twin == r[j].twin))
        return fail(ctx, GDY_ERR_ALIAS, "an output overlaps another operand or output");
  }
  return GDY_OK;
}

// What an epilogue is checked against: C, its type and batch (or groups).
struct EpiTarget {
  const char* what;
  int index;
  const void* c;
  int64_t m, n, ldc, stride_c, items;  // items of C, R and aux
  int64_t biases;                      // of bias and bias_grad
  int32_t c_type;
  int twin;                            // tag of C and of what may be C itself
};

// The fields of an epilogue, and its ranges appended to `ranges`.
gdy_status validate_epilogue(gdy_ctx* ctx, const gdy_epilogue& e, const EpiTarget& t, std::vector<Range>* ranges) {
  const int os = t.c_type == GDY_F32 ? 4 : 2;
  if (e.act < GDY_ACT_NONE || e.act > GDY_ACT_SILU)
    return fail(ctx, GDY_ERR_INVALID_ARG, "%s %d: unknown activation %d", t.what, t.index, e.act);
  if ((e.grad != 0 && e.grad != 1) || e.reserved != 0)
    return fail(ctx, GDY_ERR_INVALID_ARG, "%s %d: grad must be 0 or 1, reserved 0", t.what, t.index);
  if (e.bias && e.bias_type != t.c_type && e.bias_type != GDY_F32)
    return fail(ctx, GDY_ERR_UNSUPPORTED, "%s %d: bias type %d, C's %d", t.what, t.index, e.bias_type, t.c_type);
  if (t.n == 0 || (t.m == 0 && !e.bias_grad)) return GDY_OK;
  const bool reads_aux = e.grad && e.act != GDY_ACT_NONE;
  if (reads_aux && !e.aux && t.m > 0)
    return fail(ctx, GDY_ERR_INVALID_ARG, "%s %d: a backward activation needs aux", t.what, t.index);
  const bool many = t.items > 1, groups = t.biases > 1;
  if ((e.bias && (uintptr_t)e.bias % (e.bias_type == GDY_F32 ? 4 : os)) || (uintptr_t)e.residual % os ||
      (uintptr_t)e.aux % os || (uintptr_t)e.bias_grad % 4)
    return fail(ctx, GDY_ERR_UNSUPPORTED, "%s %d: epilogue operands not element aligned", t.what, t.index);
  if ((e.residual && e.ldr < t.n) || (e.aux && e.ldaux < t.n))
    return fail(ctx, GDY_ERR_INVALID_ARG, "%s %d: ldr or ldaux < n", t.what, t.index);
  if ((many && ((e.residual && e.stride_r < 0) || (e.aux && e.stride_aux < 0))) ||
      (groups && ((e.bias && e.stride_bias < 0) || (e.bias_grad && e.stride_bias_grad < 0))))
    return fail(ctx, GDY_ERR_INVALID_ARG, "%s %d: negative epilogue stride", t.what, t.index);
  if (groups && e.bias_grad && e.stride_bias_grad != 0 && e.stride_bias_grad < t.n)
    return fail(ctx, GDY_ERR_ALIAS, "%s %d: items of bias_grad overlap", t.what, t.index);
  if ((many && ((e.residual && e.stride_r > kMaxStride) || (e.aux && e.stride_aux > kMaxStride))) ||
      (groups && ((e.bias && e.stride_bias > kMaxStride) || (e.bias_grad && e.stride_bias_grad > kMaxStride))))
    return fail(ctx, GDY_ERR_UNSUPPORTED, "%s %d: epilogue stride too large", t.what, t.index);
  if (e.bias_grad && t.n > kMaxBiasGrad / (groups && e.stride_bias_grad ? t.biases : 1))
    return fail(ctx, GDY_ERR_UNSUPPORTED, "%s %d: bias_grad of more than %lld values", t.what, t.index,
                (long long)kMaxBiasGrad);
  // 32-bit byte offsets up to 256 rows past the edge, within an item (grouped rows: a tile)
  const int64_t tile_rows = std::min<int64_t>(t.m, t.stride_c < 0 ? 256 : t.m);
  int64_t bytes;
  if ((e.residual && !stored_extent(tile_rows, t.n, e.ldr, os, &bytes)) ||
      (e.aux && !stored_extent(tile_rows, t.n, e.ldaux, os, &bytes)))
    return fail(ctx, GDY_ERR_UNSUPPORTED, "%s %d: residual or aux extent too large", t.what, t.index);
  const bool writes_aux = e.aux && !e.grad;
  if (writes_aux && many && e.stride_aux < (t.m - 1) * e.ldaux + t.n)
    return fail(ctx, GDY_ERR_ALIAS, "%s %d: batch items of aux overlap", t.what, t.index);
  auto is_c = [&](const void* p, int64_t ld, int64_t stride) {
    return p == t.c && ld == t.ldc && (!many || stride == t.stride_c);
  };
  const int bs = e.bias_type == GDY_F32 ? 4 : os;
  ranges->push_back({matrix_range(e.bias, 1, t.n, t.n, groups ? t.biases : 1, e.stride_bias, bs), false, 0});
  ranges->push_back({matrix_range(e.residual, t.m, t.n, e.ldr, t.items, many ? e.stride_r : 0, os), false,
                     is_c(e.residual, e.ldr, e.stride_r) ? t.twin : 0});
  if (writes_aux || reads_aux)
    ranges->push_back({matrix_range(e.aux, t.m, t.n, e.ldaux, t.items, many ? e.stride_aux : 0, os), writes_aux,
                       reads_aux && is_c(e.aux, e.ldaux, e.stride_aux) ? t.twin : 0});
  ranges->push_back({matrix_range(e.bias_grad, 1, t.n, t.n, groups ? t.biases : 1, e.stride_bias_grad, 4), true, 0});
  return GDY_OK;
}

// The epilogues of a submission that validate() has accepted.
gdy_status validate_epilogues(gdy_ctx* ctx, const gdy_gemm* g, const gdy_epilogue* ep, int n) {
  std::vector<Range> ranges;
  bool any = false;
  for (int i = 0; i < n; ++i) {
    if (g[i].op == GDY_OP_ADD) {
      if (has_epilogue(ep[i]) || ep[i].grad)
        return fail(ctx, GDY_ERR_INVALID_ARG, "add %d: an add takes no epilogue", i);
    } else {
      any = any || has_epilogue(ep[i]);
      const int64_t items = std::max(g[i].batch, 1);
      const EpiTarget t = {"gemm", i, g[i].c, g[i].m, g[i].n, g[i].ldc, g[i].batch > 1 ? g[i].stride_c : 0,
                           items, items, g[i].c_type, i + 1};
      const gdy_status s = validate_epilogue(ctx, ep[i], t, &ranges);
      if (s != GDY_OK) return s;
    }
  }
  if (!any) return GDY_OK;
  for (int i = 0; i < n; ++i) {  // the members' own operands and outputs, which validate() compared
    Extent ea, eb, ec;
    validate_one(ctx, g[i], i, &ea, &eb, &ec);
    ranges.push_back({ea, false, 0});
    ranges.push_back({eb, false, 0});
    ranges.push_back({ec, true, i + 1});
  }
  return check_ranges(ctx, ranges);
}

// ---------------------------------------------------------------------------
// Bias gradients
// ---------------------------------------------------------------------------
void add_bias_sum(BiasSums* s, const float* part, float* out, int n, int rows, int items, int64_t stride) {
  const int u = s->count++;
  if (u == 0) s->many = 0;
  s->part[u] = part;
  s->out[u] = out;
  s->stride[u] = stride;
  s->n[u] = n;
  s->rows[u] = rows;
  s->first[u] = items;  // ranges are made at the launch
  if (rows >= kSumManyRows) s->many = 1;
}

hipError_t launch_bias_sums(BiasSums* s, hipStream_t hs, hipEvent_t stop) {
  if (s->count == 0) return hipSuccess;
  const int cols = sum_cols(s->many != 0);
  int wg = 0;
  for (int u = 0; u < s->count; ++u) {
    const int items = s->first[u];
    s->first[u] = wg;
    wg += items * ((s->n[u] + cols - 1) / cols);
  }
  s->first[s->count] = wg;
  const int threads = sum_threads(s->many != 0);
  const int grid = (int)std::min<int64_t>(wg, UINT32_MAX / threads);
  void* argv[] = {s};
  return hipExtLaunchKernel(bias_sum_kernel(s->many != 0), dim3(grid), dim3(threads), argv, 0, hs, nullptr, stop, 0);
}

hipError_t launch_group_sums(const GroupSums& s, hipStream_t hs) {
  const bool many = (int64_t)s.max_slots * s.per / (s.shared ? 1 : std::max(s.groups, 1)) >= kSumManyRows;
  const int64_t blocks = (s.n + sum_cols(many) - 1) / sum_cols(many);
  void* argv[] = {(void*)&s};
  return hipExtLaunchKernel(group_sum_kernel(many), dim3((unsigned)(blocks * (s.shared ? 1 : s.groups))),
                            dim3(sum_threads(many)), argv, 0, hs, nullptr, nullptr, 0);
}

// Zeros to the bias gradients of members without rows, which no launch computes.
gdy_status zero_bias_grads(gdy_ctx* ctx, const gdy_gemm* g, const gdy_epilogue* ep, int n, hipStream_t hs) {
  BiasSums s;
  s.count = 0;
  for (int i = 0; i < n; ++i) {
    if (g[i].op != GDY_OP_GEMM || active(g[i]) || g[i].n == 0 || !ep[i].bias_grad) continue;
    const bool many = g[i].batch > 1 && ep[i].stride_bias_grad != 0;
    add_bias_sum(&s, nullptr, ep[i].bias_grad, (int)g[i].n, 0, many ? g[i].batch : 1, ep[i].stride_bias_grad);
    if (s.count == kMaxFused) {
      HIP_TRY(ctx, launch_bias_sums(&s, hs, nullptr));
      s.count = 0;
    }
  }
  HIP_TRY(ctx, launch_bias_sums(&s, hs, nullptr));
  return GDY_OK;
}

// ---------------------------------------------------------------------------
// Grouped products
// ---------------------------------------------------------------------------
gdy_status validate_grouped(gdy_ctx* ctx, const gdy_grouped& g, const gdy_epilogue* ep) {
  if (g.over != GDY_OVER_ROWS && g.over != GDY_OVER_K)
    return fail(ctx, GDY_ERR_INVALID_ARG, "grouped: unknown form %d", g.over);
  const bool over_k = g.over == GDY_OVER_K;
  if (g.groups < 0 || g.rows < 0 || g.n < 0 || g.k < 0)
    return fail(ctx, GDY_ERR_INVALID_ARG, "grouped: negative size");
  if (g.groups > GDY_MAX_GROUPS)
    return fail(ctx, GDY_ERR_TOO_MANY, "grouped: %d groups > %d", g.groups, GDY_MAX_GROUPS);
  const bool t16 = (g.a_type == GDY_F16 || g.a_type == GDY_BF16) && g.b_type == g.a_type && g.c_type == g.a_type;
  const bool t8 = g.a_type == GDY_FP8_E4M3 && g.b_type == GDY_FP8_E4M3 && g.c_type == GDY_BF16;
  const bool t32 = g.a_type == GDY_F32 && g.b_type == GDY_F32 && g.c_type == GDY_F32;
  if (!t16 && !t8 && !t32)
    return fail(ctx, GDY_ERR_UNSUPPORTED, "grouped: unsupported dtype triple (%d,%d,%d)", g.a_type, g.b_type, g.c_type);
  if ((g.trans_b != 0 && g.trans_b != 1) || (over_k && g.trans_b))
    return fail(ctx, GDY_ERR_INVALID_ARG, "grouped: bad trans_b");
  if (!std::isfinite(g.scale_a) || !std::isfinite(g.scale_b) ||
      (!t8 && (g.scale_a != 1.0f || g.scale_b != 1.0f || g.scales)))
    return fail(ctx, GDY_ERR_INVALID_ARG, "grouped: scales must be finite, and 1 for 16- and 32-bit inputs");
  if (over_k && ep && (ep->act != GDY_ACT_NONE || ep->grad || ep->bias || ep->aux || ep->bias_grad))
    return fail(ctx, GDY_ERR_UNSUPPORTED, "grouped: over K the epilogue may hold a residual only");
  const int es = elem_size(g.a_type), os = g.c_type == GDY_F32 ? 4 : 2;
  const int64_t m = over_k ? g.k : g.rows;  // rows of C (of a group's, over K)
  if (g.groups == 0 || g.n == 0 || (m == 0 && !(ep && ep->bias_grad))) return GDY_OK;
  // sizes are 32-bit on the device, row tiles and their columns one 31-bit count
  if (g.rows > INT32_MAX - 4096 || g.n > INT32_MAX - 4096 || g.k > INT32_MAX - 4096 ||
      ((g.rows + 15) / 16 + g.groups) * ((g.n + 63) / 64) > INT32_MAX / 2 ||
      (over_k && ((g.k + 63) / 64 + 8) * ((g.n + 63) / 64 + 8) > INT32_MAX / 2 / g.groups))
    return fail(ctx, GDY_ERR_UNSUPPORTED, "grouped: sizes too large");
  if (!g.offsets || (uintptr_t)g.offsets % 4 || (uintptr_t)g.scales % 4)
    return fail(ctx, GDY_ERR_INVALID_ARG, "grouped: null or unaligned offsets or scales");
  if (g.groups > 1 && (over_k ? g.stride_c : g.stride_b) > kMaxStride)
    return fail(ctx, GDY_ERR_UNSUPPORTED, "grouped: stride too large");
  std::vector<Range> ranges;
  ranges.push_back({matrix_range(g.offsets, 1, g.groups + 1, 0, 1, 0, 4), false, 0});
  ranges.push_back({matrix_range(g.scales, 1, g.groups, 0, 1, 0, 4), false, 0});
  int64_t bytes;
  if (m > 0) {
    if (!g.c) return fail(ctx, GDY_ERR_INVALID_ARG, "grouped: null C");
    if (g.ldc < g.n) return fail(ctx, GDY_ERR_INVALID_ARG, "grouped: ldc < n");
    if ((uintptr_t)g.c % os) return fail(ctx, GDY_ERR_UNSUPPORTED, "grouped: C not element aligned");
    if (!stored_extent(std::min<int64_t>(m, 256), g.n, g.ldc, os, &bytes))
      return fail(ctx, GDY_ERR_UNSUPPORTED, "grouped: rows of C too long");
    if (over_k && g.groups > 1 && g.stride_c < (g.k - 1) * g.ldc + g.n)
      return fail(ctx, GDY_ERR_ALIAS, "grouped: groups of C overlap (stride_c too small)");
    ranges.push_back({matrix_range(g.c, m, g.n, g.ldc, over_k ? g.groups : 1, over_k ? g.stride_c : 0, os), true, 1});
    if (over_k ? g.rows > 0 : g.k > 0) {
      if (!g.a || !g.b) return fail(ctx, GDY_ERR_INVALID_ARG, "grouped: null A or B");
      if (((uintptr_t)g.a | (uintptr_t)g.b) % es) return fail(ctx, GDY_ERR_UNSUPPORTED, "grouped: A or B not element aligned");
      if (g.lda < g.k || g.ldb < (g.trans_b ? g.k : g.n))
        return fail(ctx, GDY_ERR_INVALID_ARG, "grouped: lda or ldb too small");
      bool ok;
      if (over_k) {  // a group may hold every row
        ok = stored_extent(g.rows, g.k, g.lda, es, &bytes) && stored_extent(g.rows, g.n, g.ldb, es, &bytes);
        ranges.push_back({matrix_range(g.b, g.rows, g.n, g.ldb, 1, 0, es), false, 0});
      } else {
        if (g.groups > 1 && g.stride_b < 0) return fail(ctx, GDY_ERR_INVALID_ARG, "grouped: negative stride_b");
        ok = stored_extent(std::min<int64_t>(g.rows, 256), g.k, g.lda, es, &bytes) &&
             (g.trans_b ? stored_extent(g.n, g.k, g.ldb, es, &bytes) : stored_extent(g.k, g.n, g.ldb, es, &bytes));
        ranges.push_back({matrix_range(g.b, g.trans_b ? g.n : g.k, g.trans_b ? g.k : g.n, g.ldb, g.groups, g.stride_b, es),
                          false, 0});
      }
      if (!ok) return fail(ctx, GDY_ERR_UNSUPPORTED, "grouped: A or B extent too large");
      ranges.push_back({matrix_range(g.a, g.rows, g.k, g.lda, 1, 0, es), false, 0});
    }
  }
  if (ep) {
    const EpiTarget t = {"grouped", 0, g.c, m, g.n, g.ldc, over_k ? g.stride_c : -1, over_k ? g.groups : 1,
                         g.groups, g.c_type, 1};
    const gdy_status s = validate_epilogue(ctx, *ep, t, &ranges);
    if (s != GDY_OK) return s;
  }
  return check_ranges(ctx, ranges);
}

// The most tiles of bm rows that `rows` rows in `groups` groups make: q groups with
// rows make at most (rows - q) / bm + q.
int64_t max_row_tiles(int64_t rows, int64_t groups, int bm) {
  const int64_t q = std::min(rows, groups);
  return (rows - q) / bm + q;
}

GroupKernel group_kernel_of(int dtype, int over_k, int tb, int tile) {
  return dtype == DT_BF16 ? group_bf16(over_k, tb, tile) : dtype == DT_F16 ? group_f16(over_k, tb, tile)
         : dtype == DT_FP8 ? group_fp8(over_k, tb, tile) : group_f32(over_k, tb, tile);
}

// What a tile of a grouped product over rows costs, in times of a 256 x 256 tile's
// step of K (fp32: of as many multiply-adds): `share` of a CU where tiles fill the
// GPU, `item` from its start to its end, `waves` where a CU holds one at a time.
// Measured at K = 2048 and 4096 in bf16, 8 to 128 groups of 64 to 8192 rows in all:
// 8192 rows in 16 groups x 4096 took 170, 198, 196, 228, 325 and 370 us on these
// tiles, 512 rows in 4 groups x 1024 83, 59, 47, 32, 26 and 26.
struct GroupTileCost {
  int tile, bm, bn;
  double share, item;
  bool waves;
};
const GroupTileCost kGroupTiles[] = {
    {0, 256, 256, 1.0, 1.0, true},     {0, 128, 256, 0.65, 0.65, true},   {1, 128, 128, 0.32, 0.57, false},
    {2, 64, 128, 0.21, 0.38, false},   {3, 32, 128, 0.145, 0.31, false},  {4, 32, 64, 0.08, 0.30, false}};
const GroupTileCost kGroupTilesF32[] = {
    {1, 128, 128, 0.25, 0.27, false},  {2, 64, 128, 0.13, 0.15, false},   {3, 32, 128, 0.07, 0.09, false},
    {4, 32, 64, 0.037, 0.06, false}};

// The kernel and tile rows of a product over rows.  The groups' sizes are unknown
// here: as exponentially distributed, E groups of T rows make E / (1 - exp(-bm E /
// T)) tiles of bm rows (E where groups are small, T / bm + E / 2 where they are
// large; the 83 tiles of 60 groups of 8192 rows by a power law, bm = 256, count as 71).
const GroupTileCost& group_rows_tile(const gdy_ctx* ctx, const gdy_grouped& g, bool copies) {
  const bool f32 = g.a_type == GDY_F32;
  const GroupTileCost* list = f32 ? kGroupTilesF32 : kGroupTiles;
  const int n = f32 ? (int)(sizeof kGroupTilesF32 / sizeof *list) : (int)(sizeof kGroupTiles / sizeof *list);
  const double cus = ctx->cus, groups = (double)std::min<int64_t>(g.groups, g.rows), avg = (double)g.rows / groups;
  const GroupTileCost* best = nullptr;
  double best_t = 0;
  for (int i = 0; i < n; ++i) {
    const GroupTileCost& c = list[i];
    if (c.tile == 0 && !copies) continue;
    const double rows = groups <= 1 ? std::ceil((double)g.rows / c.bm) : groups / (1.0 - std::exp(-c.bm / avg));
    const double tiles = rows * (double)((g.n + c.bn - 1) / c.bn);
    double t;
    if (c.waves) {  // a last wave of up to half the CUs runs as halves of 256-row tiles
      const double full = std::floor(tiles / cus), rest = tiles / cus - full;
      t = full * c.item + (rest == 0 ? 0.0 : c.bm == 256 && rest <= 0.5 ? 0.65 : c.item);
    }
    else t = tiles * c.share <= cus * c.item ? c.item : tiles * c.share / cus + 0.5 * c.item;
    if (!best || t < best_t) best = &c, best_t = t;
  }
  return *best;
}

// Whether a product over rows runs in tiles of 16 rows with K over a workgroup's waves
// (skinny.h).  Few workgroups wait for one K tile after another (32 x 64 tiles: 0.22 to 0.42 us
// each); these take a round of loads, 2 to 4 KiB of a row, in 2.5 us as the compiler has it,
// several waits for memory (skinny.h; K x N of 16-bit types, which waits for all loads two or
// three times a step, 3.6, and 1.3 TB/s of weights in place of 4), but read a group's B once for 16 rows, from L2 at 8 TB/s.  us, 32 x 64 tiles and these: bf16 nt
// 65 rows, 768 x 4096 20.7 and 11.0; 2 rows of 128 groups, 4096 x 4096 21.2 and 10.3; 64
// rows, 4096 x 4096 20.7 and 32.2; nn 2 rows of 16 groups, 72 x 4096 20.8 and 12.2, a row,
// 4096 x 14336 62.4 and 88.5; fp32 nn 65 rows, 768 x 4096 58.8 and 29.3; fp8 nt 64 rows in
// 16 groups, 2048 x 2048 13.2 and 21.2, 16 rows in 4, 256 x 16384 34.6 and 14.5.
bool group_rows_few(const gdy_grouped& g, bool copies) {
  if (!copies || g.k == 0 || !group_few(g.a_type, g.trans_b).func) return false;
  const int es = elem_size(g.a_type);
  const bool narrow = es == 2 && !g.trans_b;
  const double groups = (double)std::min<int64_t>(g.groups, g.rows), avg = (double)g.rows / groups;
  const double slots = groups <= 1 ? std::ceil((double)g.rows / kSkinnyRows)
                                   : groups / (1.0 - std::exp(-kSkinnyRows / avg));  // as group_rows_tile
  const double kbytes = (double)g.k * es, cols = skinny_cols(g.trans_b);
  const double read = slots * std::ceil(g.n / cols) * (cols + std::min<double>(kSkinnyRows, g.rows / slots)) * kbytes;
  const double rounds = std::ceil(kbytes / (8.0 * skinny_kstep(es) * skinny_ahead(es, g.trans_b)));
  const double weights = groups * g.n * kbytes;
  double few = std::max(rounds * (narrow ? 3.6 : 2.5), read / 8e6);
  double tiles = std::ceil(kbytes / 128) * (es == 4 ? 0.42 : es == 2 ? 0.25 : 0.22);
  if (narrow) few = std::max(few, weights / 1.3e6), tiles = std::max(tiles, weights / 4e6);
  return few < tiles;
}

// The kernel of a product over K: 256 x 256 tiles where they give most CUs one, 128 x 128
// ones where every CU has more than one.  us on 256, 128 and 64 (bf16, 8192 rows, tiles of 256): 16
// groups of 512 x 1024, 128 tiles, 25.2, 19.9 and 25.5; 32 groups, 256 tiles, 22.6, 24.7 and
// 33.2; one group of 4096 x 2048, 157, 138 and 286, 4096 x 4096 197, 272 and 624; 4 groups, 4096
// rows, 512 x 512, 16 tiles, 30.5, 19.2 and 10.6, 1024 x 1024, 64 tiles, 31.5, 22.0 and 20.8; fp32 8
// groups, 4096 rows, 2048 x 1024, 256 tiles, 148 on 128 and 166 on 64.
int group_k_tile(const gdy_ctx* ctx, const gdy_grouped& g, bool copies) {
  auto tiles = [&](int64_t b) { return (g.k + b - 1) / b * ((g.n + b - 1) / b) * g.groups; };
  if (copies && g.a_type != GDY_F32 && 4 * tiles(256) >= 3 * ctx->cus) return 0;
  return tiles(128) > ctx->cus ? 1 : 2;
}

// Whether both operands of a product take copies, its kernel and the rows of a tile.
struct GroupChoice {
  bool a_copies, b_copies;
  GroupKernel kern;
  int bm;
};
GroupChoice choose_group_kernel(const gdy_ctx* ctx, const gdy_grouped& g) {
  const bool over_k = g.over == GDY_OVER_K;
  const int es = elem_size(g.a_type);
  GroupChoice c;
  c.a_copies = copies_ok(g.a, g.lda, g.k, es, !over_k, 0);
  c.b_copies = copies_ok(g.b, g.ldb, g.k, es, !over_k && g.trans_b, over_k || g.groups == 1 ? 0 : g.stride_b);
  const bool copies = c.a_copies && c.b_copies;
  if (over_k) {
    c.kern = group_kernel_of(g.a_type, 1, 0, group_k_tile(ctx, g, copies));
    c.bm = c.kern.bm;
  } else if (group_rows_few(g, copies)) {
    c.kern = group_few(g.a_type, g.trans_b);
    c.bm = c.kern.bm;
  } else {
    const GroupTileCost& tile = group_rows_tile(ctx, g, copies);
    c.kern = group_kernel_of(g.a_type, 0, g.trans_b, tile.tile);
    c.bm = tile.bm;
  }
  return c;
}

// Whether a valid product computes a tile at all.
bool group_has_tiles(const gdy_grouped& g) {
  return g.groups > 0 && g.n > 0 && (g.over == GDY_OVER_K ? g.k : g.rows) > 0;
}

gdy_status launch_grouped(gdy_ctx* ctx, const gdy_grouped& g, const gdy_epilogue* ep, hipStream_t hs) {
  const bool over_k = g.over == GDY_OVER_K;
  const int es = elem_size(g.a_type), os = g.c_type == GDY_F32 ? 4 : 2;
  const int64_t m = over_k ? g.k : g.rows;
  float* bias_grad = ep ? ep->bias_grad : nullptr;
  const bool shared = g.groups > 1 && ep && ep->stride_bias_grad == 0;
  if (!group_has_tiles(g)) {
    if (g.groups == 0 || g.n == 0 || !bias_grad) return GDY_OK;
    // no rows: zero sums
    BiasSums s;
    s.count = 0;
    add_bias_sum(&s, nullptr, bias_grad, (int)g.n, 0, shared ? 1 : g.groups, ep->stride_bias_grad);
    HIP_TRY(ctx, launch_bias_sums(&s, hs, nullptr));
    return GDY_OK;
  }
  KGroup a;
  std::memset(&a, 0, sizeof a);
  a.a = (const uint8_t*)g.a;
  a.b = (const uint8_t*)g.b;
  a.c = (uint8_t*)g.c;
  a.offsets = g.offsets;
  a.scales = g.scales;
  a.stride_b = over_k || g.groups == 1 ? 0 : g.stride_b * es;
  a.stride_c = over_k && g.groups > 1 ? g.stride_c * os : 0;
  a.rows = (int32_t)g.rows;
  a.groups = g.groups;
  a.m = (int32_t)m;
  a.n = (int32_t)g.n;
  a.k = (int32_t)g.k;
  a.lda = (int32_t)g.lda;
  a.ldb = (int32_t)g.ldb;
  a.ldc = (int32_t)g.ldc;
  a.scale = g.scale_a * g.scale_b;
  auto vec = [&](const void* p, int64_t ld, int64_t stride) {
    return (uintptr_t)p % 8 == 0 && (ld * os) % 8 == 0 && (!over_k || g.groups == 1 || (stride * os) % 8 == 0);
  };
  a.c_vec = vec(g.c, g.ldc, g.stride_c);
  const GroupChoice choice = choose_group_kernel(ctx, g);
  const GroupKernel& kern = choice.kern;
  a.a_dma = choice.a_copies;
  a.b_dma = choice.b_copies;
  a.bm = choice.bm;
  a.max_slots = (int32_t)max_row_tiles(g.rows, g.groups, a.bm);
  a.xcd_cus = std::max(ctx->cus / kXcds, 1);
  const int sums_per_tile = !over_k && a.bm == 256 ? 2 : 1;
  if (ep) {
    a.epi.bias = (const uint8_t*)ep->bias;
    a.epi.bias_f32 = ep->bias && ep->bias_type == GDY_F32;
    a.epi.stride_bias = g.groups > 1 ? ep->stride_bias * (a.epi.bias_f32 ? 4 : os) : 0;
    a.epi.res = (const uint8_t*)ep->residual;
    a.epi.ldr = (int32_t)ep->ldr;
    a.epi.stride_res = over_k && g.groups > 1 ? ep->stride_r * os : 0;
    a.epi.res_vec = vec(ep->residual, ep->ldr, ep->stride_r);
    a.epi.aux = ep->grad && ep->act == GDY_ACT_NONE ? nullptr : (uint8_t*)ep->aux;
    a.epi.ldaux = (int32_t)ep->ldaux;
    a.epi.aux_vec = vec(ep->aux, ep->ldaux, 0);
    a.epi.act = ep->act;
    a.epi.grad = ep->grad;
  }
  if (bias_grad) {
    const int64_t need = (int64_t)a.max_slots * sums_per_tile * g.n * 4;
    if (need > kSplitWsBytes)
      return fail(ctx, GDY_ERR_UNSUPPORTED, "grouped: bias_grad needs %lld bytes of workspace, %lld are there",
                  (long long)need, (long long)kSplitWsBytes);
    a.epi.part = ctx->split_ws;
  }
  const int64_t tn = (g.n + kern.bn - 1) / kern.bn;
  const int64_t grid = over_k ? (m + kern.bm - 1) / kern.bm * tn * g.groups
                              : (((int64_t)a.max_slots * tn + kXcds - 1) / kXcds + a.xcd_cus / 2) * kXcds;
  if (grid * kern.threads > UINT32_MAX)  // threads of a launch
    return fail(ctx, GDY_ERR_UNSUPPORTED, "grouped: a grid of %lld workgroups", (long long)grid);
  void* argv[] = {&a};
  HIP_TRY(ctx, hipExtLaunchKernel(kern.func, dim3((unsigned)grid), dim3(kern.threads), argv, 0, hs, nullptr, nullptr, 0));
  if (bias_grad) {
    GroupSums s = {ctx->split_ws, bias_grad, g.offsets, ep->stride_bias_grad, a.n, a.rows, a.groups, a.bm,
                   a.max_slots, shared ? 1 : 0, sums_per_tile};
    HIP_TRY(ctx, launch_group_sums(s, hs));
  }
  return GDY_OK;
}

// ---------------------------------------------------------------------------
// Activation gradients
// ---------------------------------------------------------------------------
gdy_status validate_act_grad(gdy_ctx* ctx, const gdy_act_grad& g) {
  if (g.rows < 0 || g.n < 0 || g.groups < 0) return fail(ctx, GDY_ERR_INVALID_ARG, "act_grad: negative size");
  if (g.groups > GDY_MAX_GROUPS)
    return fail(ctx, GDY_ERR_TOO_MANY, "act_grad: %d groups > %d", g.groups, GDY_MAX_GROUPS);
  if (g.type != GDY_F16 && g.type != GDY_BF16 && g.type != GDY_F32)
    return fail(ctx, GDY_ERR_UNSUPPORTED, "act_grad: unsupported type %d", g.type);
  if (g.act < GDY_ACT_NONE || g.act > GDY_ACT_SILU || g.reserved != 0)
    return fail(ctx, GDY_ERR_INVALID_ARG, "act_grad: unknown activation %d, or reserved not 0", g.act);
  if (!g.dz && !g.bias_grad) return fail(ctx, GDY_ERR_INVALID_ARG, "act_grad: neither dz nor bias_grad");
  if (g.n == 0 || (g.offsets && g.groups == 0)) return GDY_OK;
  const int es = elem_size(g.type);
  const bool reads_z = g.act != GDY_ACT_NONE;
  if ((uintptr_t)g.offsets % 4 || (uintptr_t)g.bias_grad % 4 || (uintptr_t)g.dy % es || (uintptr_t)g.dz % es ||
      (reads_z && (uintptr_t)g.z % es))
    return fail(ctx, GDY_ERR_UNSUPPORTED, "act_grad: operands not element aligned");
  const int64_t groups = g.offsets ? g.groups : 1;
  if (g.bias_grad && groups > 1 && g.stride_bias_grad != 0 && g.stride_bias_grad < g.n)
    return fail(ctx, g.stride_bias_grad < 0 ? GDY_ERR_INVALID_ARG : GDY_ERR_ALIAS, "act_grad: bad stride_bias_grad");
  if (g.bias_grad && groups > 1 && g.stride_bias_grad > kMaxStride)
    return fail(ctx, GDY_ERR_UNSUPPORTED, "act_grad: stride_bias_grad too large");
  if (g.bias_grad && g.n > kMaxBiasGrad / (groups > 1 && g.stride_bias_grad ? groups : 1))
    return fail(ctx, GDY_ERR_UNSUPPORTED, "act_grad: bias_grad of more than %lld values", (long long)kMaxBiasGrad);
  if (g.rows > INT32_MAX - 4096 || g.n > INT32_MAX - 4096 ||
      ((g.rows + 15) / 16 + groups) * ((g.n + kActCols - 1) / kActCols) > INT32_MAX / 2)
    return fail(ctx, GDY_ERR_UNSUPPORTED, "act_grad: sizes too large");
  std::vector<Range> ranges;
  ranges.push_back({matrix_range(g.offsets, 1, groups + 1, 0, 1, 0, 4), false, 0});
  ranges.push_back({matrix_range(g.bias_grad, 1, g.n, g.n, groups, groups > 1 ? g.stride_bias_grad : 0, 4), true, 0});
  if (g.rows > 0) {
    if (!g.dy || (reads_z && !g.z)) return fail(ctx, GDY_ERR_INVALID_ARG, "act_grad: null dy or z");
    if (g.lddy < g.n || (reads_z && g.ldz < g.n) || (g.dz && g.lddz < g.n))
      return fail(ctx, GDY_ERR_INVALID_ARG, "act_grad: leading dimension < n");
    int64_t bytes;
    const int64_t tile = std::min<int64_t>(g.rows, 256);
    if (!stored_extent(tile, g.n, g.lddy, es, &bytes) || (reads_z && !stored_extent(tile, g.n, g.ldz, es, &bytes)) ||
        (g.dz && !stored_extent(tile, g.n, g.lddz, es, &bytes)))
      return fail(ctx, GDY_ERR_UNSUPPORTED, "act_grad: rows too long");
    const int dz = 1;
    ranges.push_back({matrix_range(g.dz, g.rows, g.n, g.lddz, 1, 0, es), true, dz});
    ranges.push_back({matrix_range(g.dy, g.rows, g.n, g.lddy, 1, 0, es), false,
                      g.dy == g.dz && g.lddy == g.lddz ? dz : 0});
    if (reads_z)
      ranges.push_back({matrix_range(g.z, g.rows, g.n, g.ldz, 1, 0, es), false, g.z == g.dz && g.ldz == g.lddz ? dz : 0});
  }
  return check_ranges(ctx, ranges);
}

gdy_status launch_act_grad(gdy_ctx* ctx, const gdy_act_grad& g, hipStream_t hs) {
  const int os = elem_size(g.type);
  const int groups = g.offsets ? g.groups : 1;
  if (g.n == 0 || groups == 0) return GDY_OK;
  const bool shared = groups > 1 && g.stride_bias_grad == 0;
  if (g.rows == 0) {
    if (!g.bias_grad) return GDY_OK;
    BiasSums s;
    s.count = 0;
    add_bias_sum(&s, nullptr, g.bias_grad, (int)g.n, 0, shared ? 1 : groups, g.stride_bias_grad);
    HIP_TRY(ctx, launch_bias_sums(&s, hs, nullptr));
    return GDY_OK;
  }
  KActGrad a;
  std::memset(&a, 0, sizeof a);
  const bool reads_z = g.act != GDY_ACT_NONE;
  auto vec = [&](const void* p, int64_t ld) { return (uintptr_t)p % 8 == 0 && (ld * os) % 8 == 0; };
  a.dy = (const uint8_t*)g.dy;
  a.z = reads_z ? (const uint8_t*)g.z : nullptr;
  a.dz = (uint8_t*)g.dz;
  a.offsets = g.offsets;
  a.rows = (int32_t)g.rows;
  a.groups = groups;
  a.n = (int32_t)g.n;
  a.lddy = (int32_t)g.lddy;
  a.ldz = (int32_t)g.ldz;
  a.lddz = (int32_t)g.lddz;
  a.act = g.act;
  a.dy_vec = vec(g.dy, g.lddy);
  a.z_vec = vec(g.z, g.ldz);
  a.dz_vec = vec(g.dz, g.lddz);
  const int64_t tn = (g.n + kActCols - 1) / kActCols;
  auto slots = [&](int bm) { return g.offsets ? max_row_tiles(g.rows, groups, bm) : (g.rows + bm - 1) / bm; };
  a.bm = kActRows;
  a.max_slots = (int32_t)slots(a.bm);
  if (g.bias_grad) {
    const int64_t need = (int64_t)a.max_slots * g.n * 4;
    if (need > kSplitWsBytes)
      return fail(ctx, GDY_ERR_UNSUPPORTED, "act_grad: bias_grad needs %lld bytes of workspace, %lld are there",
                  (long long)need, (long long)kSplitWsBytes);
    // one row tile: its sums are the bias gradient
    a.part = !g.offsets && a.max_slots == 1 ? g.bias_grad : ctx->split_ws;
  }
  if ((int64_t)a.max_slots * tn * kActThreads > UINT32_MAX)
    return fail(ctx, GDY_ERR_UNSUPPORTED, "act_grad: a grid of %lld workgroups", (long long)(a.max_slots * tn));
  void* argv[] = {&a};
  HIP_TRY(ctx, hipExtLaunchKernel(act_grad_kernel(g.type), dim3((unsigned)(a.max_slots * tn)), dim3(kActThreads), argv, 0, hs,
                                  nullptr, nullptr, 0));
  if (!g.bias_grad || a.part == g.bias_grad) return GDY_OK;
  if (!g.offsets) {
    BiasSums s;
    s.count = 0;
    add_bias_sum(&s, a.part, g.bias_grad, a.n, a.max_slots, 1, 0);
    HIP_TRY(ctx, launch_bias_sums(&s, hs, nullptr));
  } else {
    GroupSums s = {a.part, g.bias_grad, g.offsets, g.stride_bias_grad, a.n, a.rows, groups, a.bm, a.max_slots,
                   shared ? 1 : 0, 1};
    HIP_TRY(ctx, launch_group_sums(s, hs));
  }
  return GDY_OK;
}

}  // namespace
