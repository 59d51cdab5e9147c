"""Products of 8-bit integers with scales against 64-bit references: every type of C, layout and
tile, ragged and empty groups, rows of no group, odd sizes and alignments, epilogues,
the largest sums, streams, graphs, and 8-bit experts behind the operators that feed them."""
import os

import pytest

import paper_2409_02227_amd  # noqa: F401  (sets GPU_MAX_HW_QUEUES before HIP starts)

torch = pytest.importorskip("torch")

from paper_2409_02227_amd import gdy  # noqa: E402
from tests.operator_refs import ACTS, EPS32, Expected, close, padded, untouched  # noqa: E402
from tests.test_gpu_experts import reference, routed  # noqa: E402

pytestmark = pytest.mark.gpu
TABLE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                     "paper_2409_02227_amd", "tables", "gfx950.table")
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    c = gdy.Context(0, table=TABLE)
    yield c
    c.close()


def codes(gen, rows, cols, pad=0, shift=0, items=0):
    """int8 values over their whole range, rows `pad` longer, `shift` bytes into the buffer."""
    shape = ((items,) if items else ()) + (rows, cols + pad)
    count = 1
    for v in shape:
        count *= v
    whole = torch.randint(-128, 128, (count + shift + 16,), generator=gen, dtype=torch.int8).cuda()
    return whole[shift:shift + count].view(shape)[..., :cols]


class Product:
    """offsets None: dense."""

    def __init__(self, dtype, rows, offsets, n, k, tb=0, act="none", bias=None, residual=False, scales="both", pad=0, shift=0,
                 shared_b=False, inplace=False, seed=0):
        self.label = (dtype, rows, None if offsets is None else tuple(offsets[:8]), n, k, tb, act, bias, residual, scales, pad,
                      shift, inplace)
        print(self.label, flush=True)
        gen = torch.Generator().manual_seed(seed + 3 * rows + n + 7 * k)
        t = TYPES[dtype]
        groups = 0 if offsets is None else len(offsets) - 1
        self.dtype, self.t, self.rows, self.n, self.k, self.tb, self.act, self.groups = dtype, t, rows, n, k, tb, act, groups
        self.a = codes(gen, rows, k, pad, shift)
        b = codes(gen, *((n, k) if tb else (k, n)), pad, shift, 1 if shared_b else groups)
        self.b = b.expand(groups, -1, -1) if shared_b else b
        # sums of k products of deviation 73.9^2
        size = 1.0 / (5461.0 * max(k, 1) ** 0.5)
        self.rs = (torch.rand(rows, generator=gen) + 0.5).cuda() if scales in ("both", "rows") else None
        lead = (groups,) if groups and bias != "shared" else ()
        self.cs = ((torch.rand(lead + (n,), generator=gen) + 0.5) * size).cuda() if scales in ("both", "cols") else None
        if scales == "rows":
            self.rs *= size
        self.bias = None
        if bias:
            self.bias = torch.randn(lead + (n,), generator=gen).to(torch.float32 if bias == "f32" else t).cuda()
        self.c, self.c_full = padded(rows, n, t, pad)
        self.res = None
        if residual:
            self.res = torch.randn((rows, n), generator=gen).to(t).cuda()
            if inplace:
                self.c.copy_(self.res)
                self.res = self.c
        self.res64 = None if self.res is None else self.res.double().cpu()
        self.offsets = None if offsets is None else torch.tensor(offsets, dtype=torch.int32).cuda()
        self.bounds = [(0, rows)]
        if offsets is not None:
            self.bounds = []
            for lo, hi in zip(offsets[:-1], offsets[1:]):
                lo = min(max(lo, 0), rows)
                self.bounds.append((lo, min(max(hi, lo), rows)))
        self.inplace = inplace
        ep = gdy.Epilogue(self.bias, act, self.res)
        self.product = gdy.Int8(self.a, self.b, self.c, self.rs, self.cs, self.offsets, tb, ep)

    def check(self):
        covered = torch.zeros(self.rows, dtype=torch.bool)
        named = torch.zeros(self.rows, dtype=torch.int64)
        for lo, hi in self.bounds:
            named[lo:hi] += 1
        off = torch.ones((self.rows, self.n), dtype=torch.bool)  # values of rows of several groups that are none of theirs
        for e, (lo, hi) in enumerate(self.bounds):
            if lo == hi:
                continue
            covered[lo:hi] = True
            b = (self.b[e] if self.groups else self.b).double().cpu()
            z = self.a[lo:hi].double().cpu() @ (b.t() if self.tb else b)  # whole numbers below 2^53
            if self.rs is not None:
                z = z * self.rs[lo:hi].double().cpu()[:, None]
            if self.cs is not None:
                z = z * (self.cs[e] if self.cs.dim() == 2 else self.cs).double().cpu()
            # the sum as a float, two products and the bias: a rounding each
            size = z.abs()
            if self.bias is not None:
                bias = (self.bias[e] if self.bias.dim() == 2 else self.bias).double().cpu()
                z, size = z + bias, size + bias.abs()
            x = Expected(z, 4 * EPS32 * size, self.t, self.act, None if self.res64 is None else self.res64[lo:hi])
            once = named[lo:hi] == 1
            close(self.c[lo:hi][once.cuda()], x.c[once], x.c_bound[once], (e,) + self.label)
            off[lo:hi] &= ~((self.c[lo:hi].double().cpu() - x.c).abs() <= x.c_bound)
        # decreasing offsets give rows to two groups: each value is one of the two's
        assert not off[named > 1].any(), ("rows of several groups", self.label)
        if not self.inplace:
            assert torch.isnan(self.c.float().cpu()[~covered]).all(), ("rows of no group", self.label)
        untouched(self.c, self.c_full, self.label)


def run(ctx, x, **kw):
    ctx.execute_int8(x.product, **kw)
    torch.cuda.synchronize()
    x.check()


DENSE = [(1, 64, 128), (1, 2048, 2048), (3, 17, 33), (16, 130, 4096), (17, 65, 130), (64, 256, 1000), (129, 128, 128),
         (200, 300, 77), (257, 513, 256), (509, 2047, 1021), (512, 1024, 2048), (1, 1, 1), (300, 1, 64), (5, 100, 16384)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,n,k", DENSE)
@pytest.mark.parametrize("tb", [0, 1])
def test_dense(ctx, dtype, rows, n, k, tb):
    run(ctx, Product(dtype, rows, None, n, k, tb))
    q = rows + n
    run(ctx, Product(dtype, rows, None, n, k, tb, ACTS[q % 5], ("own", "f32")[q % 2], q % 3 != 0, ("both", "rows", "cols")[q % 3],
                     (0, 16, 3)[q % 3], (0, 0, 1)[q % 3]))


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("tb", [0, 1])
def test_dense_large_tiles(ctx, dtype, tb):
    """Tiles of 256 x 256, whole and of 128 rows, in both ends (with a residual and without)."""
    for rows, n, k in ((2048, 2304, 256), (4000, 4100, 128), (8192, 256, 384), (1408, 4096, 144)):
        run(ctx, Product(dtype, rows, None, n, k, tb, bias="own"))
        run(ctx, Product(dtype, rows, None, n, k, tb, "gelu", "own", True, inplace=True))


SPLITS = [(1, [0, 1]), (5, [0, 0, 2, 2, 5, 5]), (40, [3, 20, 20, 33]), (200, [0, 16, 33, 97, 161, 200]),
          (700, [0, 128, 257, 300, 620]), (1100, [10, 266, 267, 700, 1100]), (3, [0, 0, 0, 0]), (90, [-5, 30, 20, 1000])]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,offsets", SPLITS)
@pytest.mark.parametrize("tb", [0, 1])
def test_grouped(ctx, dtype, rows, offsets, tb):
    for q, (n, k) in enumerate(((264, 256), (65, 130), (130, 77), (96, 4096))):
        run(ctx, Product(dtype, rows, offsets, n, k, tb, ACTS[(q + rows) % 5], ("own", "shared", None, "f32")[q], q == 1,
                         ("both", "both", "rows", "cols")[q], (0, 3, 0, 16)[q], (0, 1, 0, 0)[q], shared_b=q == 3))


@pytest.mark.parametrize("tb", [0, 1])
def test_grouped_many_rows(ctx, tb):
    """Large tiles, last waves as halves, groups of every size."""
    for rows, groups, n, k in ((8192, 16, 1024, 256), (5000, 60, 512, 128), (3000, 3, 2048, 160)):
        gen = torch.Generator().manual_seed(rows)
        cuts = sorted(torch.randint(0, rows + 1, (groups - 1,), generator=gen).tolist())
        run(ctx, Product("bf16", rows, [0] + cuts + [rows - 7 if cuts[-1] < rows - 7 else rows], n, k, tb, "silu", "own"))


def test_largest_sums(ctx):
    """k = 131071 products of -128 * -128 stay below 2^31, and of 127 * -128 above -2^31; a float's rounding of them."""
    k = 131071
    a = torch.full((17, k), -128, dtype=torch.int8, device="cuda")
    for value in (-128, 127):
        b = torch.full((65, k), value, dtype=torch.int8, device="cuda")
        for rows in (1, 17):
            c = torch.zeros(rows, 65, device="cuda")
            ctx.execute_int8(gdy.Int8(a[:rows], b, c, trans_b=1))
            torch.cuda.synchronize()
            assert (c == float(torch.tensor(-128 * value * k, dtype=torch.float32))).all(), (value, rows)
        c = torch.zeros(17, 65, device="cuda")
        ctx.execute_int8(gdy.Int8(a, b.t().contiguous(), c))
        torch.cuda.synchronize()
        assert (c == float(torch.tensor(-128 * value * k, dtype=torch.float32))).all()


def test_sums_are_exact(ctx):
    """Sums of whole numbers below 2^24 come out as they are, on every tile, whatever their order."""
    gen = torch.Generator().manual_seed(2)
    for rows, n, k in ((1, 64, 1000), (16, 96, 1024), (48, 64, 1000), (60, 300, 512), (300, 300, 900), (2100, 2100, 512)):
        for tb in (0, 1):
            a, b = codes(gen, rows, k), codes(gen, *((n, k) if tb else (k, n)))
            c = torch.zeros(rows, n, device="cuda")
            ctx.execute_int8(gdy.Int8(a, b, c, trans_b=tb))
            torch.cuda.synchronize()
            want = a.double() @ (b.t() if tb else b).double()
            assert torch.equal(c.double(), want), (rows, n, k, tb)


def test_nothing_to_do(ctx):
    """No k: the bias; no rows, columns or groups: nothing; all offsets behind the rows."""
    c = torch.full((5, 8), 7.0, device="cuda")
    e8 = lambda *s: torch.zeros(s, dtype=torch.int8, device="cuda")  # noqa: E731
    bias = torch.randn(8, device="cuda")
    for tb in (0, 1):
        ctx.execute_int8(gdy.Int8(e8(5, 0), e8(8, 0) if tb else e8(0, 8), c, trans_b=tb, epilogue=gdy.Epilogue(bias)))
        torch.cuda.synchronize()
        assert torch.equal(c, bias.expand(5, 8))
        c.fill_(7.0)
    off = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    ctx.execute_int8(gdy.Int8(e8(5, 16), e8(0, 16, 8), c, offsets=off(0)))
    ctx.execute_int8(gdy.Int8(e8(5, 16), e8(2, 16, 8), c, offsets=off(9, 9, 9)))
    ctx.execute_int8(gdy.Int8(e8(5, 16), e8(2, 16, 8), c, offsets=off(4, 3, 2)))
    ctx.execute_int8(gdy.Int8(e8(0, 16), e8(16, 8), c[:0]))
    ctx.execute_int8(gdy.Int8(e8(5, 16), e8(16, 0), c[:, :0]))
    torch.cuda.synchronize()
    assert (c == 7.0).all()


def test_scales_that_are_no_numbers(ctx):
    """A row whose scale is infinite or NaN is NaN where its sums are 0 (a quantised row without numbers), the
    others as ever."""
    gen = torch.Generator().manual_seed(4)
    a, b = codes(gen, 20, 64), codes(gen, 40, 64)
    a[3], a[18] = 0, 0
    rs = torch.ones(20, device="cuda")
    rs[3], rs[18] = float("inf"), float("nan")
    c = torch.zeros(20, 40, device="cuda")
    ctx.execute_int8(gdy.Int8(a, b, c, rs, trans_b=1))
    torch.cuda.synchronize()
    want = a.double() @ b.double().t()
    bad = torch.zeros(20, dtype=torch.bool)
    bad[3] = bad[18] = True
    assert torch.isnan(c[bad.cuda()]).all() and torch.equal(c[~bad.cuda()].double(), want[~bad.cuda()])


def test_rows_past_two_gib(ctx):
    """A and C end past 2^31 and 2^32 bytes; the last rows are right."""
    rows, k, n = 1 << 20, 4096, 1024  # A 4 GiB, C (fp32) 4 GiB
    a = torch.zeros((rows, k), dtype=torch.int8, device="cuda")
    gen = torch.Generator().manual_seed(6)
    some = [0, (1 << 19) - 1, 1 << 19, rows - 1]
    a[some] = codes(gen, 4, k)
    b = codes(gen, n, k)
    c = torch.full((rows, n), 3.0, device="cuda")
    ctx.execute_int8(gdy.Int8(a, b, c, trans_b=1))
    torch.cuda.synchronize()
    want = a[some].double() @ b.double().t()
    close(c[some], want.cpu(), 2 * EPS32 * want.abs().cpu(), "rows past 2 GiB")
    assert int(torch.count_nonzero(c)) == int(torch.count_nonzero(c[some]))


class Experts:
    """8-bit experts: route, quantise to the experts' rows, two products, combine."""

    def __init__(self, ctx, tokens, top_k, experts, n, hidden, seed=0):
        gen = torch.Generator().manual_seed(seed)
        self.ctx = ctx
        self.ids = torch.randint(-1, experts, (tokens, top_k), generator=gen).cuda()
        self.x = torch.randn((tokens, n), generator=gen).to(torch.bfloat16).cuda()
        self.w = torch.rand((tokens, top_k), generator=gen).cuda()
        self.w1, self.w2 = codes(gen, hidden, n, items=experts), codes(gen, n, hidden, items=experts)
        self.s1 = ((torch.rand((experts, hidden), generator=gen) + 0.5) / (74 * n ** 0.5)).cuda()
        self.s2 = ((torch.rand((experts, n), generator=gen) + 0.5) / (74 * hidden ** 0.5)).cuda()
        rows = tokens * top_k
        z = lambda *s, t=torch.bfloat16: torch.zeros(s, dtype=t, device="cuda")  # noqa: E731
        self.slots, self.offsets = z(tokens, top_k, t=torch.int32), z(experts + 1, t=torch.int32)
        self.q1, self.r1 = z(rows, n, t=torch.int8), z(rows, t=torch.float32)
        self.h, self.q2, self.r2 = z(rows, hidden), z(rows, hidden, t=torch.int8), z(rows, t=torch.float32)
        self.o, self.y = z(rows, n), z(tokens, n)

    def run(self, stream=None):
        c, kw = self.ctx, {"stream": stream}
        c.execute_route(gdy.Route(self.ids, self.slots, self.offsets), **kw)
        c.execute_quantize(gdy.Quantize(self.x, self.q1, self.r1, self.slots), **kw)
        c.execute_int8(gdy.Int8(self.q1, self.w1, self.h, self.r1, self.s1, self.offsets, 1, gdy.Epilogue(act="silu")), **kw)
        c.execute_quantize(gdy.Quantize(self.h, self.q2, self.r2), **kw)
        c.execute_int8(gdy.Int8(self.q2, self.w2, self.o, self.r2, self.s2, self.offsets, 1), **kw)
        c.execute_combine(gdy.Combine(self.o, self.slots, self.y, self.w, self.x), **kw)

    def reference(self):
        """In 64 bits, with the roundings that the formulas have: codes of both activations, bf16 of the first's rows."""
        q, s = reference(self.x)
        x = q.double() * s[:, None]
        y = self.x.double().cpu()
        ids = self.ids.cpu()
        for i, j in (ids >= 0).nonzero().tolist():
            e = int(ids[i, j])
            h = torch.nn.functional.silu((x[i] @ self.w1[e].double().cpu().t()) * self.s1[e].double().cpu())
            q2, s2 = reference(h.to(torch.bfloat16)[None])
            o = (q2[0].double() * s2[0]) @ self.w2[e].double().cpu().t() * self.s2[e].double().cpu()
            y[i] += float(self.w[i, j]) * o
        return y


def test_8bit_experts(ctx):
    """The rows between the products are bf16: a value next to a rounding may come out a step (2^-8) to the side and
    a code with it, and the second product's rows and y are rounded to bf16: below 3 * 2^-8 in the 2-norm."""
    for tokens, top_k, experts, n, hidden in ((21, 2, 5, 128, 256), (150, 3, 8, 80, 112)):
        x = Experts(ctx, tokens, top_k, experts, n, hidden, tokens)
        x.run()
        torch.cuda.synchronize()
        slots, offsets = routed(x.ids, experts)
        assert torch.equal(x.slots.cpu(), slots) and torch.equal(x.offsets.cpu(), offsets)
        ref = x.reference()
        off = float((x.y.double().cpu() - ref).norm() / ref.norm())
        print(off, flush=True)
        assert off < 3 * 2.0 ** -8


def test_8bit_experts_in_a_graph(ctx):
    x = Experts(ctx, 300, 2, 6, 128, 192, 1)
    side = torch.cuda.Stream()
    x.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        x.run(side)
    torch.cuda.synchronize()
    for rep in range(3):
        x.ids.copy_(x.ids.roll(1 + rep, 0))
        x.x.add_(0.25)
        torch.cuda.synchronize()
        x.run()
        torch.cuda.synchronize()
        want = x.y.clone()
        x.y.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(x.y, want), rep
    del graph
    torch.cuda.synchronize()


# products that between them run on all tiles, for operands that take copies and for others
TILES = [(20, 512, 144), (100, 16390, 144), (200, 8200, 130), (250, 8200, 300), (300, 16390, 144), (200, 16400, 144),
         (700, 2050, 150), (500, 8208, 144), (20, 16400, 144)]


@pytest.mark.parametrize("tb", [0, 1])
@pytest.mark.parametrize("pad", [16, 3])
def test_every_tile(ctx, tb, pad):
    """Each tile dense, in ragged groups, with and without a residual; both sides of a K tile."""
    found = set()
    for rows, n, k in TILES:
        n += (-n) % 16 if pad == 16 else 0
        k += (-k) % 16 if pad == 16 else 0
        for offsets in (None, [0, rows // 2 - 3, rows // 2 - 3, rows - 5]):
            for residual in (False, True):
                x = Product("bf16", rows, offsets, n, k, tb, "gelu" if residual else "none", "own", residual, pad=pad)
                run(ctx, x)
                found.add(ctx.int8_tile(x.product))
    few = Product("f16", 3, None, 200, 4096, tb, pad=pad)  # B stored N x K
    run(ctx, few)
    found.add(ctx.int8_tile(few.product))
    if pad == 16:
        assert found == {(256, 256), (64, 128), (64, 64), (32, 64)} | ({(16, 16)} if tb else set()), found
    else:
        assert found == {(128, 128), (64, 128), (32, 128), (32, 64)}, found


@pytest.mark.parametrize("tb", [0, 1])
def test_short_tiles_behind_whole_ones(ctx, tb):
    """Groups' ends of one row to a whole tile, in more groups than a wave's lanes; each way that the last tiles run."""
    ends = [1, 127, 128, 129, 255, 256, 257, 383, 384, 385, 0, 640]
    for groups, n, scale in ((100, 608, 1), (9, 2064, 1), (70, 1008, 1), (13, 1040, 3)):
        counts = [scale * ends[(7 * e) % len(ends)] for e in range(groups)]
        offsets = [3]
        for c in counts:
            offsets.append(offsets[-1] + c)
        x = Product("bf16", offsets[-1] + 5, offsets, n, 128, tb, "relu", "own", groups == 9, pad=16)
        assert ctx.int8_tile(x.product) == (256, 256)
        run(ctx, x)


def test_groups_past_four_gib(ctx):
    """The B of groups 2^31 bytes apart."""
    groups, n, k = 4, 96, 64
    gen = torch.Generator().manual_seed(9)
    whole = torch.zeros(3 * 2 ** 31 + n * k, dtype=torch.int8, device="cuda")
    b = whole.as_strided((groups, n, k), (2 ** 31, k, 1))
    b.copy_(codes(gen, n, k, items=groups))
    a = codes(gen, 40, k)
    c = torch.zeros(40, n, device="cuda")
    ctx.execute_int8(gdy.Int8(a, b, c, offsets=torch.arange(0, 41, 10, dtype=torch.int32).cuda(), trans_b=1))
    torch.cuda.synchronize()
    for e in range(groups):
        want = a[10 * e:10 * e + 10].double() @ b[e].double().t()
        assert torch.equal(c[10 * e:10 * e + 10].double(), want), e


@pytest.mark.parametrize("tb", [0, 1])
def test_no_k_on_large_tiles(ctx, tb):
    """The bias and the residual alone, dense and by group; A and B have no addresses."""
    bias, res = torch.randn(2304, device="cuda"), torch.randn((2100, 2304), device="cuda")
    for groups in (0, 3):
        a = torch.zeros((2100, 0), dtype=torch.int8, device="cuda")
        b = torch.zeros(((groups,) if groups else ()) + ((2304, 0) if tb else (0, 2304)), dtype=torch.int8, device="cuda")
        c = torch.zeros((2100, 2304), device="cuda")
        offsets = torch.tensor([0, 700, 700, 2100], dtype=torch.int32).cuda() if groups else None
        for residual in (None, res):
            ctx.execute_int8(gdy.Int8(a, b, c, offsets=offsets, trans_b=tb, epilogue=gdy.Epilogue(bias, "none", residual)))
            torch.cuda.synchronize()
            assert (c == bias + (0 if residual is None else residual)).all(), (groups, residual is None)


def bounds_of_many(groups, rows, kind):
    """Offsets of more groups than a wave has lanes.  spread: rows all over, empty groups on both sides of the first
    64; behind: no rows in the first 64; across: rows in the first and last group of each 64 alone; back: as
    spread, with an offset past the first 64 that decreases."""
    gen = torch.Generator().manual_seed(groups + rows)
    if kind == "behind":
        ends = [2] * 65 + sorted(torch.randint(2, rows, (groups - 65,), generator=gen).tolist())
        return ends + [rows - 1]
    if kind == "across":
        own = [e for e in range(groups) if e % 64 in (0, 63)]
        ends, at = [1], 1
        for e in range(groups):
            at = min(at + (1 + (rows - 4) // len(own) if e in own else 0), rows - 1)
            ends.append(at)
        return ends
    inner = torch.randint(3, rows - 2, (groups - 1,), generator=gen)
    ends = [3] + sorted(inner.tolist()) + [rows - 2]
    ends[63] = ends[62]  # group 62 is empty, and 64 where it is not the last
    if groups > 65:
        ends[65] = ends[64]
    if kind == "back":
        ends[groups - 1] = ends[groups - 2] - min(5, ends[groups - 2])
    return ends


MANY = [  # groups, rows, n, k, and the tiles of operands that take copies (B stored K x N, N x K) and of others
    (65, 100, 80, 144, (32, 64), (16, 16), (32, 64)), (130, 100, 64, 1024, (32, 64), (16, 16), (32, 64)),
    (130, 300, 256, 512, (32, 64), (32, 64), (32, 128)), (257, 300, 256, 512, (64, 128), (64, 128), (32, 128)),
    (65, 3000, 2064, 80, (64, 128), (64, 128), (64, 128)), (257, 100, 80, 144, (32, 64), (16, 16), (32, 64))]


@pytest.mark.parametrize("groups,rows,n,k,nn,nt,others", MANY)
@pytest.mark.parametrize("kind", ["spread", "behind", "across", "back"])
@pytest.mark.parametrize("tb", [0, 1])
def test_small_tiles_of_many_groups(ctx, groups, rows, n, k, nn, nt, others, kind, tb):
    """More groups than a wave reads at a time, each with few rows, on the tiles that such products take."""
    offsets = bounds_of_many(groups, rows, kind)
    assert len(offsets) == groups + 1 and (kind == "back") == (offsets != sorted(offsets))
    for pad, tile in ((0, nt if tb else nn), (3, others)):
        x = Product("bf16", rows, offsets, n, k, tb, "silu" if pad else "none", "own", kind == "spread", pad=pad)
        assert ctx.int8_tile(x.product) == tile
        run(ctx, x)
