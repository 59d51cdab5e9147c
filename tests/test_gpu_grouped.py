"""Products grouped by expert and activation gradients against 64-bit references:
every type, form and tile, ragged and empty groups, rows of no group, odd sizes,
offsets outside the rows, streams, graphs, and an expert layer's training step."""
import os

import pytest

import paper_2409_02227_amd  # noqa: F401  (sets GPU_MAX_HW_QUEUES before HIP starts)

torch = pytest.importorskip("torch")

from paper_2409_02227_amd import gdy  # noqa: E402
from tests.operator_refs import (ACTS, OUT, Expected, close, operand, padded, product, slope,  # noqa: E402
                                 untouched, value)

pytestmark = pytest.mark.gpu
TABLE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                     "paper_2409_02227_amd", "tables", "gfx950.table")


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    c = gdy.Context(0, table=TABLE)
    yield c
    c.close()


def bounds_of(offsets, rows):
    """The rows of each group, clamped as documented."""
    out = []
    for lo, hi in zip(offsets[:-1], offsets[1:]):
        lo = min(max(lo, 0), rows)
        out.append((lo, min(max(hi, lo), rows)))
    return out


class Rows:
    """A product over rows, operands on the GPU."""

    def __init__(self, dtype, rows, offsets, n, k, tb=0, act="none", grad=False, bias=None, residual=False, aux=False,
                 sums=None, scales=False, pad=0, seed=0, shared_b=False):
        groups = len(offsets) - 1
        self.label = (dtype, rows, tuple(offsets[:8]), groups, n, k, tb, act, grad, bias, residual, aux, sums, pad)
        print(self.label, flush=True)
        self.__dict__.update(dtype=dtype, rows=rows, n=n, k=k, tb=tb, act=act, grad=grad, groups=groups)
        gen = torch.Generator().manual_seed(seed + 3 * rows + n + 7 * k)
        out = OUT[dtype]
        odt = "bf16" if dtype == "fp8" else dtype
        sc = 8.0 if dtype == "fp8" else 1.0
        self.a = operand(gen, rows, k, dtype, pad, 0, sc)
        b = operand(gen, *((n, k) if tb else (k, n)), dtype, pad, 1 if shared_b else groups, sc)
        self.b = b.expand(groups, -1, -1) if shared_b else b
        self.sa, self.sb = (0.25, 0.0625) if dtype == "fp8" else (1.0, 1.0)
        self.scales = (torch.rand(groups, generator=gen) + 0.5).cuda() if scales else None
        self.c, self.c_full = padded(rows, n, out, pad)
        lead = {"groups": (groups,), "shared": ()}.get(bias)
        self.bias = None if bias is None else torch.randn(lead + (n,), generator=gen).to(out).cuda()
        self.res = operand(gen, rows, n, odt, pad) if residual else None
        self.aux = self.aux_full = None
        if grad:
            self.aux = operand(gen, rows, n, odt, pad, 0, 4.0)
        elif aux:
            self.aux, self.aux_full = padded(rows, n, out, pad)
        self.sums = None
        if sums:
            self.sums = torch.full((groups, n) if sums == "groups" else (n,), float("nan"), device="cuda")
        self.offsets = torch.tensor(offsets, dtype=torch.int32).cuda()
        self.bounds = bounds_of(offsets, rows)
        ep = gdy.Epilogue(self.bias, act, self.res, self.aux, grad, self.sums)
        self.product = gdy.Grouped(self.a, self.b, self.c, self.offsets, trans_b=tb, scale_a=self.sa, scale_b=self.sb,
                                   scales=self.scales, epilogue=ep)

    def check(self):
        covered = torch.zeros(self.rows, dtype=torch.bool)
        total = []
        for e, (lo, hi) in enumerate(self.bounds):
            covered[lo:hi] = True
            b = self.b[e].float()
            bias = self.bias if self.bias is None or self.bias.dim() == 1 else self.bias[e]
            scale = self.sa * self.sb * (1.0 if self.scales is None else float(self.scales[e]))
            z, s = product(self.a[lo:hi].float(), b.t() if self.tb else b, scale, bias, self.dtype == "fp8")
            x = Expected(z, s, OUT[self.dtype], self.act, None if self.res is None else self.res[lo:hi],
                         self.aux[lo:hi] if self.grad else None, self.grad)
            close(self.c[lo:hi], x.c, x.c_bound, (e,) + self.label)
            if self.aux_full is not None:
                close(self.aux[lo:hi], x.aux, x.aux_bound, ("aux", e) + self.label)
            total.append(x.sums())
            if self.sums is not None and self.sums.dim() == 2:
                close(self.sums[e], *total[-1], ("sums", e) + self.label)
        if self.sums is not None and self.sums.dim() == 1:
            extra = 2.0 ** -24 * len(total) * sum(r.abs() for r, _ in total)
            close(self.sums, sum(r for r, _ in total), sum(b for _, b in total) + extra, ("sums",) + self.label)
        assert torch.isnan(self.c.float().cpu()[~covered]).all(), ("rows of no group", self.label)
        untouched(self.c, self.c_full, self.label)
        if self.aux_full is not None:
            assert torch.isnan(self.aux.float().cpu()[~covered]).all()
            untouched(self.aux, self.aux_full, self.label)


def run(ctx, x, **kw):
    ctx.execute_grouped(x.product, **kw)
    torch.cuda.synchronize()
    x.check()


# (rows, offsets): one row, an empty group first, last and between, rows of no group in
# front and behind, groups of every tile's height and one more
SPLITS = [(1, [0, 1]), (5, [0, 0, 2, 2, 5, 5]), (40, [3, 20, 20, 33]), (200, [0, 16, 33, 97, 161, 200]),
          (700, [0, 128, 257, 300, 620]), (1100, [10, 266, 267, 700, 1100]), (3, [0, 0, 0, 0])]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "fp8", "f32"])
@pytest.mark.parametrize("rows,offsets", SPLITS)
@pytest.mark.parametrize("tb", [0, 1])
def test_rows(ctx, dtype, rows, offsets, tb):
    for q, (n, k) in enumerate(((264, 256), (65, 130), (130, 77))):
        run(ctx, Rows(dtype, rows, offsets, n, k, tb, ACTS[(q + rows) % 5], bias=("groups", "shared", None)[q],
                      residual=q == 1, aux=q != 2, sums=("groups", "shared", None)[q], scales=dtype == "fp8" and q != 1))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,offsets", SPLITS)
def test_rows_backward(ctx, dtype, rows, offsets):
    for q, (n, k) in enumerate(((128, 512), (67, 33))):
        run(ctx, Rows(dtype, rows, offsets, n, k, 1 - q, ACTS[(q + rows) % 5], grad=True, residual=q == 1,
                      sums="groups"))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "fp8", "f32"])
@pytest.mark.parametrize("rows,offsets,n,k", [(1, [0, 0, 1], 112, 2592), (65, [0, 65], 72, 4096),
                                              (40, [3, 20, 20, 33], 200, 4096), (100, [0, 16, 33, 34, 90], 136, 8192),
                                              (17, [0, 17], 16, 4112), (300, [0, 40, 290, 290, 300], 24, 4096)])
@pytest.mark.parametrize("tb", [0, 1])
def test_rows_of_a_long_k(ctx, dtype, rows, offsets, n, k, tb):
    """Few rows and columns and a long K, on tiles of 16 rows where operands are aligned."""
    q = rows + n + tb
    run(ctx, Rows(dtype, rows, offsets, n, k, tb, ACTS[q % 5], bias="groups", residual=True, aux=True, sums="groups",
                  scales=dtype == "fp8", pad=(0, 16)[tb]))
    run(ctx, Rows(dtype, rows, offsets, n, k, tb, ACTS[(q + 1) % 5], grad=True, sums="shared", seed=1))
    run(ctx, Rows(dtype, rows, offsets, n, k, tb, bias="shared", seed=2))


def test_many_groups(ctx):
    """More groups than a wave has lanes, and the largest number."""
    gen = torch.Generator().manual_seed(5)
    for groups, top in ((64, 9), (65, 9), (200, 40), (1000, 3)):
        sizes = torch.randint(0, top, (groups,), generator=gen).tolist()
        off = [2]
        for s in sizes:
            off.append(off[-1] + s)
        run(ctx, Rows("bf16", off[-1] + 7, off, 72, 64, 1, "silu", bias="groups", sums="groups"))
    run(ctx, Rows("bf16", 50, [0] * 4000 + [20] * 90 + [50] * 7, 16, 16, 0, sums="groups"))


def test_one_large_group_among_small_ones(ctx):
    for dtype in ("bf16", "fp8", "f32"):
        off = [0, 1, 1501, 1501, 1504, 1600]
        run(ctx, Rows(dtype, 1600, off, 384, 256, 0, "gelu_tanh", bias="groups", aux=True, sums="groups"))
        run(ctx, Rows(dtype, 1600, off, 384, 256, 1, "silu"))


@pytest.mark.parametrize("pad", [1, 4, 8])
def test_pitches(ctx, pad):
    for dtype in ("bf16", "fp8", "f32"):
        run(ctx, Rows(dtype, 300, [0, 17, 250, 300], 130, 96, 0, "gelu", bias="groups", residual=True, aux=True,
                      sums="groups", pad=pad))
        run(ctx, Rows(dtype, 300, [0, 17, 250, 300], 130, 100, 1, "silu", grad=True, pad=pad))


def test_shared_weights_and_no_k(ctx):
    run(ctx, Rows("bf16", 300, [0, 100, 290], 200, 128, 0, "silu", shared_b=True))
    run(ctx, Rows("bf16", 300, [0, 100, 290], 200, 0, 0, "silu", bias="groups", sums="groups"))


def test_offsets_outside_the_rows(ctx):
    """Offsets are clamped to the rows: nothing outside the operands is touched."""
    run(ctx, Rows("bf16", 100, [-5, 40, 90, 2000], 130, 64, 0, "silu", bias="groups", sums="groups"))
    run(ctx, Rows("bf16", 100, [2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1], 130, 64, 1, sums="groups"))
    run(ctx, Rows("f32", 600, [-2 ** 31, -7, 0, 599, 601], 130, 64, 1, sums="shared"))


def test_no_rows(ctx):
    x = Rows("bf16", 0, [0, 0, 0], 70, 64, bias="groups", sums="groups")
    ctx.execute_grouped(x.product)
    torch.cuda.synchronize()
    assert torch.count_nonzero(x.sums).item() == 0 and not torch.isnan(x.sums).any()


class OverK:
    def __init__(self, dtype, rows, offsets, k, n, residual=None, pad=0, seed=0, scales=False):
        groups = len(offsets) - 1
        self.label = (dtype, rows, tuple(offsets[:8]), k, n, residual, pad)
        print(self.label, flush=True)
        self.__dict__.update(dtype=dtype, rows=rows, k=k, n=n)
        gen = torch.Generator().manual_seed(seed + rows + n + 7 * k)
        sc = 8.0 if dtype == "fp8" else 1.0
        self.a, self.b = operand(gen, rows, k, dtype, pad, 0, sc), operand(gen, rows, n, dtype, pad, 0, sc)
        self.sa, self.sb = (0.25, 0.0625) if dtype == "fp8" else (1.0, 1.0)
        self.scales = (torch.rand(groups, generator=gen) + 0.5).cuda() if scales else None
        self.c, self.c_full = padded(k, n, OUT[dtype], pad, items=groups)
        self.res = None
        odt = "bf16" if dtype == "fp8" else dtype
        if residual:
            self.res = operand(gen, k, n, odt, pad, groups)
            if residual == "c":
                self.c.copy_(self.res)
        self.offsets = torch.tensor(offsets, dtype=torch.int32).cuda()
        self.bounds = bounds_of(offsets, rows)
        ep = None if not residual else gdy.Epilogue(residual=self.c if residual == "c" else self.res)
        self.product = gdy.Grouped(self.a, self.b, self.c, self.offsets, over="k", scale_a=self.sa, scale_b=self.sb,
                                   scales=self.scales, epilogue=ep)

    def check(self):
        for e, (lo, hi) in enumerate(self.bounds):
            scale = self.sa * self.sb * (1.0 if self.scales is None else float(self.scales[e]))
            z, s = product(self.a[lo:hi].float().t(), self.b[lo:hi].float(), scale, None, self.dtype == "fp8")
            x = Expected(z, s, OUT[self.dtype], residual=None if self.res is None else self.res[e])
            close(self.c[e], x.c, x.c_bound, (e,) + self.label)
        untouched(self.c, self.c_full, self.label)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "fp8", "f32"])
@pytest.mark.parametrize("rows,offsets", SPLITS)
def test_over_k(ctx, dtype, rows, offsets):
    for q, (k, n) in enumerate(((264, 384), (65, 31), (1, 130))):
        run(ctx, OverK(dtype, rows, offsets, k, n, (None, "own", "c")[q], scales=dtype == "fp8"))


def test_over_k_tiles(ctx):
    """Few and many tiles, pitches, offsets outside the rows."""
    run(ctx, OverK("bf16", 700, [0, 300, 300, 690], 2048, 3000, "c"))
    run(ctx, OverK("bf16", 500, [-3, 100, 777], 640, 1280, None))
    run(ctx, OverK("fp8", 700, [0, 300, 300, 690], 1024, 2560))
    for pad in (1, 8):
        run(ctx, OverK("bf16", 130, [0, 1, 64, 130], 96, 200, "own", pad=pad))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,n", [(1, 1), (3, 130), (65, 512), (300, 1001), (2100, 520)])
@pytest.mark.parametrize("act", ACTS)
def test_act_grad(ctx, dtype, rows, n, act):
    gen = torch.Generator().manual_seed(rows + n)
    for pad, offsets, place in ((0, None, None), (1, None, "dy"), (8, [0, 0, rows // 3, rows // 3, rows], "z"),
                                (0, [rows // 4, rows // 2 + 1, rows + 5], None)):
        dy, z = operand(gen, rows, n, dtype, pad), operand(gen, rows, n, dtype, pad, 0, 5.0)
        dy0, z0 = dy.clone(), z.clone()
        dz, full = padded(rows, n, OUT[dtype], pad)
        if place and not (place == "z" and act == "none"):
            dz = {"dy": dy, "z": z}[place]
            full = None
        groups = len(offsets) - 1 if offsets else 0
        sums = torch.full((groups, n) if groups else (n,), float("nan"), device="cuda")
        off = torch.tensor(offsets, dtype=torch.int32).cuda() if offsets else None
        ctx.execute_act_grad(gdy.ActGrad(dy, z, dz, sums, act, off))
        torch.cuda.synchronize()
        v = dy0.double().cpu()
        x = Expected(v, torch.zeros_like(v), OUT[dtype], act, None, z0, True)
        covered = torch.zeros(rows, dtype=torch.bool)
        for e, (lo, hi) in enumerate(bounds_of(offsets, rows) if offsets else [(0, rows)]):
            covered[lo:hi] = True
            close(dz[lo:hi], x.c[lo:hi], x.c_bound[lo:hi], (dtype, rows, n, act, e))
            close(sums[e] if groups else sums, *x.sums(slice(lo, hi)), ("sums", dtype, rows, n, act, e))
        if full is not None:
            assert torch.isnan(dz.float().cpu()[~covered]).all()
            untouched(dz, full, (dtype, rows, n, act))
        else:
            before = dy0 if place == "dy" else z0
            assert torch.equal(dz.cpu()[~covered], before.cpu()[~covered])
        # one output without the other, and sums over all groups
        only = torch.full_like(sums[0] if groups else sums, float("nan"))
        ctx.execute_act_grad(gdy.ActGrad(dy0, z0, None, only, act, off))
        torch.cuda.synchronize()
        close(only, *x.sums(covered), ("all sums", dtype, rows, n, act))
        if act != "none":
            dz2 = torch.full((rows, n), float("nan"), dtype=OUT[dtype], device="cuda")
            ctx.execute_act_grad(gdy.ActGrad(dy0, z0, dz2, None, act, off))
            torch.cuda.synchronize()
            close(dz2[covered.cuda()], x.c[covered], x.c_bound[covered], ("dz", dtype, rows, n, act))


def test_act_grad_infinities(ctx):
    z = torch.tensor([[float("inf"), float("-inf"), 70.0, -70.0, 0.0]] * 2, dtype=torch.float32, device="cuda")
    dy = torch.full_like(z, 3.0)
    for act, at0 in (("relu", 0.0), ("gelu", 1.5), ("gelu_tanh", 1.5), ("silu", 1.5)):
        dz = torch.empty_like(z)
        ctx.execute_act_grad(gdy.ActGrad(dy, z, dz, None, act))
        torch.cuda.synchronize()
        assert torch.allclose(dz[0].cpu(), torch.tensor([3.0, 0.0, 3.0, 0.0, at0]), atol=1e-6, rtol=1e-6), (act, dz[0])


def test_streams_and_graphs(ctx):
    """Another stream than the current one, a captured call replayed beside eager ones,
    with the counts changed between replays."""
    side = torch.cuda.Stream()
    x = Rows("bf16", 300, [0, 17, 17, 250, 290], 264, 256, 0, "silu", bias="groups", aux=True, sums="groups")
    w = OverK("bf16", 300, [0, 17, 17, 250, 290], 264, 256)
    torch.cuda.synchronize()
    ctx.execute_grouped(x.product, stream=side)
    ctx.execute_grouped(w.product, stream=side)
    side.synchronize()
    x.check()
    w.check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        ctx.execute_grouped(x.product, stream=side)
        ctx.execute_grouped(w.product, stream=side)
    other = Rows("bf16", 64, [0, 60], 128, 64, 0, "silu", sums="groups")
    for off in ([0, 17, 17, 250, 290], [0, 0, 150, 290, 300], [0, 300, 300, 300, 300], [5, 5, 5, 5, 5]):
        for t in (x.c_full, x.aux_full, x.sums, w.c_full):
            t.fill_(float("nan"))
        for y in (x, w):
            y.offsets.copy_(torch.tensor(off, dtype=torch.int32))
            y.bounds = bounds_of(off, 300)
        run(ctx, other)
        graph.replay()
        torch.cuda.synchronize()
        x.check()
        w.check()
    del graph
    torch.cuda.synchronize()


def test_runs_repeat_bit_for_bit(ctx):
    x = Rows("bf16", 900, [0, 130, 131, 500, 900], 520, 512, 1, "gelu", grad=True, sums="groups")
    first = None
    for _ in range(3):
        run(ctx, x)
        now = [x.c.clone(), x.sums.clone()]
        assert first is None or all(torch.equal(p, q) for p, q in zip(first, now))
        first = now


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_expert_layer_forward_and_backward(ctx, dtype):
    """y = act(x W1[e] + b1[e]) W2[e] + b2[e] over routed rows, its gradients against
    64-bit autograd and against differences of the 64-bit function."""
    off = [0, 70, 70, 110, 250]
    t, d, h, groups, act = 250, 96, 160, 4, "silu"
    gen = torch.Generator().manual_seed(21)
    ty = OUT[dtype]
    x, w1, w2 = (torch.randn(s, generator=gen).mul(q).to(ty).cuda() for s, q in
                 (((t, d), 1.0), ((groups, d, h), d ** -0.5), ((groups, h, d), h ** -0.5)))
    b1, b2 = torch.randn(groups, h, generator=gen).cuda(), torch.randn(groups, d, generator=gen).cuda()
    dy = torch.randn((t, d), generator=gen).to(ty).cuda()
    o = torch.tensor(off, dtype=torch.int32).cuda()
    z, u, dz, y, dx = (torch.empty(t, n, dtype=ty, device="cuda") for n in (h, h, h, d, d))
    dw1, dw2, db1, db2 = torch.empty_like(w1), torch.empty_like(w2), torch.empty_like(b1), torch.empty_like(b2)
    ctx.execute_grouped(gdy.Grouped(x, w1, u, o, epilogue=gdy.Epilogue(b1, act, aux=z)))
    ctx.execute_grouped(gdy.Grouped(u, w2, y, o, epilogue=gdy.Epilogue(b2)))
    ctx.execute_act_grad(gdy.ActGrad(dy, bias_grad=db2, offsets=o))
    ctx.execute_grouped(gdy.Grouped(dy, w2, dz, o, trans_b=1,
                                    epilogue=gdy.Epilogue(act=act, aux=z, grad=True, bias_grad=db1)))
    ctx.execute_grouped(gdy.Grouped(u, dy, dw2, o, over="k"))
    ctx.execute_grouped(gdy.Grouped(dz, w1, dx, o, trans_b=1))
    ctx.execute_grouped(gdy.Grouped(x, dz, dw1, o, over="k"))
    torch.cuda.synchronize()
    leaves = [v.double().cpu().requires_grad_(True) for v in (x, w1, b1, w2, b2)]

    def f(x, w1, b1, w2, b2):
        return torch.cat([value(x[a:b] @ w1[e] + b1[e], act) @ w2[e] + b2[e]
                          for e, (a, b) in enumerate(zip(off[:-1], off[1:]))])
    out = f(*leaves)
    loss_w = dy.double().cpu()
    grads = torch.autograd.grad((out * loss_w).sum(), leaves)
    # four roundings to the type on the way, half a step each, and four fp32 sums
    tol = 8 * torch.finfo(ty).eps / 2 if dtype == "bf16" else 64 * 2.0 ** -24 * 16
    for name, got, ref in (("y", y, out), ("dx", dx, grads[0]), ("dw1", dw1, grads[1]), ("db1", db1, grads[2]),
                           ("dw2", dw2, grads[3]), ("db2", db2, grads[4])):
        err = (got.double().cpu() - ref).abs().max() / ref.abs().max()
        assert err <= tol, (name, float(err), tol)
    for got, i in ((dw1, 1), (db1, 2), (dw2, 3), (db2, 4), (dx, 0)):
        v = torch.randn(leaves[i].shape, generator=gen, dtype=torch.float64)
        ends = []
        for sign in (1, -1):
            args = [q.detach() for q in leaves]
            args[i] = args[i] + sign * 1e-4 * v
            ends.append((f(*args) * loss_w).sum())
        diff = float((ends[0] - ends[1]) / 2e-4)
        mine = float((got.double().cpu() * v).sum())
        assert abs(diff - mine) <= tol * float((got.double().cpu().abs() * v.abs()).sum()), (i, diff, mine)
