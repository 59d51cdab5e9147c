"""GEMMs with epilogues through gdy_execute_epilogue against 64-bit references:
every type, layout and tile, batches, odd sizes and pitches, in-place operands,
bias gradients, mixed submissions, other streams and captured graphs."""
import os

import numpy as np
import pytest

import paper_2409_02227_amd  # noqa: F401  (sets GPU_MAX_HW_QUEUES before HIP starts)

torch = pytest.importorskip("torch")

from paper_2409_02227_amd import gdy  # noqa: E402
from tests.operator_refs import (ACTS, IN, OUT, Expected, close, operand, padded, product,  # noqa: E402
                                 untouched)

pytestmark = pytest.mark.gpu
TABLE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                     "paper_2409_02227_amd", "tables", "gfx950.table")
LAYOUTS = {"nn": (0, 0), "nt": (0, 1), "tn": (1, 0), "tt": (1, 1)}


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    c = gdy.Context(0, table=TABLE)
    yield c
    c.close()


class Case:
    """One GEMM with its epilogue, operands on the GPU."""

    def __init__(self, dtype, m, n, k, layout="nn", act="none", grad=False, bias=None, residual=False, aux=False,
                 sums=None, items=0, pad=0, seed=0, in_place=False, bias_items=False):
        self.__dict__.update(dtype=dtype, m=m, n=n, k=k, act=act, grad=grad, items=items, in_place=in_place)
        self.label = (dtype, m, n, k, layout, act, "grad" if grad else "", bias, residual, aux, sums, items, pad)
        print(self.label, flush=True)
        gen = torch.Generator().manual_seed(1000 * seed + 7 * m + 3 * n + k)
        ta, tb = LAYOUTS[layout]
        out = OUT[dtype]
        odt = "bf16" if dtype == "fp8" else dtype
        sc = 1.0 if dtype != "fp8" else 8.0
        self.a = operand(gen, *((k, m) if ta else (m, k)), dtype, pad, items, sc)
        self.b = operand(gen, *((n, k) if tb else (k, n)), dtype, pad, items, sc)
        self.sa, self.sb = (0.25, 0.0625) if dtype == "fp8" else (1.0, 1.0)
        self.c, self.c_full = padded(m, n, out, pad, items=items)
        lead = (items,) if items and bias_items else ()
        self.bias = None if bias is None else torch.randn(lead + (n,), generator=gen).to(
            torch.float32 if bias == "f32" else out).cuda()
        self.res = operand(gen, m, n, odt, pad, items, 2.0) if residual else None
        self.aux = self.aux_full = None
        if grad:
            self.aux = operand(gen, m, n, odt, pad, items, 4.0)
        elif aux:
            self.aux, self.aux_full = padded(m, n, out, pad, items=items)
        self.sums = None
        if sums:
            self.sums = torch.full((items, n) if sums == "items" else (n,), float("nan"), device="cuda")
        if in_place:  # C over the residual, or over the saved pre-activation
            src = self.aux if grad else self.res
            self.c.copy_(src)
            self.src = src.clone()
            if grad:
                self.aux = self.c
            else:
                self.res = self.c
        ep = gdy.Epilogue(self.bias, act, self.res, self.aux, grad, self.sums)
        self.gemm = gdy.Gemm(self.a, self.b, self.c, ta, tb, self.sa, self.sb, epilogue=ep)
        self.ta, self.tb = ta, tb

    def check(self):
        item_sums = []
        res = self.src if self.in_place and not self.grad else self.res
        aux = self.src if self.in_place and self.grad else self.aux
        for i in range(max(self.items, 1)):
            at = (lambda t: None if t is None else t[i] if self.items else t)  # noqa: E731
            a, b = at(self.a).float(), at(self.b).float()
            bias = self.bias if self.bias is None or self.bias.dim() == 1 else self.bias[i]
            z, s = product(a.t() if self.ta else a, b.t() if self.tb else b, self.sa * self.sb, bias,
                           self.dtype == "fp8")
            e = Expected(z, s, OUT[self.dtype], self.act, at(res), at(aux) if self.grad else None, self.grad)
            close(at(self.c), e.c, e.c_bound, self.label)
            if self.aux is not None and not self.grad:
                close(at(self.aux), e.aux, e.aux_bound, ("aux",) + self.label)
            item_sums.append(e.sums())
        if self.sums is not None:
            if self.sums.dim() == 2:
                for i, (ref, bound) in enumerate(item_sums):
                    close(self.sums[i], ref, bound, ("sums",) + self.label)
            else:
                ref, bound = sum(r for r, _ in item_sums), sum(b for _, b in item_sums)
                extra = len(item_sums) * 2.0 ** -24 * sum(e.abs() for e, _ in item_sums)
                close(self.sums, ref, bound + extra, ("sums",) + self.label)
        untouched(self.c, self.c_full, self.label)
        if self.aux_full is not None:
            untouched(self.aux, self.aux_full, ("aux",) + self.label)


def run(ctx, cases, mode="selector", **kw):
    plan = ctx.execute([c.gemm for c in cases], mode=mode, want_plan=True, **kw)
    torch.cuda.synchronize()
    for c in cases:
        c.check()
    return plan


# sizes that reach the tiles of 16 to 256 rows, split-K, odd edges and single elements
SIZES = [(1, 1, 1), (1, 200, 300), (3, 130, 64), (17, 65, 129), (33, 257, 515), (64, 512, 4096), (100, 1000, 2040),
         (130, 257, 96), (300, 520, 256), (512, 1024, 512), (257, 264, 1024)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "fp8", "f32"])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_forward(ctx, dtype, m, n, k):
    for q, layout in enumerate(LAYOUTS):
        act = ACTS[(q + m) % len(ACTS)]
        run(ctx, [Case(dtype, m, n, k, layout, act, bias=("own", "f32", None)[q % 3] if dtype != "f32" else "f32",
                       residual=q % 2 == 0, aux=q != 2, sums="all" if q != 1 else None, seed=q)])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "fp8", "f32"])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_backward(ctx, dtype, m, n, k):
    for q, layout in enumerate(LAYOUTS):
        run(ctx, [Case(dtype, m, n, k, layout, ACTS[(q + n) % len(ACTS)], grad=True, residual=q == 3,
                       bias="f32" if q == 1 else None, sums="all", seed=q)])


@pytest.mark.parametrize("act", ACTS)
def test_every_activation_on_every_path(ctx, act):
    """The 256 x 256 and smaller tiles, the split reduction, both directions."""
    for m, n, k in ((512, 768, 1024), (192, 320, 256), (32, 256, 4096)):
        for grad in (False, True):
            run(ctx, [Case("bf16", m, n, k, "nt", act, grad=grad, bias="f32", sums="all")])
            run(ctx, [Case("f32", m, n, k, "nn", act, grad=grad, residual=True)])


@pytest.mark.parametrize("variant", ["bf16_nn_256x256_w2x4_d2_c0", "bf16_nn_256x128_w2x2_d3_c0",
                                     "bf16_nn_128x128_w2x2_d2_c32", "bf16_nn_64x256_w1x4_m32_c0",
                                     "bf16_nn_64x64_w2x2_d4_c0", "bf16_nn_32x128_w1x4_m32_c64",
                                     "bf16_nn_16x256_w1x4_m16_c0", "fp8_nn_256x256_w2x4_d2_c0",
                                     "fp8_nn_64x128_w2x2_d4_c0", "f32_nn_256x256_w2x4_m32_c0",
                                     "f32_nn_16x64_w1x4_m16_c0"])
def test_every_tile_by_name(ctx, variant):
    vid = ctx.find(variant)
    assert vid >= 0, variant
    dtype = variant.split("_")[0]
    for m, n, k in ((384, 520, 512), (70, 300, 1024)):
        c = Case(dtype, m, n, k, "nn", "gelu_tanh", bias="f32", residual=True, aux=True, sums="all")
        c.gemm.variant = vid
        run(ctx, [c], mode="forced")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "fp8", "f32"])
@pytest.mark.parametrize("m,n,k", [(1, 64, 64), (1, 2048, 2048), (2, 72, 136), (5, 200, 1000), (15, 24, 8192),
                                   (16, 136, 520), (16, 16, 16), (16, 1000, 24)])
def test_few_rows(ctx, dtype, m, n, k):
    """The kernel of at most 16 rows: sizes below a wave's K step and not multiples of
    it, one column block and many, batches, padded and aligned pitches."""
    if dtype == "fp8":
        k, n = (k + 15) // 16 * 16, (n + 15) // 16 * 16
    for q, layout in enumerate(("nn", "nt")):
        run(ctx, [Case(dtype, m, n, k, layout, ACTS[(q + m) % 5], bias="f32", residual=True, aux=True, sums="all",
                       pad=(0, 16)[q]),
                  Case(dtype, m, n, k, layout, ACTS[(q + n) % 5], grad=True, sums="all", seed=1),
                  Case(dtype, m, n, k, layout, "silu", bias="own", sums=("items", "all")[q], items=3, bias_items=q == 0),
                  Case(dtype, m, n, k, layout, seed=2)])


def test_few_rows_give_the_same_bits_alone_and_beside_others(ctx):
    gen = torch.Generator().manual_seed(9)
    one = Case("bf16", 3, 520, 2048, "nt", "silu", bias="f32", sums="all")
    run(ctx, [one])
    ref = one.c.clone(), one.sums.clone()
    x, y = operand(gen, 64, 128, "bf16"), operand(gen, 64, 128, "bf16")
    for others in ([], [Case("bf16", 300, 520, 512, "nt", "gelu", grad=True, sums="all")],
                   [Case("bf16", 2, 64, 512, "nn", "relu", bias="own"), Case("bf16", 700, 520, 512, "nn")]):
        for add in ([], [gdy.Add(x, y, torch.empty_like(x)), gdy.Add(x.float(), y.float(), torch.empty(64, 128, device="cuda"))]):
            for mode in ("selector", "sequential", "go"):
                one.c.fill_(float("nan"))
                ctx.execute([one.gemm] + [o.gemm for o in others] + add, mode=mode)
                torch.cuda.synchronize()
                assert torch.equal(one.c, ref[0]) and torch.equal(one.sums, ref[1])
                for o in others:
                    o.check()
                for a in add:
                    assert torch.equal(a.c, (a.a.float() + a.b.float()).to(a.c.dtype))


@pytest.mark.parametrize("pad", [1, 3, 4, 8])
def test_pitches(ctx, pad):
    for dtype in ("bf16", "f32", "fp8"):
        run(ctx, [Case(dtype, 130, 250, 200, "nn", "silu", bias="f32", residual=True, aux=True, sums="all", pad=pad),
                  Case(dtype, 61, 127, 1030, "nt", "gelu", grad=True, sums="all", pad=pad, seed=1)])


def test_batches(ctx):
    for dtype in ("bf16", "f32"):
        for sums in ("items", "all"):
            run(ctx, [Case(dtype, 70, 130, 96, "nn", "silu", bias="f32", residual=True, aux=True, sums=sums, items=3,
                           bias_items=sums == "items"),
                      Case(dtype, 33, 72, 4096, "nt", "gelu", grad=True, sums=sums, items=2, pad=8)])
    run(ctx, [Case("bf16", 300, 512, 512, "nn", "relu", bias="own", sums="items", items=2)])


def test_in_place(ctx):
    """C over its residual (accumulation), and over the pre-activation it replaces;
    whole tiles, ragged ones and split ones."""
    for m, n, k in ((300, 520, 256), (512, 512, 512), (32, 256, 4096), (5, 33, 40)):
        run(ctx, [Case("bf16", m, n, k, "nn", "silu", residual=True, in_place=True, pad=8)])
        run(ctx, [Case("f16", m, n, k, "nt", "gelu", grad=True, in_place=True, sums="all")])


def test_empty_sizes(ctx):
    run(ctx, [Case("bf16", 40, 70, 0, "nn", "silu", bias="f32", residual=True, aux=True, sums="all")])
    run(ctx, [Case("bf16", 300, 300, 0, "nt", "gelu", grad=True, bias="own", sums="all")])
    # no rows: the bias gradient is zero, nothing else is written
    c = Case("bf16", 0, 70, 64, "nn", "none", bias="own", sums="all")
    d = Case("bf16", 9, 70, 64, "nn", "none", bias="own", sums="all")
    ctx.execute([c.gemm, d.gemm])
    torch.cuda.synchronize()
    assert torch.count_nonzero(c.sums).item() == 0 and not torch.isnan(c.sums).any()
    d.check()


def mixed(seed=0):
    return [Case("bf16", 512, 1024, 1024, "nn", "gelu_tanh", bias="f32", aux=True, seed=seed),
            Case("bf16", 37, 512, 4096, "nt", "silu", bias="own", residual=True, sums="all", seed=seed + 1),
            Case("bf16", 300, 200, 100, "tn", seed=seed + 2),  # no epilogue
            Case("bf16", 129, 1000, 515, "nn", "gelu", grad=True, sums="all", seed=seed + 3),
            Case("f32", 64, 96, 320, "nn", "relu", residual=True, seed=seed + 4),
            Case("fp8", 64, 256, 2048, "nt", "silu", bias="own", seed=seed + 5),
            Case("bf16", 16, 300, 2000, "nn", "none", bias="f32", seed=seed + 6)]


@pytest.mark.parametrize("mode", ["sequential", "default", "go", "selector"])
def test_submissions(ctx, mode):
    """Members with and without epilogues, of several types, in every mode."""
    run(ctx, mixed(), mode=mode)


@pytest.mark.parametrize("mode", ["sequential", "go", "selector"])
def test_plain_members_and_adds_beside_epilogues_keep_their_bits(ctx, mode):
    gen = torch.Generator().manual_seed(3)
    plain = [Case("bf16", m, n, k, lay, seed=m) for m, n, k, lay in
             ((300, 512, 1024, "nn"), (40, 256, 4096, "nt"), (512, 512, 512, "tn"))]
    x, y = operand(gen, 256, 512, "bf16"), operand(gen, 256, 512, "bf16")
    add = gdy.Add(x, y, torch.empty_like(x))
    alone = [gdy.Gemm(c.a, c.b, c.c, c.ta, c.tb) for c in plain]
    ctx.execute(alone + [add], mode=mode)
    torch.cuda.synchronize()
    ref = [c.c.clone() for c in plain] + [add.c.clone()]
    for c in plain:
        c.c.fill_(float("nan"))
    add.c.fill_(float("nan"))
    # the same members with one that has an epilogue: an identity, so that plans agree
    plain[0].gemm.epilogue = gdy.Epilogue(bias=torch.zeros(512, device="cuda"))
    for c in plain[1:]:
        c.gemm.epilogue = None
    ctx.execute([c.gemm for c in plain] + [add], mode=mode)
    torch.cuda.synchronize()
    for r, c in zip(ref, [c.c for c in plain] + [add.c]):
        assert torch.equal(r, c)


def test_runs_repeat_bit_for_bit(ctx):
    c = Case("bf16", 700, 520, 640, "nn", "gelu", grad=True, sums="all")
    d = Case("bf16", 48, 520, 4096, "nn", "silu", bias="f32", sums="all")
    first = None
    for _ in range(3):
        run(ctx, [c, d])
        now = [t.clone() for t in (c.c, c.sums, d.c, d.sums)]
        assert first is None or all(torch.equal(p, q) for p, q in zip(first, now))
        first = now


def test_static_entry_and_another_stream(ctx):
    side = torch.cuda.Stream()
    cases = mixed(20)
    torch.cuda.synchronize()
    ctx.execute_static([c.gemm for c in cases], stream=side)
    side.synchronize()
    for c in cases:
        c.check()
    with torch.cuda.stream(side):
        run(ctx, mixed(40))


def test_captured_graph(ctx):
    cases = mixed(60)
    ctx.execute_static([c.gemm for c in cases])
    torch.cuda.synchronize()
    outs = [t for c in cases for t in (c.c, c.sums, c.aux if not c.grad else None) if t is not None]
    ref = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        ctx.execute_static([c.gemm for c in cases], stream=side)
    other = Case("bf16", 64, 256, 4096, "nn", "silu", bias="f32", sums="all")
    for _ in range(3):
        for t in outs:
            t.fill_(float("nan"))
        run(ctx, [other])  # eager work of the same context between replays
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(r, t) for r, t in zip(ref, outs))
    del graph
    torch.cuda.synchronize()


def test_infinite_pre_activations(ctx):
    """An aux that passed its type's range: the slope is 0 or 1, not NaN."""
    for act in ACTS[1:]:
        c = Case("f16", 4, 64, 32, "nn", act, grad=True)
        c.aux[0, :], c.aux[1, :] = float("inf"), float("-inf")
        plain = Case("f16", 4, 64, 32, "nn")
        plain.gemm.a, plain.gemm.b = c.a, c.b
        ctx.execute([c.gemm, plain.gemm])
        torch.cuda.synchronize()
        assert torch.equal(c.c[0], plain.c[0]), act
        assert torch.count_nonzero(c.c[1]).item() == 0, act


def test_timed_submission(ctx):
    cases = mixed(80)
    ctx.set_timing(True)
    try:
        run(ctx, cases)
        start, end = ctx.kernel_times(len(cases))
    finally:
        ctx.set_timing(False)
    assert all(0 <= s < e for s, e in zip(start, end))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_two_layers_forward_and_backward(ctx, dtype):
    """y = x + act(x W1 + b1) W2 + b2, its gradients against 64-bit autograd and
    against differences of the 64-bit function."""
    t, d, h, act = 96, 128, 256, "gelu_tanh"
    gen = torch.Generator().manual_seed(11)
    ty = OUT[dtype]
    x, w1, w2 = (torch.randn(s, generator=gen).mul(q).to(ty).cuda() for s, q in
                 (((t, d), 1.0), ((d, h), d ** -0.5), ((h, d), h ** -0.5)))
    b1, b2 = torch.randn(h, generator=gen).cuda(), torch.randn(d, generator=gen).cuda()
    dy = torch.randn((t, d), generator=gen).to(ty).cuda()
    z, u, dz, dx = (torch.empty(t, n, dtype=ty, device="cuda") for n in (h, h, h, d))
    y = torch.empty(t, d, dtype=ty, device="cuda")
    dw1, dw2 = torch.empty_like(w1), torch.empty_like(w2)
    db1, db2 = torch.empty(h, device="cuda"), torch.empty(d, device="cuda")
    ctx.execute([gdy.Gemm(x, w1, u, epilogue=gdy.Epilogue(b1, act, aux=z))])
    ctx.execute([gdy.Gemm(u, w2, y, epilogue=gdy.Epilogue(b2, residual=x))])
    ctx.execute_act_grad(gdy.ActGrad(dy, bias_grad=db2))
    ctx.execute([gdy.Gemm(dy, w2, dz, 0, 1, epilogue=gdy.Epilogue(act=act, aux=z, grad=True, bias_grad=db1)),
                 gdy.Gemm(u, dy, dw2, 1, 0)])
    ctx.execute([gdy.Gemm(dz, w1, dx, 0, 1, epilogue=gdy.Epilogue(residual=dy)), gdy.Gemm(x, dz, dw1, 1, 0)])
    torch.cuda.synchronize()
    from tests.operator_refs import value
    leaves = [v.double().cpu().requires_grad_(True) for v in (x, w1, b1, w2, b2)]

    def f(x, w1, b1, w2, b2):
        return x + value(x @ w1 + b1, act) @ w2 + b2
    out = f(*leaves)
    loss_w = dy.double().cpu()
    grads = torch.autograd.grad((out * loss_w).sum(), leaves)
    # every tensor on the way is rounded to the type once: a chain of four roundings and
    # four fp32 sums; half a step each, over values up to the tensor's largest
    tol = 8 * torch.finfo(ty).eps / 2 if dtype == "bf16" else 64 * 2.0 ** -24 * 16
    for name, got, ref in (("y", y, out), ("dx", dx, grads[0]), ("dw1", dw1, grads[1]), ("db1", db1, grads[2]),
                           ("dw2", dw2, grads[3]), ("db2", db2, grads[4])):
        err = (got.double().cpu() - ref).abs().max() / ref.abs().max()
        assert err <= tol, (name, float(err), tol)
    # differences: the loss along a direction, from the function alone
    for got, i in ((dw1, 1), (db1, 2), (dw2, 3), (db2, 4), (dx, 0)):
        v = torch.randn(leaves[i].shape, generator=gen, dtype=torch.float64)
        h_ = 1e-4
        ends = []
        for sign in (1, -1):
            args = [q.detach() for q in leaves]
            args[i] = args[i] + sign * h_ * v
            ends.append((f(*args) * loss_w).sum())
        diff = float((ends[0] - ends[1]) / (2 * h_))
        mine = float((got.double().cpu() * v).sum())
        scale = float((got.double().cpu().abs() * v.abs()).sum())
        assert abs(diff - mine) <= tol * scale, (i, diff, mine)
