"""Epilogues, grouped products and activation gradients at their ends: offsets past 32
bits, plain launches' bits, contexts on two streams at once, captured and replayed
calls of few rows, views of unusual strides."""
import os

import pytest

import paper_2409_02227_amd  # noqa: F401  (sets GPU_MAX_HW_QUEUES before HIP starts)

torch = pytest.importorskip("torch")

from paper_2409_02227_amd import gdy  # noqa: E402
from tests.operator_refs import Expected, close, operand, product  # noqa: E402
from tests.test_gpu_epilogue import Case, TABLE  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    c = gdy.Context(0, table=TABLE)
    yield c
    c.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "fp8", "f32"])
@pytest.mark.parametrize("m,n,k", [(17, 65, 129), (64, 1024, 1024), (64, 512, 4096), (100, 1000, 2040), (128, 256, 128),
                                   (300, 2048, 512), (512, 512, 4608), (509, 1023, 1021), (1024, 1024, 64),
                                   (2048, 2048, 128), (9, 256, 16384)])
def test_an_epilogue_that_changes_nothing_gives_the_plain_launchs_bits(ctx, dtype, m, n, k):
    """Every tile that an epilogue may run on in place of the plan's adds in the same
    order: the saved pre-activation, and C, are the plain C."""
    for layout in ("nn", "nt", "tn") if dtype != "fp8" else ("nt", "nn"):
        plain = Case(dtype, m, n, k, layout)
        plain.gemm.epilogue = None
        saved = Case(dtype, m, n, k, layout, aux=True, sums="all")
        for mode in ("selector", "sequential"):
            plain.c.fill_(float("nan")), saved.c.fill_(float("nan")), saved.aux.fill_(float("nan"))
            ctx.execute([plain.gemm], mode=mode)
            ctx.execute([saved.gemm], mode=mode)
            torch.cuda.synchronize()
            assert torch.equal(plain.c, saved.c) and torch.equal(plain.c, saved.aux), (layout, mode)
        saved.check()


def test_grouped_rows_past_32_bits(ctx):
    """A and C of over 4 GiB, the groups in their last rows; rows before stay."""
    rows, n, k = 1 << 21, 1152, 64
    gen = torch.Generator().manual_seed(1)
    a = torch.zeros(rows, 1152, dtype=torch.bfloat16, device="cuda")[:, :k]
    c = torch.full((rows, n), 7.0, dtype=torch.bfloat16, device="cuda")
    off = [rows - 300, rows - 299, rows - 299, rows - 130, rows - 5]
    a[rows - 300:] = operand(gen, 300, k, "bf16")
    b = operand(gen, k, n, "bf16", items=4)
    bias = torch.randn(4, n, generator=gen).cuda()
    o = torch.tensor(off, dtype=torch.int32).cuda()
    ctx.execute_grouped(gdy.Grouped(a, b, c, o, epilogue=gdy.Epilogue(bias, "silu")))
    torch.cuda.synchronize()
    for e, (lo, hi) in enumerate(zip(off[:-1], off[1:])):
        z, s = product(a[lo:hi].float(), b[e].float(), 1.0, bias[e])
        x = Expected(z, s, torch.bfloat16, "silu")
        close(c[lo:hi], x.c, x.c_bound, ("rows", e))
    assert bool((c[rows - 5:] == 7.0).all()) and bool((c[rows - 400:rows - 300] == 7.0).all())
    assert bool((c[:4096] == 7.0).all()) and bool((c[rows // 2 - 64:rows // 2 + 64] == 7.0).all())
    # the activation gradient over the same rows, in place of C
    dz = torch.full((rows, n), 7.0, dtype=torch.bfloat16, device="cuda")
    ctx.execute_act_grad(gdy.ActGrad(c, c, dz, None, "gelu", o))
    torch.cuda.synchronize()
    for lo, hi in zip(off[:-1], off[1:]):
        y = c[lo:hi].double().cpu()
        x = Expected(y, 0 * y, torch.bfloat16, "gelu", aux=c[lo:hi], grad=True)
        close(dz[lo:hi], x.c, x.c_bound, "act_grad")
    assert bool((dz[rows - 5:] == 7.0).all()) and bool((dz[:4096] == 7.0).all())
    assert bool((dz[rows - 400:rows - 300] == 7.0).all())


def test_group_strides_past_32_bits(ctx):
    """Weights, and weight gradients, over 4 GiB apart."""
    gen = torch.Generator().manual_seed(2)
    n, k, far = 136, 264, (1 << 31) + 4096
    pool = torch.empty(far + k * n, dtype=torch.bfloat16, device="cuda")
    w = torch.as_strided(pool, (2, k, n), (far, n, 1))
    w.copy_(operand(gen, k, n, "bf16", items=2))
    x = operand(gen, 90, k, "bf16")
    y = torch.empty(90, n, dtype=torch.bfloat16, device="cuda")
    o = torch.tensor([0, 33, 90], dtype=torch.int32).cuda()
    ctx.execute_grouped(gdy.Grouped(x, w, y, o))
    torch.cuda.synchronize()
    for e, (lo, hi) in enumerate(((0, 33), (33, 90))):
        t = Expected(*product(x[lo:hi].float(), w[e].float()), torch.bfloat16)
        close(y[lo:hi], t.c, t.c_bound, ("rows", e))
    r = w.clone()
    ctx.execute_grouped(gdy.Grouped(x, y, w, o, "k", epilogue=gdy.Epilogue(residual=w)))
    torch.cuda.synchronize()
    for e, (lo, hi) in enumerate(((0, 33), (33, 90))):
        t = Expected(*product(x[lo:hi].float().t(), y[lo:hi].float()), torch.bfloat16, residual=r[e])
        close(w[e], t.c, t.c_bound, ("over K", e))


def test_batch_strides_past_32_bits(ctx):
    gen = torch.Generator().manual_seed(3)
    m, n, k, far = 40, 136, 264, (1 << 31) + 4096
    pool = torch.empty(far + m * n, dtype=torch.bfloat16, device="cuda")
    aux = torch.as_strided(pool, (2, m, n), (far, n, 1))
    aux.copy_(operand(gen, m, n, "bf16", items=2, scale=4.0))
    a, b = operand(gen, m, k, "bf16", items=2), operand(gen, k, n, "bf16")
    c = torch.empty(2, m, n, dtype=torch.bfloat16, device="cuda")
    sums = torch.empty(n, device="cuda")
    saved = aux.clone()
    for out in (c, aux):  # into a tensor of its own, and over the saved values
        ctx.execute([gdy.Gemm(a, b, out, epilogue=gdy.Epilogue(act="silu", aux=aux, grad=True, bias_grad=sums))])
        torch.cuda.synchronize()
        parts = []
        for i in range(2):
            t = Expected(*product(a[i].float(), b.float()), torch.bfloat16, "silu", aux=saved[i], grad=True)
            close(out[i], t.c, t.c_bound, i)
            parts.append(t.sums())
        extra = 2 * 2.0 ** -24 * sum(p.abs() for p, _ in parts)
        close(sums, parts[0][0] + parts[1][0], parts[0][1] + parts[1][1] + extra, "sums")


def test_two_contexts_on_two_streams(ctx):
    """Calls of two contexts at once: each has a workspace of its own."""
    second = gdy.Context(0, table=TABLE)
    try:
        cases = [[Case("bf16", 700, 520, 640, "nn", "gelu", grad=True, sums="all", seed=s),
                  Case("bf16", 40, 520, 4096, "nn", "silu", bias="f32", sums="all", seed=s + 1)] for s in (1, 2)]
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        z = [torch.randn(900, 264, device="cuda") for _ in range(2)]
        dy = [torch.randn(900, 264, device="cuda") for _ in range(2)]
        db = [torch.empty(264, device="cuda") for _ in range(2)]
        torch.cuda.synchronize()
        for _ in range(4):
            for c, s, x, q, p, g in zip((ctx, second), streams, cases, z, dy, db):
                c.execute([t.gemm for t in x], stream=s)
                c.execute_act_grad(gdy.ActGrad(p, q, None, g, "silu"), stream=s)
        torch.cuda.synchronize()
        for x, q, p, g in zip(cases, z, dy, db):
            for t in x:
                t.check()
            y = p.double().cpu()
            close(g, *Expected(y, 0 * y, torch.float32, "silu", aux=q, grad=True).sums(), "act_grad")
    finally:
        second.close()


def test_few_rows_and_activation_gradients_in_a_graph(ctx):
    few = [Case("bf16", 4, 520, 2048, "nt", "silu", bias="f32", residual=True, sums="all"),
           Case("bf16", 16, 136, 1024, "nn", "gelu", aux=True, seed=1),
           Case("bf16", 7, 136, 512, "nn", "gelu", grad=True, sums="items", items=3, seed=2)]
    x, y = torch.randn(2, 1500, 200, device="cuda").unbind(0)
    dz, db = torch.empty_like(x), torch.empty(3, 200, device="cuda")
    o = torch.tensor([0, 700, 700, 1500], dtype=torch.int32).cuda()
    op = gdy.ActGrad(x, y, dz, db, "gelu_tanh", o)

    def work(stream=None):
        ctx.execute_static([c.gemm for c in few], stream=stream)
        ctx.execute_act_grad(op, stream=stream)
    work()
    torch.cuda.synchronize()
    for c in few:
        c.check()
    outs = [t for c in few for t in (c.c, c.sums) if t is not None] + [few[1].aux, dz, db]
    ref = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        work(side)
    other = gdy.ActGrad(torch.randn(5000, 72, device="cuda"), bias_grad=torch.empty(72, device="cuda"))
    for _ in range(3):
        for t in outs:
            t.fill_(float("nan"))
        ctx.execute_act_grad(other)  # eager work of the same context between replays
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(ref, outs))
    del graph
    torch.cuda.synchronize()


def test_views(ctx):
    """Rows of a wider matrix that start off any alignment, every second row, a
    broadcast bias of one layer's groups, one vector as bias of two members."""
    gen = torch.Generator().manual_seed(5)
    wide = operand(gen, 200, 700, "bf16")
    a = wide[1::2, 3:267]
    w = operand(gen, 264, 300, "bf16")[:, 1:250]
    bias = torch.randn(251, generator=gen).to(torch.bfloat16).cuda()[1:250]  # 2 bytes off a dword
    full = torch.full((101, 300), float("nan"), dtype=torch.bfloat16, device="cuda")
    c, c2 = full[1:, 5:254], torch.empty(100, 249, dtype=torch.bfloat16, device="cuda")
    res = wide[::2, 301:550]
    ctx.execute([gdy.Gemm(a, w, c, epilogue=gdy.Epilogue(bias, "relu", res)),
                 gdy.Gemm(a, w, c2, epilogue=gdy.Epilogue(bias, "none"))])
    torch.cuda.synchronize()
    z, s = product(a.float(), w.float(), 1.0, bias)
    t = Expected(z, s, torch.bfloat16, "relu", res)
    close(c, t.c, t.c_bound, "views")
    t = Expected(z, s, torch.bfloat16)
    close(c2, t.c, t.c_bound, "shared bias")
    assert torch.isnan(full[0].float()).all() and torch.isnan(full[:, :5].float()).all()
    assert torch.isnan(full[:, 254:].float()).all()


def test_nan_and_infinity_stay_in_their_rows(ctx):
    """Operands' NaN and infinities reach the outputs of their rows and columns alone,
    also where a tile's edge holds rows of the next group."""
    gen = torch.Generator().manual_seed(6)
    off = [0, 33, 70, 128, 200]
    a, b = operand(gen, 200, 136, "bf16"), operand(gen, 136, 200, "bf16", items=4)
    a[33:70] = float("nan")
    c, sums = torch.empty(200, 200, dtype=torch.bfloat16, device="cuda"), torch.empty(4, 200, device="cuda")
    o = torch.tensor(off, dtype=torch.int32).cuda()
    ctx.execute_grouped(gdy.Grouped(a, b, c, o, epilogue=gdy.Epilogue(act="silu", bias_grad=sums)))
    dw = torch.empty(4, 136, 200, dtype=torch.bfloat16, device="cuda")
    y = operand(gen, 200, 200, "bf16")
    ctx.execute_grouped(gdy.Grouped(a, y, dw, o, "k"))
    torch.cuda.synchronize()
    assert torch.isnan(c[33:70].float()).all() and torch.isnan(sums[1]).all() and torch.isnan(dw[1].float()).all()
    keep = [0, 2, 3]
    assert torch.isfinite(c[:33].float()).all() and torch.isfinite(c[70:].float()).all()
    assert torch.isfinite(sums[keep]).all() and torch.isfinite(dw[keep].float()).all()
    one = Case("bf16", 12, 200, 512, "nt", "gelu", bias="f32", sums="all")
    one.a[5] = float("inf")
    ctx.execute([one.gemm])
    torch.cuda.synchronize()
    rest = [i for i in range(12) if i != 5]
    assert torch.isfinite(one.c[rest].float()).all() and not torch.isfinite(one.c[5].float()).any()


@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
def test_slopes_far_from_zero(ctx, act):
    """fp32 slopes where they are small, and the limits 0 and 1 at infinity (exactly, whatever they multiply).
    Down to 2^-119, a slope's exponentials have arguments y of at most 128 in base 2, off by 1.5 * 2^-24 of
    themselves: a relative error of 1.5 * 2^-24 * 128 ln 2 = 133 * 2^-24 (gelu: the square's rounding too, 178 *
    2^-24); the reciprocal, the exponential and the products add less than 12 * 2^-24 and its polynomial 2^-20,
    16 * 2^-24.  The slope of gelu is exp(-x^2/2) (Q - x / sqrt(2 pi)), that of gelu_tanh and silu p (1 + x ...):
    from 5 on the terms' difference is at least 0.79 of the larger.  Below 5 they are left to other tests."""
    inf = float("inf")
    xs = [-inf, -3e38, -1e5, -129.0, -128.0, -120.0, -104.0, -100.0] + \
        [x for x in (-85.0, -80.0, -75.5, -70.0, -66.0, -64.5, -64.0, -63.0, -50.25, -30.0, -20.0, -12.0, -9.0, -7.5, -6.0, -5.0)] + \
        [5.0, 20.0, 64.0, 65.0, 100.0, 128.0, 129.0, 1e5, 3e38, inf]
    z = torch.tensor(xs, device="cuda").repeat(3, 1)
    dy = torch.tensor([1.0, 2.0 ** 100, -2.0 ** 127], device="cuda")[:, None].expand(3, len(xs)).contiguous()
    dz = torch.full_like(z, float("nan"))
    ctx.execute_act_grad(gdy.ActGrad(dy, z, dz, None, act))
    torch.cuda.synchronize()
    x = z.double().cpu().clamp(-1000.0, 1000.0)
    if act == "relu":
        want = (x > 0).double()
    elif act == "silu":
        p = torch.sigmoid(x)
        want = p * (1 + x * torch.sigmoid(-x))
    elif act == "gelu":
        want = torch.special.erfc(-x / 2 ** 0.5) / 2 + x * torch.exp(-x * x / 2) / (2 * torch.pi) ** 0.5
    else:
        c = (8 / torch.pi) ** 0.5
        u = c * (x + 0.044715 * x ** 3)
        want = torch.sigmoid(u) * (1 + x * torch.sigmoid(-u) * c * (1 + 3 * 0.044715 * x * x))
    want = want * dy.double().cpu()
    bound = 2.0 ** -16 * want.abs() + 2.0 ** -119 * dy.double().cpu().abs()
    close(dz, want, bound, act)
    ends = z.cpu().abs() >= 128.0
    exact = torch.where(z.cpu() > 0, dy.cpu(), torch.zeros(()))
    assert torch.equal(dz.cpu()[ends], exact[ends])
