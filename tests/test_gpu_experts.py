"""Routing, rows to the experts and back, and quantised rows against plain references: ragged and
odd sizes, pairs without a row, rows of no token, every type, pitch and alignment,
values next to halves, streams, graphs, and the operators together as a layer's
forward and backward passes run them."""
import os

import pytest

import paper_2409_02227_amd  # noqa: F401  (sets GPU_MAX_HW_QUEUES before HIP starts)

torch = pytest.importorskip("torch")

from paper_2409_02227_amd import gdy  # noqa: E402
from tests.operator_refs import EPS32, close, half_step, tiny  # noqa: E402

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


# ---- routing ----------------------------------------------------------------------
def routed(ids, experts):
    """(slots, offsets) by the definition, on the CPU."""
    flat = ids.cpu().reshape(-1).tolist()
    rows, offsets = [], [0]
    by = [[] for _ in range(experts)]
    for p, e in enumerate(flat):
        if 0 <= e < experts:
            by[e].append(p)
    for e in range(experts):
        rows += by[e]
        offsets.append(len(rows))
    slots = [-1] * len(flat)
    for r, p in enumerate(rows):
        slots[p] = r
    return torch.tensor(slots, dtype=torch.int32).reshape(ids.shape), torch.tensor(offsets, dtype=torch.int32)


def route(ctx, ids, experts, **kw):
    slots = torch.full(ids.shape, -7, dtype=torch.int32, device="cuda")
    offsets = torch.full((experts + 1,), -7, dtype=torch.int32, device="cuda")
    ctx.execute_route(gdy.Route(ids, slots, offsets), **kw)
    return slots, offsets


def check_route(ctx, ids, experts):
    print("route", tuple(ids.shape), experts, ids.dtype, flush=True)
    slots, offsets = route(ctx, ids, experts)
    torch.cuda.synchronize()
    want = routed(ids, experts)
    assert torch.equal(offsets.cpu(), want[1]) and torch.equal(slots.cpu(), want[0])


@pytest.mark.parametrize("tokens,top_k,experts", [
    (1, 1, 1), (1, 8, 8), (7, 3, 5), (64, 1, 16), (65, 1, 16), (1024, 1, 255), (1025, 1, 256), (1023, 4, 257), (1024, 4, 64),
    (1025, 4, 64), (4097, 1, 3), (777, 64, 100), (5000, 2, 4096), (16384, 8, 128), (131073, 1, 60), (40000, 8, 4096), (2048, 1, 9), (2049, 1, 9), (16384, 8, 129),
    (0, 2, 16), (33, 2, 0)])
@pytest.mark.parametrize("wide", [False, True])
def test_route(ctx, tokens, top_k, experts, wide):
    gen = torch.Generator().manual_seed(tokens + 31 * top_k + experts)
    ids = torch.randint(-2, experts + 2, (tokens, top_k), generator=gen)
    check_route(ctx, ids.to(torch.int64 if wide else torch.int32).cuda(), experts)


def test_route_uneven_and_padded(ctx):
    """Everything to one expert, nothing to any, one id far outside 32 bits, ids in a wider matrix."""
    for tokens in (1, 1000, 9000):
        for e in (0, 15, -1, 16):
            check_route(ctx, torch.full((tokens, 2), e, dtype=torch.int32).cuda(), 16)
    ids = torch.randint(0, 16, (300, 2)).cuda()
    ids[7, 0], ids[8, 1], ids[9, 0], ids[10, 0] = 1 << 32, -(1 << 32), (1 << 32) + 3, -(1 << 63)
    check_route(ctx, ids, 16)
    wide = torch.randint(0, 60, (3001, 9)).cuda()
    check_route(ctx, wide[:, :4], 60)
    check_route(ctx, wide[:, 3:4], 60)
    check_route(ctx, wide.int()[:, 1:3], 60)


def test_route_largest(ctx):
    """2^24 pairs: parts of many steps; against sorting on the device."""
    tokens, top_k, experts = 1 << 21, 8, 200
    ids = torch.randint(-1, experts + 1, (tokens, top_k), device="cuda", dtype=torch.int32)
    slots, offsets = route(ctx, ids, experts)
    flat = ids.reshape(-1).long()
    key = torch.where((flat >= 0) & (flat < experts), flat, experts)
    order = key.argsort(stable=True)
    want = torch.empty_like(flat)
    want[order] = torch.arange(flat.numel(), device="cuda")
    want = torch.where(key < experts, want, -1)
    assert torch.equal(slots.reshape(-1).long(), want)
    counts = torch.bincount(key, minlength=experts + 1)[:experts]
    assert offsets[0] == 0 and torch.equal(offsets[1:].long(), counts.cumsum(0))


# ---- rows to the experts and back -------------------------------------------------------
def matrix(gen, rows, n, dtype, pad=0, shift=0):
    """Normal values in rows `pad` longer, `shift` elements into their buffer; NaN around."""
    whole = torch.full((rows * (n + pad) + shift + 8,), float("nan"))
    x = whole[shift:shift + rows * (n + pad)].view(rows, n + pad)
    x[:, :n] = torch.randn((rows, n), generator=gen)
    whole = whole.to(dtype).cuda()
    return whole[shift:shift + rows * (n + pad)].view(rows, n + pad)[:, :n], whole


def output(rows, n, dtype, pad=0, shift=0):
    whole = torch.full((rows * (n + pad) + shift + 8,), float("nan"), dtype=dtype, device="cuda")
    return whole[shift:shift + rows * (n + pad)].view(rows, n + pad)[:, :n], whole


def only(view, whole, rows, label):
    """Of a NaN buffer, nothing but these rows of the view was written."""
    n, ld = view.shape[1], view.stride(0)
    mask = torch.ones(whole.numel(), dtype=torch.bool, device="cuda")
    at = view.storage_offset()
    for r in rows:
        mask[at + r * ld:at + r * ld + n] = False
    assert torch.isnan(whole.float()[mask]).all().item(), ("wrote outside", label)


def some_slots(gen, tokens, top_k, rows, drop):
    """Different rows for the pairs, some of them none (-1 and values outside)."""
    perm = torch.randperm(max(rows, tokens * top_k), generator=gen)[:tokens * top_k]
    slots = torch.where(perm < rows, perm, -1)
    gone = torch.rand(tokens * top_k, generator=gen) < drop
    out = torch.tensor([-1, rows, -(1 << 31), (1 << 31) - 1])[torch.randint(0, 4, (tokens * top_k,), generator=gen)]
    slots = torch.where(gone, out, slots).reshape(tokens, top_k).to(torch.int32)
    good = (slots >= 0) & (slots < rows)
    return slots.cuda(), torch.where(good, slots, -1).long(), good


SHAPES = [(1, 1, 1, 1), (1, 2, 3, 64), (5, 3, 20, 1001), (33, 8, 300, 72), (64, 2, 100, 4096), (7, 5, 30, 9000), (300, 4, 1200, 17),
          (3, 64, 200, 130)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("tokens,top_k,rows,n", SHAPES)
@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 0), (3, 1)])
def test_scatter_and_combine(ctx, dtype, tokens, top_k, rows, n, pad, shift):
    label = (dtype, tokens, top_k, rows, n, pad, shift)
    print(label, flush=True)
    t = TYPES[dtype]
    gen = torch.Generator().manual_seed(tokens + 7 * n + 13 * pad + rows)
    slots, at, good = some_slots(gen, tokens, top_k, rows, 0.2 if tokens > 1 else 0.0)
    x, _ = matrix(gen, tokens, n, t, pad, shift)
    z, _ = matrix(gen, rows, n, t, pad, shift)
    used = at[good].tolist()
    for weights in (None, torch.float32, t):
        w = None if weights is None else torch.randn((tokens, top_k), generator=gen).to(weights).cuda()
        w64 = torch.ones((tokens, top_k), dtype=torch.float64) if w is None else w.double().cpu()
        x64, z64 = x.double().cpu(), z.double().cpu()
        # rows to the experts, with and without the gradient of the weights
        for grad in (False, True) if w is not None else (False,):
            out, whole = output(rows, n, t, pad, shift)
            dw = torch.full((tokens, top_k), float("nan"), device="cuda") if grad else None
            ctx.execute_scatter(gdy.Scatter(x, slots, out, w, z if grad else None, dw))
            torch.cuda.synchronize()
            only(out, whole, used, label)
            for i, j in good.nonzero().tolist():
                ref = w64[i, j] * x64[i]
                if w is None:
                    assert torch.equal(out[at[i, j]], x[i]), label
                else:
                    bound = half_step(t) * ref.abs() + 2 * EPS32 * ref.abs() + tiny(t)
                    close(out[at[i, j]], ref, bound, ("scatter", weights) + label)
            if grad:
                prod = x64[:, None, :] * z64[at.clamp(min=0)] * good[:, :, None]
                close(dw, prod.sum(2), (n + 4) * EPS32 * prod.abs().sum(2), ("weight_grad", weights) + label)
        # and back, onto a residual of its own, none, and y itself
        for res in ("own", None, "y"):
            y, whole = output(tokens, n, t, pad, shift)
            r = None
            if res == "own":
                r, _ = matrix(gen, tokens, n, t, pad, shift)
            elif res == "y":
                y.copy_(x)
                r = y
            r64 = torch.zeros((tokens, n), dtype=torch.float64) if r is None else r.double().cpu()
            ctx.execute_combine(gdy.Combine(z, slots, y, w, r))
            torch.cuda.synchronize()
            only(y, whole, range(tokens), label)
            terms = w64[:, :, None] * z64[at.clamp(min=0)] * good[:, :, None]
            ref, size = terms.sum(1) + r64, terms.abs().sum(1) + r64.abs()
            err = (top_k + 3) * EPS32 * size
            close(y, ref, half_step(t) * ref.abs() + 2 * err + tiny(t), ("combine", weights, res) + label)


def test_scatter_copies_bytes(ctx):
    """Without weights rows are copied, bit by bit, NaN and infinity as they are; fp8 rows too."""
    gen = torch.Generator().manual_seed(5)
    slots, at, good = some_slots(gen, 50, 2, 110, 0.1)
    for t, word in ((torch.float8_e4m3fn, torch.uint8), (torch.bfloat16, torch.int16), (torch.float32, torch.int32)):
        for n in (1, 15, 16, 33, 1000):
            print(t, n, flush=True)
            size = word.itemsize
            x = torch.randint(0, 256, (50, n * size), dtype=torch.uint8, generator=gen).cuda().view(word).view(t)
            out = torch.zeros((110, n), dtype=word, device="cuda").view(t)
            ctx.execute_scatter(gdy.Scatter(x, slots, out))
            torch.cuda.synchronize()
            want = torch.zeros((110, n), dtype=word)
            for i, j in good.nonzero().tolist():
                want[at[i, j]] = x.view(word)[i].cpu()
            assert torch.equal(out.view(word).cpu(), want), (t, n)


def test_values_in_rows_without_a_pair(ctx):
    """Infinities and NaN in rows that no slot names, and in row 0 where pairs have none, reach nothing; in
    rows that are named they do what the formula says."""
    t, n = torch.bfloat16, 100
    z = torch.randn(6, n).to(t).cuda()
    z[0], z[5] = float("nan"), float("inf")
    x = torch.randn(3, n).to(t).cuda()
    w = torch.ones(3, 2, device="cuda")
    slots = torch.tensor([[1, -1], [-1, -1], [4, 2]], dtype=torch.int32, device="cuda")
    y = torch.zeros(3, n, dtype=t, device="cuda")
    ctx.execute_combine(gdy.Combine(z, slots, y, w))
    out, dw = torch.zeros_like(z), torch.zeros_like(w)
    ctx.execute_scatter(gdy.Scatter(x, slots, out, w, z, dw))
    torch.cuda.synchronize()
    assert torch.isfinite(y.float()).all() and torch.equal(y[0], z[1]) and not y[1].any()
    assert torch.isfinite(dw).all() and dw[0, 1] == 0 and not dw[1].any()
    assert not out[0].any() and not out[3].any() and not out[5].any()
    slots[1, 0], slots[0, 1] = 5, 0
    ctx.execute_combine(gdy.Combine(z, slots, y, w))
    torch.cuda.synchronize()
    assert torch.isnan(y[0].float()).all() and torch.isinf(y[1].float()).all()


def test_no_rows_and_no_tokens(ctx):
    t = torch.bfloat16
    x, none = torch.randn(4, 32).to(t).cuda(), torch.zeros((0, 32), dtype=t, device="cuda")
    slots = torch.full((4, 2), 3, dtype=torch.int32, device="cuda")
    w, dw = torch.ones(4, 2, device="cuda"), torch.full((4, 2), 9.0, device="cuda")
    ctx.execute_scatter(gdy.Scatter(x, slots, none))
    ctx.execute_scatter(gdy.Scatter(x, slots, none, w, none, dw))
    y = torch.full((4, 32), 7.0, dtype=t, device="cuda")
    ctx.execute_combine(gdy.Combine(none, slots, y, w, x))
    q, s = torch.full((8, 32), 5, dtype=torch.int8, device="cuda"), torch.full((8,), 5.0, device="cuda")
    ctx.execute_quantize(gdy.Quantize(none, q, s, slots[:0]))
    ctx.execute_quantize(gdy.Quantize(x, q[:0], s[:0], slots))
    ctx.execute_combine(gdy.Combine(x, slots[:0], none))
    torch.cuda.synchronize()
    assert not dw.any() and torch.equal(y, x) and (q == 5).all() and (s == 5).all()
    # columns of nothing: gradients of 0, scales of 0
    e = torch.zeros((4, 0), dtype=t, device="cuda")
    dw.fill_(9.0)
    ctx.execute_scatter(gdy.Scatter(e, slots, e, w, e, dw))
    ctx.execute_quantize(gdy.Quantize(e, torch.zeros((4, 0), dtype=torch.int8, device="cuda"), s[:4]))
    torch.cuda.synchronize()
    assert not dw.any() and s.tolist() == [0.0] * 4 + [5.0] * 4


def test_offsets_past_32_bits(ctx):
    """Rows whose byte offsets pass 32 bits, on every side."""
    t, n, far = torch.bfloat16, 1024, 1 << 22
    big = torch.empty((far, n), dtype=t, device="cuda")  # 8 GiB
    rows = [0, 1 << 21, (1 << 21) + 1, far - 1]
    big[rows] = torch.randn(4, n).to(t).cuda()
    slots = torch.tensor([[rows[3]], [rows[0]], [rows[1]], [rows[2]]], dtype=torch.int32, device="cuda")
    y = torch.zeros(4, n, dtype=t, device="cuda")
    ctx.execute_combine(gdy.Combine(big, slots, y))
    torch.cuda.synchronize()
    assert torch.equal(y, big[slots[:, 0].long()])
    x = torch.randn(4, n).to(t).cuda()
    dw, w = torch.zeros(4, 1, device="cuda"), torch.full((4, 1), 2.0, device="cuda")
    want = (x.double() * y.double()).sum(1)
    ctx.execute_scatter(gdy.Scatter(x, slots, big, w))
    torch.cuda.synchronize()
    assert torch.equal(big[slots[:, 0].long()], x * 2)
    bound = (n + 4) * EPS32 * (x.double() * y.double()).abs().sum(1)
    small = torch.zeros((far, n), dtype=torch.int8, device="cuda")
    scales = torch.zeros(far, device="cuda")
    ctx.execute_quantize(gdy.Quantize(big[rows], small, scales, slots))
    torch.cuda.synchronize()
    q, s = reference(big[rows])
    assert torch.equal(small[slots[:, 0].long()].cpu(), q) and int(small.abs().sum(dtype=torch.int64)) == int(q.abs().sum(dtype=torch.int64))
    del small
    z = torch.empty((far, n), dtype=t, device="cuda")
    z[slots[:, 0].long()] = y
    ctx.execute_scatter(gdy.Scatter(x, slots, big, w, z, dw))
    torch.cuda.synchronize()
    close(dw[:, 0], want.cpu(), bound.cpu(), "weight_grad past 32 bits")


# ---- quantised rows -------------------------------------------------------------------
def reference(x):
    """(codes, scales in 64 bits): 127 x / max by a division in 64 bits, which cannot cross a half: the
    quotient of a 31-bit and a 24-bit number is a half or 2^-33 away from one."""
    x = x.double().cpu()
    most = x.abs().amax(1) if x.shape[1] else torch.zeros(x.shape[0], dtype=torch.float64)
    over = torch.where(most > 0, most, torch.ones_like(most))
    return torch.round(x * 127.0 / over[:, None]).to(torch.int8), most / 127.0


def check_quantize(ctx, x, pad=0, shift=0, label=""):
    rows, n = x.shape
    whole = torch.full((rows * (n + pad) + shift + 16,), 99, dtype=torch.int8, device="cuda")
    q = whole[shift:shift + rows * (n + pad)].view(rows, n + pad)[:, :n]
    s = torch.full((rows,), float("nan"), device="cuda")
    ctx.execute_quantize(gdy.Quantize(x, q, s))
    torch.cuda.synchronize()
    want, scale = reference(x)
    bad = (q.cpu() != want).nonzero()
    assert not len(bad), (label, len(bad), bad[0].tolist(), int(q.cpu()[tuple(bad[0])]), int(want[tuple(bad[0])]))
    close(s, scale, EPS32 * scale + 2.0 ** -150, ("scales", label))
    q.fill_(99)
    assert (whole == 99).all(), ("wrote outside", label)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,n", [(1, 1), (3, 7), (65, 16), (33, 17), (5, 1024), (300, 1001), (4, 4096), (3, 9000), (2, 20000), (2, 16385), (3, 16384),
                                     (1030, 8192), (2100, 4096), (5000, 48), (1, 40000)])
def test_quantize(ctx, dtype, rows, n):
    gen = torch.Generator().manual_seed(rows + n)
    for pad, shift in ((0, 0), (16, 0), (3, 1)):
        print(dtype, rows, n, pad, shift, flush=True)
        x, _ = matrix(gen, rows, n, TYPES[dtype], pad, shift)
        check_quantize(ctx, x, pad, shift, (dtype, rows, n, pad, shift))


def test_quantize_next_to_halves(ctx):
    """Quotients that are halves, and values one and two steps beside them, of both signs; rows from the
    smallest to the largest numbers."""
    n = 2 * 127 * 5
    rows = []
    gen = torch.Generator().manual_seed(3)
    for most in [254.0, 127.0, 1.0, 3.3, 0.7] + torch.rand(40, generator=gen).tolist():
        m = torch.tensor(most, dtype=torch.float32)
        half = (torch.arange(127, dtype=torch.float64) + 0.5) * m.double() / 127.0
        v = half.float()
        up, down = torch.nextafter(v, v + 1), torch.nextafter(v, v - 1)
        row = torch.cat([v, up, down, torch.nextafter(up, up + 1), torch.nextafter(down, down - 1)])
        row = torch.cat([row, -row])
        row[0] = m
        rows.append(row.clamp(-float(m), float(m)))
    x = torch.stack(rows)
    assert x.shape[1] == n
    check_quantize(ctx, x.cuda(), label="fp32")
    for scale in (2.0 ** -126, 2.0 ** -110, 2.0 ** -99, 2.0 ** 99, 2.0 ** 118):
        check_quantize(ctx, (x * scale).cuda(), label=("fp32", scale))
    for scale in (2.0 ** -140, 2.0 ** -149):  # subnormal rows: codes of what is left
        check_quantize(ctx, (x * scale).cuda(), label=("fp32", scale))
    odd = torch.arange(1, 255, 2, dtype=torch.float32)
    halves = torch.cat([odd, -odd, torch.tensor([254.0])])[None]
    for t in TYPES.values():
        check_quantize(ctx, halves.to(t).cuda(), label=("halves", t))


def test_quantize_without_numbers(ctx):
    """Rows of zeros have scale 0; rows with an infinity or a NaN a scale that is one, and codes of 0."""
    for t in TYPES.values():
        x = torch.randn(6, 300).to(t).cuda()
        x[0], x[1, 7], x[2, 299], x[3, 0], x[4, 5], x[4, 6] = 0.0, float("nan"), float("inf"), -float("inf"), float("inf"), float("nan")
        q, s = torch.full((6, 300), 9, dtype=torch.int8, device="cuda"), torch.full((6,), 9.0, device="cuda")
        ctx.execute_quantize(gdy.Quantize(x, q, s))
        torch.cuda.synchronize()
        assert not q[:5].any() and s[0] == 0 and s[1].isnan() and s[2] == s[3] == float("inf") and s[4].isnan()
        assert torch.equal(q[5:].cpu(), reference(x[5:])[0])


@pytest.mark.parametrize("dtype", list(TYPES))
def test_quantize_to_slots(ctx, dtype):
    gen = torch.Generator().manual_seed(11)
    for tokens, top_k, rows, n in ((1, 1, 1, 64), (20, 3, 80, 1001), (40, 8, 400, 2048), (3, 2, 10, 20000)):
        print(dtype, tokens, top_k, rows, n, flush=True)
        slots, at, good = some_slots(gen, tokens, top_k, rows, 0.2 if tokens > 1 else 0.0)
        x, _ = matrix(gen, tokens, n, TYPES[dtype], 8)
        q = torch.full((rows, n + 3), 99, dtype=torch.int8, device="cuda")
        s = torch.full((rows,), float("nan"), device="cuda")
        ctx.execute_quantize(gdy.Quantize(x, q[:, :n], s, slots))
        torch.cuda.synchronize()
        codes, scale = reference(x)
        want, want_s = torch.full((rows, n + 3), 99, dtype=torch.int8), torch.full((rows,), float("nan"), dtype=torch.float64)
        for i, j in good.nonzero().tolist():
            want[at[i, j], :n], want_s[at[i, j]] = codes[i], scale[i]
        assert torch.equal(q.cpu(), want)
        named = ~torch.isnan(want_s)
        close(s[named.cuda()], want_s[named], EPS32 * want_s[named], "scales")
        assert torch.isnan(s.cpu()[~named]).all()


# ---- together -----------------------------------------------------------------------------
class Layer:
    """A mixture of experts: route, scatter, two grouped products, combine, and the way back."""

    def __init__(self, ctx, tokens, top_k, experts, n, hidden, seed=0, dtype=torch.bfloat16):
        gen = torch.Generator().manual_seed(seed)
        self.ctx, self.t = ctx, dtype
        self.ids = torch.stack([torch.randperm(experts, generator=gen)[:top_k] for _ in range(tokens)])
        self.ids[torch.rand(tokens, top_k, generator=gen) < 0.1] = -1
        self.ids = self.ids.cuda()
        def rand(*shape, scale=1.0):
            return (torch.randn(shape, generator=gen) * scale).to(dtype).cuda()
        self.x, self.dy, self.res = rand(tokens, n), rand(tokens, n), rand(tokens, n)
        self.w1, self.w2 = rand(experts, n, hidden, scale=n ** -0.5), rand(experts, hidden, n, scale=hidden ** -0.5)
        self.w = torch.rand((tokens, top_k), generator=gen).cuda()
        rows = tokens * top_k
        zeros = lambda *s, t=dtype: torch.zeros(s, dtype=t, device="cuda")  # noqa: E731
        self.slots, self.offsets = zeros(tokens, top_k, t=torch.int32), zeros(experts + 1, t=torch.int32)
        self.xs, self.h, self.z1, self.z2, self.y = zeros(rows, n), zeros(rows, hidden), zeros(rows, hidden), zeros(rows, n), zeros(tokens, n)
        self.dz2, self.dw, self.dz1, self.dxs, self.dx = zeros(rows, n), zeros(tokens, top_k, t=torch.float32), zeros(rows, hidden), zeros(rows, n), zeros(tokens, n)
        self.dw1, self.dw2 = zeros(experts, n, hidden), zeros(experts, hidden, n)

    def run(self, stream=None):
        c, E = self.ctx, gdy.Epilogue
        kw = {"stream": stream}
        c.execute_route(gdy.Route(self.ids, self.slots, self.offsets), **kw)
        c.execute_scatter(gdy.Scatter(self.x, self.slots, self.xs), **kw)
        c.execute_grouped(gdy.Grouped(self.xs, self.w1, self.h, self.offsets, epilogue=E(act="silu", aux=self.z1)), **kw)
        c.execute_grouped(gdy.Grouped(self.h, self.w2, self.z2, self.offsets), **kw)
        c.execute_combine(gdy.Combine(self.z2, self.slots, self.y, self.w, self.res), **kw)
        c.execute_scatter(gdy.Scatter(self.dy, self.slots, self.dz2, self.w, self.z2, self.dw), **kw)
        c.execute_grouped(gdy.Grouped(self.dz2, self.w2, self.dz1, self.offsets, trans_b=1,
                                      epilogue=E(act="silu", aux=self.z1, grad=True)), **kw)
        c.execute_grouped(gdy.Grouped(self.h, self.dz2, self.dw2, self.offsets, over="k"), **kw)
        c.execute_grouped(gdy.Grouped(self.dz1, self.w1, self.dxs, self.offsets, trans_b=1), **kw)
        c.execute_grouped(gdy.Grouped(self.xs, self.dz1, self.dw1, self.offsets, over="k"), **kw)
        c.execute_combine(gdy.Combine(self.dxs, self.slots, self.dx), **kw)

    def results(self):
        return {k: getattr(self, k) for k in ("slots", "offsets", "y", "dx", "dw", "dw1", "dw2")}

    def reference(self):
        """The layer by its formula, token by token, and its gradients by autograd, in 64 bits."""
        leaf = lambda v: v.double().cpu().requires_grad_(True)  # noqa: E731
        x, w1, w2, w = leaf(self.x), leaf(self.w1), leaf(self.w2), leaf(self.w)
        ids = self.ids.cpu()
        rows = []
        for i in range(x.shape[0]):
            y = self.res[i].double().cpu()
            for j in range(ids.shape[1]):
                e = int(ids[i, j])
                if e >= 0:
                    y = y + w[i, j] * (torch.nn.functional.silu(x[i] @ w1[e]) @ w2[e])
            rows.append(y)
        y = torch.stack(rows)
        y.backward(self.dy.double().cpu())
        return {"y": y.detach(), "dx": x.grad, "dw": w.grad, "dw1": w1.grad, "dw2": w2.grad}


def relative(got, ref):
    return float((got.double().cpu() - ref).norm() / ref.norm())


def test_layer_forward_and_backward(ctx):
    """Rounded to bf16 six times on the way to dx, each by at most half a step of 2^-8: a relative error
    (2-norm) of each result below 6 * 2^-8 (roundings of different elements add up as their squares,
    so it is far below)."""
    for tokens, top_k, experts, n, hidden in ((37, 3, 8, 96, 160), (130, 2, 5, 128, 64)):
        x = Layer(ctx, tokens, top_k, experts, n, hidden, tokens)
        x.run()
        torch.cuda.synchronize()
        slots, offsets = routed(x.ids, experts)
        assert torch.equal(x.slots.cpu(), slots) and torch.equal(x.offsets.cpu(), offsets)
        for name, ref in x.reference().items():
            off = relative(getattr(x, name), ref)
            print(name, off, flush=True)
            assert off < 6 * 2.0 ** -8, (name, off)


def test_layer_gradients_against_differences(ctx):
    """In fp32: <dL/dv, u> by the operators against (L(v + h u) - L(v - h u)) / 2h of the forward pass in fp32. The
    difference carries the sums' roundings, n terms of 2^-24 relative to |L|'s terms, over h = 2^-6, and
    h^2 / 6 of the third derivative: 2% of the larger of the slope and the terms' norm covers both."""
    x = Layer(ctx, 40, 2, 6, 64, 96, 9, torch.float32)
    x.run()
    torch.cuda.synchronize()
    grads = {k: v.clone() for k, v in x.results().items() if v.dtype == torch.float32}
    gen = torch.Generator().manual_seed(1)
    h = 2.0 ** -6
    for leaf, grad in (("x", "dx"), ("w", "dw"), ("w1", "dw1"), ("w2", "dw2")):
        v = getattr(x, leaf)
        u = torch.randn(v.shape, generator=gen).cuda()
        u = u / u.norm()
        keep, losses = v.clone(), []
        for sign in (1, -1):
            v.copy_(keep + sign * h * u)
            x.run()
            torch.cuda.synchronize()
            losses.append(float((x.y.double() * x.dy.double()).sum()))
        v.copy_(keep)
        slope, want = (losses[0] - losses[1]) / (2 * h), float((grads[grad].double() * u.double()).sum())
        print(leaf, slope, want, flush=True)
        assert abs(slope - want) <= 0.02 * max(abs(want), float(grads[grad].norm()) / 10), (leaf, slope, want)


def test_layer_in_a_graph_and_on_a_stream(ctx):
    """The whole layer captured and replayed on other inputs, with eager work between the replays; routing of many
    pairs, with its workspace, among it."""
    for tokens in (50, 2100):
        x = Layer(ctx, tokens, 2, 7, 64, 96, 3)
        side = torch.cuda.Stream()
        x.run()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            x.run(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            x.run(side)
        torch.cuda.synchronize()
        other = Layer(ctx, 600, 8, 16, 64, 64, 4)
        for rep in range(3):
            x.ids.copy_(x.ids.roll(rep + 1, 0))
            x.x.mul_(0.5)
            torch.cuda.synchronize()
            x.run()
            torch.cuda.synchronize()
            want = {k: v.clone() for k, v in x.results().items()}
            for v in x.results().values():
                v.fill_(0)
            other.run()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            for k, v in x.results().items():
                assert torch.equal(v, want[k]), (tokens, rep, k)
        del graph
        torch.cuda.synchronize()


def test_two_contexts_and_repeated_results(ctx):
    """Calls of two contexts on two streams at once, and the same bits every time."""
    second = gdy.Context(0, table=TABLE)
    try:
        a, b = Layer(ctx, 3000, 2, 16, 64, 64, 5), Layer(second, 3000, 2, 16, 64, 64, 5)
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        torch.cuda.synchronize()
        for _ in range(3):
            a.run(streams[0])
            b.run(streams[1])
        torch.cuda.synchronize()
        for k, v in a.results().items():
            assert torch.equal(v, b.results()[k]), k
    finally:
        second.close()


def test_more_rows_than_workgroups(ctx):
    """Rows of a workgroup each, more of them than a launch has workgroups: the first are followed by others."""
    t, n, tokens = torch.bfloat16, 2064, (1 << 21) + 5
    gen = torch.Generator(device="cuda").manual_seed(8)
    x = torch.empty((tokens, n), dtype=t, device="cuda").normal_(generator=gen)
    some = torch.cat([torch.arange(16), torch.arange(tokens - 16, tokens), torch.randint(0, tokens, (200,))]).cuda()
    q, s = torch.zeros((tokens, n), dtype=torch.int8, device="cuda"), torch.zeros(tokens, device="cuda")
    ctx.execute_quantize(gdy.Quantize(x, q, s))
    torch.cuda.synchronize()
    want, scale = reference(x[some])
    assert torch.equal(q[some].cpu(), want)
    close(s[some], scale, EPS32 * scale, "scales")
    assert int(torch.count_nonzero(s)) == tokens
    del q, s
    # backward, to the rows in reverse: out = 2 x exactly, sums of n products in fp32
    slots = torch.arange(tokens - 1, -1, -1, dtype=torch.int32, device="cuda")[:, None].contiguous()
    w, dw = torch.full((tokens, 1), 2.0, device="cuda"), torch.full((tokens, 1), float("nan"), device="cuda")
    z = torch.empty((tokens, n), dtype=t, device="cuda").normal_(generator=gen)
    out = torch.zeros_like(x)
    ctx.execute_scatter(gdy.Scatter(x, slots, out, w, z, dw))
    torch.cuda.synchronize()
    other = tokens - 1 - some
    assert torch.equal(out[other], x[some] * 2) and not torch.isnan(dw).any()
    a, b = x[some].double(), z[other].double()
    close(dw[some, 0], (a * b).sum(1).cpu(), (n + 4) * EPS32 * (a * b).abs().sum(1).cpu(), "weight_grad")
    del out
    y = torch.zeros_like(x)
    ctx.execute_combine(gdy.Combine(z, slots, y, None, x))
    torch.cuda.synchronize()
    sums = z[other].double() + x[some].double()
    close(y[some], sums.cpu(), (half_step(t) * sums.abs() + 2 * EPS32 * (z[other].abs() + x[some].abs()).double()).cpu(), "combine")


@pytest.mark.parametrize("tokens,top_k,experts", [(64, 4, 256), (256, 1, 256), (256, 1, 257), (257, 1, 256), (129, 1, 64), (32, 8, 65),
                                                   (4, 64, 200), (1, 1, 256), (63, 1, 2), (2, 1, 4096)])
def test_route_few_pairs(ctx, tokens, top_k, experts):
    """Around the pairs and experts that a small workgroup takes."""
    gen = torch.Generator().manual_seed(tokens + experts)
    ids = torch.randint(-1, experts + 1, (tokens, top_k), generator=gen)
    check_route(ctx, ids.cuda(), experts)
    check_route(ctx, torch.full((tokens, top_k), experts - 1, dtype=torch.int32).cuda(), experts)


class Bounded:
    """A value in 64 bits and how far an fp32 computation of it may be off, element by element.  A sum of K products in
    any order is off by (K + 4) * 2^-24 of their absolute sum, one operation by 2^-24 of its result, on top of what the
    operands bring along."""

    def __init__(self, v, e=None):
        self.v, self.e = v, torch.zeros_like(v) if e is None else e

    def most(self):
        return self.v.abs() + self.e

    def __matmul__(self, o):
        k = self.v.shape[1]
        return Bounded(self.v @ o.v, self.most() @ o.most() - self.v.abs() @ o.v.abs() +
                       (k + 4) * EPS32 * (self.most() @ o.most()))

    def __mul__(self, o):
        return Bounded(self.v * o.v, self.most() * o.most() - (self.v * o.v).abs() + EPS32 * self.most() * o.most())

    def t(self):
        return Bounded(self.v.t(), self.e.t())

    def __getitem__(self, i):
        return Bounded(self.v[i], self.e[i])


def forward64(x, w1, w2, w, res, ids):
    """y of the layer by its formula, in 64 bits."""
    y = [res]
    for e in range(w1.shape[0]):
        i, j = (ids == e).nonzero(as_tuple=True)
        z = torch.nn.functional.silu(x[i] @ w1[e]) @ w2[e]
        y.append(torch.zeros_like(res).index_put((i,), w[i, j][:, None] * z, accumulate=True))
    return sum(y)


def bounded_layer(x):
    """The results of a Layer in fp32 with their bounds.  silu: its slope is below 1.2, its second derivative below 0.6,
    and the kernels' are within 2^-17 of the value and 2^-30, and within 2^-17 of what a slope multiplies."""
    leaf = lambda v: Bounded(v.double().cpu())  # noqa: E731
    a, w1, w2, w, dy, res = (leaf(v) for v in (x.x, x.w1, x.w2, x.w, x.dy, x.res))
    ids = x.ids.cpu()
    parts = {k: ([], []) for k in ("y", "dx")}
    out = {"dw": Bounded(torch.zeros_like(w.v)), "dw1": Bounded(torch.zeros_like(w1.v)), "dw2": Bounded(torch.zeros_like(w2.v))}
    for e in range(w1.v.shape[0]):
        i, j = (ids == e).nonzero(as_tuple=True)
        if not len(i):
            continue
        xs, g = a[i], dy[i]
        z1 = xs @ w1[e]
        s = torch.sigmoid(z1.v)
        h = Bounded(z1.v * s)
        h.e = 1.2 * z1.e + 2.0 ** -17 * (h.v.abs() + 1.2 * z1.e) + 2.0 ** -30
        z2 = h @ w2[e]
        weight = w[i, j]
        weight = Bounded(weight.v[:, None], weight.e[:, None])
        dz2 = weight * g
        dot = Bounded(g.v, g.e) * z2
        dw = Bounded(dot.v.sum(1), dot.e.sum(1) + (dot.v.shape[1] + 4) * EPS32 * dot.most().sum(1))
        dh = dz2 @ w2[e].t()
        slope = s * (1 + z1.v * (1 - s))
        dz1 = Bounded(dh.v * slope, 1.2 * dh.e + dh.most() * (0.6 * z1.e + 2.0 ** -17) + 2.0 ** -30)
        dxs = dz1 @ w1[e].t()
        out["dw"].v[i, j], out["dw"].e[i, j] = dw.v, dw.e
        for name, l, r in (("dw2", h, dz2), ("dw1", xs, dz1)):
            p = l.t() @ r
            out[name].v[e], out[name].e[e] = p.v, p.e
        for name, p in (("y", weight * z2), ("dx", dxs)):
            parts[name][0].append(i), parts[name][1].append(p)
    for name, start in (("y", res), ("dx", Bounded(torch.zeros_like(a.v)))):
        v, e, most = start.v.clone(), start.e.clone(), start.v.abs()
        for i, p in zip(*parts[name]):
            v.index_put_((i,), p.v, accumulate=True), e.index_put_((i,), p.e, accumulate=True)
            most = most.index_put((i,), p.most(), accumulate=True)
        out[name] = Bounded(v, e + (w.v.shape[1] + 4) * EPS32 * most)
    return out


@pytest.mark.parametrize("tokens,top_k,experts,n,hidden", [(40, 2, 6, 64, 96), (37, 3, 8, 96, 160), (1, 1, 1, 5, 7), (130, 5, 5, 33, 130)])
def test_layer_in_fp32(ctx, tokens, top_k, experts, n, hidden):
    """Forward and backward in fp32 against autograd in 64 bits, each element within the roundings that lead to it."""
    x = Layer(ctx, tokens, top_k, experts, n, hidden, tokens, torch.float32)
    x.run()
    torch.cuda.synchronize()
    ref = x.reference()
    for name, b in bounded_layer(x).items():
        assert torch.allclose(b.v, ref[name], rtol=1e-10, atol=1e-11), name  # the bounds' values are autograd's
        print(name, float((getattr(x, name).double().cpu() - b.v).abs().max()), float(b.e.max()), flush=True)
        close(getattr(x, name), b.v, b.e, (name, tokens, top_k, experts, n, hidden))


def test_layer_gradients_along_themselves(ctx):
    """Slopes along directions that are mostly the gradient's own, so that they are as large as it: (L(v + h u) - L(v - h
    u)) / 2h of the layer in 64 bits, h = 2^-16, against <g, u> of the operators in fp32, which may be off by the
    roundings of g's elements.  The difference itself is off by less than 2^-18 of |g|, which is above 2^4: by h^2 / 6 = 2^-34.6
    times a third derivative below 2^16 (a unit step changes no z by more than 2^4, the norm of a row of x, their squares' sum
    by 2^8, and what they are weighted with is below 2^4), and by 2^-53 of L < 2^12 over h."""
    x = Layer(ctx, 40, 2, 6, 64, 96, 9, torch.float32)
    x.run()
    torch.cuda.synchronize()
    bounds = bounded_layer(x)
    leaves = {k: getattr(x, k).double().cpu() for k in ("x", "w1", "w2", "w")}
    res, dy, ids = x.res.double().cpu(), x.dy.double().cpu(), x.ids.cpu()
    gen = torch.Generator().manual_seed(1)
    h = 2.0 ** -16
    for leaf, grad in (("x", "dx"), ("w", "dw"), ("w1", "dw1"), ("w2", "dw2")):
        g = getattr(x, grad).double().cpu()
        r = torch.randn(g.shape, generator=gen, dtype=torch.float64)
        u = g / g.norm() + 0.25 * r / r.norm()
        u /= u.norm()
        ends = [float((forward64(**dict(leaves, **{leaf: leaves[leaf] + sign * h * u}), res=res, ids=ids) * dy).sum())
                for sign in (1, -1)]
        slope, mine = (ends[0] - ends[1]) / (2 * h), float((g * u).sum())
        bound = float((bounds[grad].e * u.abs()).sum()) + 2.0 ** -18 * float(g.norm())
        print(leaf, slope, mine, bound, float(g.norm()), flush=True)
        assert mine > 0.9 * float(g.norm()) and abs(slope - mine) <= bound, (leaf, slope, mine, bound)
