"""Epilogues, grouped products and activation gradients without a GPU: the
binding's structures against the C compiler's, tensors that disagree, and every
refusal of the library, on a host-only context (which checks a call in full
before it says that it cannot run one)."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest

from paper_2409_02227_amd import gdy
from tests import test_copy_wait_states as waits

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, UNSUPPORTED, ALIAS, TOO_MANY = 0, 1, 2, 3, 4
BF = torch.bfloat16


@pytest.fixture(scope="module")
def ctx():
    c = gdy.Context(-1)
    yield c
    c.close()


def status(ctx, fn, *args):
    """The status of a call that passes its checks only to find no device."""
    st = fn(ctx.h, *args)
    msg = ctx.last_error()
    if st == UNSUPPORTED and "host-only" in msg:
        return OK
    assert st != OK and msg, st
    return st


def test_layouts_equal_the_c_compilers(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    structs = {"gdy_epilogue": gdy.EpilogueDesc, "gdy_grouped": gdy.GroupedDesc, "gdy_act_grad": gdy.ActGradDesc}
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "gdy.h"', "int main(void) {"]
    for cname, py in structs.items():
        lines.append(f'  printf("{cname} size %zu\\n", sizeof({cname}));')
        lines += [f'  printf("{cname} {f} %zu\\n", offsetof({cname}, {f}));' for f, _ in py._fields_]
    lines += ['  printf("const acts %d\\n", GDY_ACT_SILU);', '  printf("const groups %d\\n", GDY_MAX_GROUPS);',
              "  return 0;", "}"]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines) + "\n")
    exe = tmp_path / "layout"
    subprocess.run([cc, "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split("\n")
    got = {(a, b): int(c) for a, b, c in (l.split() for l in out if l)}
    assert got[("const", "acts")] == gdy.ACT_SILU and got[("const", "groups")] == gdy.MAX_GROUPS
    for cname, py in structs.items():
        assert got[(cname, "size")] == ctypes.sizeof(py), cname
        for f, _ in py._fields_:
            assert got[(cname, f)] == getattr(py, f).offset, (cname, f)


# ---- the binding --------------------------------------------------------------
def test_epilogue_shapes():
    c, n = torch.zeros(8, 4, dtype=BF), 4
    batch = torch.zeros(3, 8, 4, dtype=BF)
    good = gdy.Epilogue(torch.zeros(n), "silu", torch.zeros(8, 6, dtype=BF)[:, :4], torch.zeros_like(c), False,
                        torch.zeros(n)).desc(c)
    assert (good.act, good.bias_type, good.ldr, good.ldaux) == (gdy.ACT_SILU, gdy.F32, 6, 4)
    e = gdy.Epilogue(torch.zeros(3, n, dtype=BF), residual=batch, bias_grad=torch.zeros(3, n)).desc(batch, 3)
    assert (e.stride_bias, e.stride_r, e.stride_bias_grad, e.bias_type) == (4, 32, 4, gdy.BF16)
    assert gdy.Epilogue(bias_grad=torch.zeros(n)).desc(batch, 3).stride_bias_grad == 0
    bad = [gdy.Epilogue(act="swish"), gdy.Epilogue(bias=torch.zeros(5)), gdy.Epilogue(bias=torch.zeros(8)[::2]),
           gdy.Epilogue(bias=torch.zeros(3, 4)), gdy.Epilogue(residual=torch.zeros(8, 4)),
           gdy.Epilogue(residual=torch.zeros(4, 8, dtype=BF).t()), gdy.Epilogue(aux=torch.zeros(7, 4, dtype=BF)),
           gdy.Epilogue(bias_grad=torch.zeros(4, dtype=BF)), gdy.Epilogue(bias_grad=torch.zeros(5))]
    for x in bad:
        with pytest.raises(ValueError):
            x.desc(c)
    a, b = torch.zeros(8, 16, dtype=BF), torch.zeros(16, 4, dtype=BF)
    assert gdy.epilogue_descs([gdy.Gemm(a, b, c)]) is None
    eps = gdy.epilogue_descs([gdy.Gemm(a, b, c), gdy.Gemm(a, b, c, epilogue=gdy.Epilogue(act="relu"))])
    assert [x.act for x in eps] == [0, gdy.ACT_RELU]


def test_grouped_shapes():
    a, w, c = torch.zeros(10, 16, dtype=BF), torch.zeros(3, 16, 8, dtype=BF), torch.zeros(10, 8, dtype=BF)
    off = torch.zeros(4, dtype=torch.int32)
    d, e = gdy.Grouped(a, w, c, off).descs()
    assert (d.over, d.groups, d.rows, d.n, d.k, d.lda, d.ldb, d.stride_b, d.ldc) == (0, 3, 10, 8, 16, 16, 8, 128, 8)
    assert e is None
    d, e = gdy.Grouped(a, c, w, off, over="k", epilogue=gdy.Epilogue(residual=w)).descs()
    assert (d.over, d.rows, d.n, d.k, d.stride_c, e.stride_r) == (1, 10, 8, 16, 128, 128)
    d, _ = gdy.Grouped(a, w.transpose(1, 2).contiguous(), c, off, trans_b=1).descs()
    assert (d.n, d.k, d.ldb) == (8, 16, 16)
    bad = [gdy.Grouped(a, w, c, off.long()), gdy.Grouped(a, w, c, off[:3]), gdy.Grouped(a, w, c, off, trans_b=1),
           gdy.Grouped(a, w, c[:9], off), gdy.Grouped(a, w, w, off), gdy.Grouped(a, w, c, off, over="n"),
           gdy.Grouped(a, w.transpose(1, 2).contiguous().transpose(1, 2), c, off),
           gdy.Grouped(a, c, w[:2], off, over="k"), gdy.Grouped(a, w, c, off, scales=torch.zeros(2)),
           gdy.Grouped(a, w, c, off, epilogue=gdy.Epilogue(bias=torch.zeros(2, 8)))]
    for g in bad:
        with pytest.raises(ValueError):
            g.descs()


def test_act_grad_shapes():
    x = torch.zeros(10, 8, dtype=BF)
    d = gdy.ActGrad(x, x, x, torch.zeros(2, 8), "gelu", torch.zeros(3, dtype=torch.int32)).desc()
    assert (d.rows, d.n, d.groups, d.stride_bias_grad, d.ldz) == (10, 8, 2, 8, 8)
    for bad in (gdy.ActGrad(x, None, x, act="gelu"), gdy.ActGrad(x, x.float(), x), gdy.ActGrad(x[0]),
                gdy.ActGrad(x, x, x.t().contiguous().t()), gdy.ActGrad(x, x, None, torch.zeros(9))):
        with pytest.raises(ValueError):
            bad.desc()


def test_expanded_and_single_rows():
    """A matrix expanded from one row has no leading dimension, one column wide least of all (stride 0 was taken as
    1: rows behind the only one were read).  A single row's stride says nothing."""
    column, wide = torch.zeros(1, 1, dtype=BF).expand(100, 1), torch.zeros(1, 8, dtype=BF).expand(100, 8)
    full, one, off = torch.zeros(100, 8, dtype=BF), torch.zeros(100, 1, dtype=BF), torch.zeros(3, dtype=torch.int32)
    sums = torch.zeros(1, 8).expand(2, 8)
    w = torch.zeros(2, 1, 8, dtype=BF)
    bad = [lambda: gdy.ActGrad(column, None, one).desc(), lambda: gdy.ActGrad(one, column, one, act="relu").desc(),
           lambda: gdy.ActGrad(one, None, column).desc(), lambda: gdy.ActGrad(wide, None, full).desc(),
           lambda: gdy.ActGrad(full, None, full, sums, offsets=off).desc(),
           lambda: gdy.Grouped(column, w, full, off).descs(), lambda: gdy.Grouped(one, w, wide, off).descs(),
           lambda: gdy.Grouped(one, w, full, off, epilogue=gdy.Epilogue(residual=wide)).descs(),
           lambda: gdy.Grouped(one, w, full, off, epilogue=gdy.Epilogue(bias_grad=sums)).descs(),
           lambda: gdy.Epilogue(aux=column).desc(one),
           lambda: gdy.Gemm(column, w[0], full).desc(), lambda: gdy.Gemm(one, w[0], wide).desc(),
           lambda: gdy.Gemm(torch.zeros(8, 100, dtype=BF), column, torch.zeros(8, 1, dtype=BF)).desc(),
           lambda: gdy.Add(one, one, column).desc(), lambda: gdy.Add(column, one, one).desc()]
    for x in bad:
        with pytest.raises(ValueError, match="expanded"):
            x()
    row = torch.zeros(16, 1, dtype=BF).t()  # 1 x 16, strides (1, 1)
    d = gdy.Gemm(row, torch.zeros(16, 8, dtype=BF), torch.zeros(8, 1, dtype=BF).t()).desc()
    assert (d.lda, d.ldb, d.ldc) == (16, 8, 8)
    assert gdy.Gemm(torch.zeros(4, 32, dtype=BF)[:1, :16], torch.zeros(16, 8, dtype=BF), torch.zeros(1, 8, dtype=BF)).desc().lda == 32
    assert gdy.Add(row, row, row).desc().ldc == 16 and gdy.ActGrad(row, None, row).desc().lddy == 16
    assert gdy.Gemm(one.t(), one, torch.zeros(1, 1, dtype=BF)).desc().k == 100


def test_tensors_of_another_device(monkeypatch):
    """Operands that the context's device cannot read (offsets left on the host, above all) never reach the library."""
    class NoLibrary:
        def __getattr__(self, name):
            raise AssertionError(f"{name} reached")

    class Elsewhere:
        """A tensor's shape and strides on cuda:`at`."""
        def __init__(self, t, at):
            self.t, self.at, self.device = t, at, f"cuda:{at}"

        def get_device(self):
            return self.at

        def __getattr__(self, name):
            return getattr(self.t, name)

        def __getitem__(self, i):
            return Elsewhere(self.t[i], self.at)

    ctx = object.__new__(gdy.Context)
    ctx.h, ctx.lib, ctx.device = None, NoLibrary(), 1
    def here(*shape, dtype=BF):
        return Elsewhere(torch.zeros(*shape, dtype=dtype), 1)
    def operators(change, to):
        def t(name, *shape, dtype=BF):
            x = here(*shape, dtype=dtype)
            return to(x) if name == change else x
        off = t("offsets", 4, dtype=torch.int32)
        e = gdy.Epilogue(t("bias", 8), "gelu", t("residual", 10, 8), t("aux", 10, 8), True, t("bias_grad", 8, dtype=torch.float32))
        yield "gemm", lambda: ctx.execute([gdy.Gemm(t("a", 10, 16), t("b", 16, 8), t("c", 10, 8), epilogue=e)])
        yield "static", lambda: ctx.execute_static([gdy.Gemm(t("a", 10, 16), t("b", 16, 8), t("c", 10, 8), epilogue=e)])
        yield "grouped", lambda: ctx.execute_grouped(gdy.Grouped(t("a", 10, 16), t("b", 3, 16, 8), t("c", 10, 8), off, epilogue=e))
        yield "act_grad", lambda: ctx.execute_act_grad(gdy.ActGrad(t("dy", 10, 8), t("z", 10, 8), t("dz", 10, 8),
                                                                   t("bias_grad", 8, dtype=torch.float32), "gelu", off))
    monkeypatch.setattr(gdy, "_stream_handle", lambda *a: None)
    takes = {"gemm": ("a", "b", "c", "bias", "residual", "aux", "bias_grad"),
             "grouped": ("a", "b", "c", "bias", "residual", "aux", "bias_grad", "offsets"),
             "act_grad": ("dy", "z", "dz", "bias_grad", "offsets")}
    takes["static"] = takes["gemm"]
    for change in sorted({n for names in takes.values() for n in names}) + [None]:
        for to in (lambda x: x.t, lambda x: Elsewhere(x.t, 0)):
            for kind, call in operators(change, to):
                if change in takes[kind]:
                    with pytest.raises(ValueError, match="cuda:1"):
                        call()
                else:
                    with pytest.raises(AssertionError, match="reached"):
                        call()


def test_the_current_stream_is_the_contexts_devices(monkeypatch):
    """Without a stream a call runs on the current stream of the context's device, whichever device is current."""
    import types
    seen = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: seen.append((name, [a.value for a in args if isinstance(a, ctypes.c_void_p)])) or 0

    monkeypatch.setattr(torch.cuda, "current_stream",
                        lambda device=None: types.SimpleNamespace(cuda_stream=100 + (0 if device is None else device)))
    monkeypatch.setattr(gdy, "_check_device", lambda *a: None)
    ctx = object.__new__(gdy.Context)
    ctx.h, ctx.lib, ctx.device = None, Library(), 3
    a, b, c, off = torch.zeros(10, 16, dtype=BF), torch.zeros(16, 8, dtype=BF), torch.zeros(10, 8, dtype=BF), torch.zeros(2, dtype=torch.int32)
    for g in (gdy.Gemm(a, b, c), gdy.Gemm(a, b, c, epilogue=gdy.Epilogue(act="relu"))):
        ctx.execute([g])
        ctx.execute_static([g])
    ctx.execute_grouped(gdy.Grouped(a, b[None], c, off))
    ctx.execute_act_grad(gdy.ActGrad(c, c, c, act="relu"))
    ctx.execute([gdy.Gemm(a, b, c)], stream=7)
    names = [n for n, _ in seen]
    assert names == ["gdy_execute", "gdy_execute_static", "gdy_execute_epilogue", "gdy_execute_epilogue_static",
                     "gdy_execute_grouped", "gdy_execute_act_grad", "gdy_execute"]
    assert [v[-1] for _, v in seen] == [103] * 6 + [7], seen


# ---- the library's refusals -------------------------------------------------------
BASE = 1 << 32  # addresses that nothing reads on a host-only context


def gemm(**kw):
    g = gdy.GemmDesc()
    g.m, g.n, g.k = 64, 96, 128
    g.a_type = g.b_type = g.c_type = gdy.BF16
    g.a, g.lda, g.b, g.ldb, g.c, g.ldc = BASE, 128, BASE + (1 << 24), 96, BASE + (2 << 24), 96
    g.scale_a = g.scale_b = 1.0
    for k, v in kw.items():
        setattr(g, k, v)
    return g


def epilogue(**kw):
    e = gdy.EpilogueDesc()
    e.act, e.bias, e.bias_type = gdy.ACT_SILU, BASE + (3 << 24), gdy.BF16
    e.residual, e.ldr, e.aux, e.ldaux = BASE + (4 << 24), 96, BASE + (5 << 24), 96
    e.bias_grad = BASE + (6 << 24)
    for k, v in kw.items():
        setattr(e, k, v)
    return e


def run_epilogue(ctx, gemms, epilogues, mode=gdy.SELECTOR, static=False):
    ga = (gdy.GemmDesc * len(gemms))(*gemms)
    ea = (gdy.EpilogueDesc * len(epilogues))(*epilogues)
    fn = ctx.lib.gdy_execute_epilogue_static if static else ctx.lib.gdy_execute_epilogue
    return status(ctx, fn, ga, ea, len(gemms), mode, 0, None, None)


@pytest.mark.parametrize("g,e,want", [
    ({}, {}, OK),
    ({}, {"act": 5}, INVALID), ({}, {"act": -1}, INVALID), ({}, {"grad": 2}, INVALID), ({}, {"reserved": 1}, INVALID),
    ({}, {"bias_type": gdy.F16}, UNSUPPORTED), ({}, {"bias_type": gdy.F32}, OK), ({}, {"bias_type": 9}, UNSUPPORTED),
    ({}, {"bias": None, "bias_type": 9}, OK),
    ({}, {"ldr": 95}, INVALID), ({}, {"ldaux": 95}, INVALID),
    ({}, {"bias": BASE + (3 << 24) + 1}, UNSUPPORTED), ({}, {"bias": BASE + 2, "bias_type": gdy.F32}, UNSUPPORTED),
    ({}, {"residual": BASE + (4 << 24) + 1}, UNSUPPORTED), ({}, {"aux": BASE + (5 << 24) + 1}, UNSUPPORTED),
    ({}, {"bias_grad": BASE + (6 << 24) + 2}, UNSUPPORTED),
    ({}, {"grad": 1, "aux": None}, INVALID), ({}, {"grad": 1, "aux": None, "act": 0}, OK),
    ({}, {"ldr": 1 << 21, "residual": 1 << 40}, OK), ({}, {"ldr": 1 << 23}, UNSUPPORTED), ({}, {"ldaux": 1 << 23}, UNSUPPORTED),
    # C over its own residual, and over the pre-activation it replaces; nothing else overlaps
    ({}, {"residual": BASE + (2 << 24)}, OK), ({}, {"residual": BASE + (2 << 24) + 2}, ALIAS),
    ({}, {"residual": BASE + (2 << 24), "ldr": 100}, ALIAS),
    ({}, {"aux": BASE + (2 << 24)}, ALIAS), ({}, {"aux": BASE + (2 << 24), "grad": 1}, OK),
    ({}, {"aux": BASE + (2 << 24), "grad": 1, "act": 0}, OK),  # not read
    ({}, {"aux": BASE + 64}, ALIAS), ({}, {"bias_grad": BASE + 64}, ALIAS),
    ({}, {"bias_grad": BASE + (2 << 24) + 64}, ALIAS), ({}, {"bias": BASE + (2 << 24)}, ALIAS),
    ({}, {"bias_grad": BASE + (3 << 24)}, ALIAS), ({}, {"aux": BASE + (4 << 24)}, ALIAS),
    # batches
    ({"batch": 3, "stride_c": 64 * 96}, {"stride_r": 64 * 96, "stride_aux": 64 * 96}, OK),
    ({"batch": 3, "stride_c": 64 * 96}, {"stride_aux": 64 * 96 - 1}, ALIAS),
    ({"batch": 3, "stride_c": 64 * 96}, {"stride_aux": 0, "grad": 1}, OK),
    ({"batch": 3, "stride_c": 64 * 96}, {"stride_aux": 64 * 96, "stride_r": -1}, INVALID),
    ({"batch": 3, "stride_c": 64 * 96}, {"stride_aux": 64 * 96, "stride_bias": -96}, INVALID),
    ({"batch": 3, "stride_c": 64 * 96}, {"stride_aux": 64 * 96, "stride_bias_grad": 95}, ALIAS),
    ({"batch": 3, "stride_c": 64 * 96}, {"stride_aux": 64 * 96, "stride_bias_grad": 96}, OK),
    # strides and sums past what the launches' byte offsets and threads hold
    ({"batch": 3, "stride_c": 64 * 96}, {"stride_aux": 64 * 96, "stride_r": 1 << 62}, UNSUPPORTED),
    ({"batch": 3, "stride_c": 64 * 96}, {"stride_aux": (1 << 63) - 1}, UNSUPPORTED),
    ({"batch": 3, "stride_c": 64 * 96}, {"stride_aux": 64 * 96, "stride_bias": 1 << 61}, UNSUPPORTED),
    ({"batch": 3, "stride_c": 64 * 96}, {"stride_aux": 64 * 96, "stride_bias_grad": 1 << 61}, UNSUPPORTED),
    ({"batch": 1 << 20, "stride_c": 64 * 96, "c": 1 << 42},
     {"aux": None, "stride_bias_grad": 96, "residual": None, "bias_grad": 1 << 41}, UNSUPPORTED),
    # sizes of nothing
    ({"m": 0}, {"residual": None, "aux": None}, OK), ({"m": 0}, {"bias_grad": BASE + 2}, UNSUPPORTED),
    ({"n": 0}, {"bias_grad": 3}, OK), ({"k": 0}, {}, OK),
    # the GEMM's own checks hold
    ({"ldc": 95}, {}, INVALID), ({"c_type": gdy.F16}, {}, UNSUPPORTED),
])
def test_epilogue_checks(ctx, g, e, want):
    assert run_epilogue(ctx, [gemm(**g)], [epilogue(**e)]) == want
    assert run_epilogue(ctx, [gemm(**g)], [epilogue(**e)], gdy.SEQUENTIAL, static=True) == want


def test_epilogues_across_members(ctx):
    far = {k: BASE + (q << 24) for q, k in enumerate(("a", "b", "c"), 20)}
    ep2 = {"bias": BASE + (23 << 24), "residual": BASE + (24 << 24), "aux": BASE + (25 << 24),
           "bias_grad": BASE + (26 << 24)}
    two = [gemm(), gemm(**far)]
    assert run_epilogue(ctx, two, [epilogue(), epilogue(**ep2)]) == OK
    assert run_epilogue(ctx, two, [epilogue(), epilogue()]) == ALIAS  # both write one aux
    for field, at in (("residual", 2 << 24), ("bias", 5 << 24), ("aux", 0)):  # reads or writes the first's
        assert run_epilogue(ctx, two, [epilogue(), epilogue(**dict(ep2, **{field: BASE + at}))]) == ALIAS
    zero = gdy.EpilogueDesc()
    assert run_epilogue(ctx, two, [zero, zero]) == OK
    add = gemm(op=gdy.ADD, k=0, m=64, n=96, lda=96, a=far["a"], b=far["b"], c=far["c"])
    assert run_epilogue(ctx, [gemm(), add], [epilogue(), zero]) == OK
    assert run_epilogue(ctx, [gemm(), add], [epilogue(), epilogue(**ep2)]) == INVALID
    # no array of epilogues at all
    assert status(ctx, ctx.lib.gdy_execute_epilogue, (gdy.GemmDesc * 1)(gemm()), None, 1, gdy.SELECTOR, 0, None, None) == OK
    assert ctx.lib.gdy_execute_epilogue(None, None, None, 0, 0, 0, None, None) == INVALID


def grouped(**kw):
    g = gdy.GroupedDesc()
    g.over, g.groups, g.rows, g.n, g.k = 0, 4, 64, 96, 128
    g.a_type = g.b_type = g.c_type = gdy.BF16
    g.offsets = BASE + (30 << 24)
    g.a, g.lda, g.b, g.ldb, g.stride_b = BASE, 128, BASE + (1 << 24), 96, 128 * 96
    g.c, g.ldc, g.stride_c = BASE + (2 << 24), 96, 0
    if kw.get("over"):
        g.stride_b, g.stride_c = 0, 128 * 96
    g.scale_a = g.scale_b = 1.0
    for k, v in kw.items():
        setattr(g, k, v)
    return g


FP8 = {"a_type": gdy.FP8_E4M3, "b_type": gdy.FP8_E4M3}
ONLY_R = {"act": 0, "bias": None, "aux": None, "bias_grad": None}


@pytest.mark.parametrize("g,e,want", [
    ({}, None, OK), ({}, {}, OK), ({"over": 1}, None, OK),
    ({"over": 2}, None, INVALID), ({"groups": -1}, None, INVALID), ({"rows": -1}, None, INVALID),
    ({"n": -1}, None, INVALID), ({"k": -1}, None, INVALID), ({"groups": 4097}, None, TOO_MANY),
    ({"groups": 4096, "b": 1 << 40}, None, OK), ({"groups": 0, "offsets": None}, None, OK),
    ({"a_type": gdy.F16}, None, UNSUPPORTED), ({"c_type": gdy.F32}, None, UNSUPPORTED), (FP8, None, OK),
    ({"trans_b": 2}, None, INVALID), ({"trans_b": 1, "ldb": 128}, None, OK), ({"over": 1, "trans_b": 1}, None, INVALID),
    ({"scale_a": 2.0}, None, INVALID), ({"scales": BASE + (31 << 24)}, None, INVALID),
    (dict(FP8, scales=BASE + (31 << 24), scale_b=0.5), None, OK), (dict(FP8, scale_a=float("nan")), None, INVALID),
    ({"offsets": None}, None, INVALID), ({"offsets": BASE + (30 << 24) + 2}, None, INVALID),
    ({"a": None}, None, INVALID), ({"b": None}, None, INVALID), ({"c": None}, None, INVALID),
    ({"lda": 127}, None, INVALID), ({"ldb": 95}, None, INVALID), ({"ldc": 95}, None, INVALID),
    ({"a": BASE + 1}, None, UNSUPPORTED), ({"b": BASE + (1 << 24) + 1}, None, UNSUPPORTED),
    ({"c": BASE + (2 << 24) + 1}, None, UNSUPPORTED), ({"stride_b": -1}, None, INVALID), ({"stride_b": 0}, None, OK),
    ({"over": 1, "stride_c": 128 * 96 - 1}, None, ALIAS), ({"over": 1, "stride_c": 0, "groups": 1}, None, OK),
    ({"c": BASE + 64}, None, ALIAS), ({"c": BASE + (1 << 24)}, None, ALIAS), ({"c": BASE + (30 << 24)}, None, ALIAS),
    ({"c": BASE + (1 << 24) + 2 * (4 * 128 * 96 - 1)}, None, ALIAS),  # the last element of the last group's B
    ({"k": 0}, None, OK), ({"n": 0, "c": None}, None, OK), ({"rows": 0, "c": None}, None, OK),
    ({"over": 1, "rows": 0, "a": None, "b": None}, None, OK),
    # extents: over K the operands end within 2 GiB, over rows a group's B and a tile's rows
    ({"rows": 1 << 24, "a": 1 << 40, "c": 2 << 40}, None, OK), ({"rows": (1 << 31) - 4096}, None, UNSUPPORTED),
    ({"over": 1, "rows": 1 << 24}, None, UNSUPPORTED), ({"lda": 1 << 22}, None, UNSUPPORTED), ({"lda": 1 << 20, "a": 1 << 40}, None, OK),
    ({"ldc": 1 << 22}, None, UNSUPPORTED), ({"ldb": 1 << 23, "stride_b": 1 << 40, "b": 1 << 45}, None, UNSUPPORTED),
    ({"stride_b": 1 << 62}, None, UNSUPPORTED), ({"over": 1, "stride_c": (1 << 63) - 1}, None, UNSUPPORTED),
    ({"groups": 4096, "rows": 0, "n": 1 << 15, "k": 0, "c": None},
     dict(ONLY_R, residual=None, stride_bias_grad=1 << 15, bias_grad=1 << 41), UNSUPPORTED),
    # epilogues
    ({}, {"act": 7}, INVALID), ({}, {"ldr": 95}, INVALID), ({}, {"stride_bias": -1}, INVALID),
    ({}, {"stride_bias_grad": 10}, ALIAS), ({}, {"stride_bias_grad": 96}, OK), ({}, {"grad": 1, "aux": None}, INVALID),
    ({}, {"residual": BASE + (2 << 24)}, OK), ({}, {"aux": BASE + (2 << 24)}, ALIAS),
    ({}, {"residual": BASE + (2 << 24), "stride_r": 5}, OK),  # ignored over rows
    ({}, {"aux": BASE + (30 << 24)}, ALIAS), ({}, {"bias_grad": BASE}, ALIAS), ({}, {"ldr": 1 << 22}, UNSUPPORTED),
    ({"rows": 0, "c": None}, {"bias_grad": 2}, UNSUPPORTED),
    ({"over": 1}, {}, UNSUPPORTED), ({"over": 1}, dict(ONLY_R, bias_grad=BASE + (6 << 24)), UNSUPPORTED),
    ({"over": 1}, dict(ONLY_R, stride_r=128 * 96), OK),
    ({"over": 1}, dict(ONLY_R, residual=BASE + (2 << 24), stride_r=128 * 96), OK),
    ({"over": 1}, dict(ONLY_R, residual=BASE + (2 << 24), stride_r=0), ALIAS),
])
def test_grouped_checks(ctx, g, e, want):
    ep = None if e is None else ctypes.byref(epilogue(**e))
    assert status(ctx, ctx.lib.gdy_execute_grouped, ctypes.byref(grouped(**g)), ep, None) == want


def act_grad(**kw):
    g = gdy.ActGradDesc()
    g.rows, g.n, g.type, g.act, g.groups = 64, 96, gdy.BF16, gdy.ACT_GELU, 4
    g.offsets = BASE + (30 << 24)
    g.dy, g.lddy, g.z, g.ldz, g.dz, g.lddz = BASE, 96, BASE + (1 << 24), 96, BASE + (2 << 24), 96
    g.bias_grad, g.stride_bias_grad = BASE + (3 << 24), 96
    for k, v in kw.items():
        setattr(g, k, v)
    return g


@pytest.mark.parametrize("g,want", [
    ({}, OK), ({"offsets": None, "groups": 0}, OK), ({"type": gdy.F32}, OK), ({"type": gdy.FP8_E4M3}, UNSUPPORTED),
    ({"rows": -1}, INVALID), ({"n": -1}, INVALID), ({"groups": -1}, INVALID), ({"groups": 4097}, TOO_MANY),
    ({"act": 9}, INVALID), ({"reserved": 1}, INVALID), ({"dz": None, "bias_grad": None}, INVALID),
    ({"dz": None}, OK), ({"bias_grad": None}, OK), ({"dy": None}, INVALID), ({"z": None}, INVALID),
    ({"z": None, "act": 0}, OK), ({"lddy": 95}, INVALID), ({"ldz": 95}, INVALID), ({"lddz": 95}, INVALID),
    ({"dy": BASE + 1}, UNSUPPORTED), ({"z": BASE + (1 << 24) + 1}, UNSUPPORTED), ({"offsets": BASE + 2}, UNSUPPORTED),
    ({"bias_grad": BASE + (3 << 24) + 2}, UNSUPPORTED), ({"stride_bias_grad": 0}, OK), ({"stride_bias_grad": 95}, ALIAS),
    ({"stride_bias_grad": -96}, INVALID), ({"dz": BASE}, OK), ({"dz": BASE + (1 << 24)}, OK), ({"dz": BASE + 2}, ALIAS),
    ({"dz": BASE, "lddz": 100}, ALIAS), ({"bias_grad": BASE}, ALIAS), ({"dz": BASE + (30 << 24)}, ALIAS),
    ({"stride_bias_grad": 1 << 62}, UNSUPPORTED),
    ({"rows": 0, "groups": 4096, "n": 1 << 15, "stride_bias_grad": 1 << 15, "bias_grad": 1 << 41}, UNSUPPORTED),
    ({"rows": 0, "groups": 4096, "n": 1 << 14, "stride_bias_grad": 1 << 14, "bias_grad": 1 << 41}, OK),
    ({"rows": 0, "dy": None}, OK), ({"n": 0}, OK), ({"rows": (1 << 31) - 4096}, UNSUPPORTED), ({"ldz": 1 << 23}, UNSUPPORTED),
])
def test_act_grad_checks(ctx, g, want):
    assert status(ctx, ctx.lib.gdy_execute_act_grad, ctypes.byref(act_grad(**g)), None) == want


@pytest.mark.parametrize("ld", [(1 << 31) - 1, 1 << 55, (1 << 55) + 96, 1 << 61, 1 << 62, (1 << 62) + 96, (1 << 63) - 1])
def test_leading_dimensions_past_every_offset(ctx, ld):
    """Pitches whose product with rows and element size leaves 64 bits, and the largest of 32, are refused as
    the ones just past the limit are."""
    for e in ({"ldr": ld}, {"ldaux": ld}):
        assert run_epilogue(ctx, [gemm()], [epilogue(**e)]) == UNSUPPORTED
        assert run_epilogue(ctx, [gemm(m=1)], [epilogue(**e)]) == UNSUPPORTED
        assert status(ctx, ctx.lib.gdy_execute_grouped, ctypes.byref(grouped()), ctypes.byref(epilogue(**e)), None) == UNSUPPORTED
    for g in ({"lda": ld}, {"ldb": ld}, {"ldc": ld}):
        assert run_epilogue(ctx, [gemm(**g)], [gdy.EpilogueDesc()]) == UNSUPPORTED
        assert status(ctx, ctx.lib.gdy_execute, (gdy.GemmDesc * 1)(gemm(**g)), 1, gdy.SELECTOR, 0, None, None) == UNSUPPORTED
        add = gemm(op=gdy.ADD, k=0, lda=96, **{k: v for k, v in g.items() if k != "lda"})
        add.lda = g.get("lda", 96)
        assert status(ctx, ctx.lib.gdy_execute, (gdy.GemmDesc * 1)(add), 1, gdy.SELECTOR, 0, None, None) == UNSUPPORTED
        for over in (0, 1):
            assert status(ctx, ctx.lib.gdy_execute_grouped, ctypes.byref(grouped(over=over, **g)), None, None) == UNSUPPORTED
    for a in ({"lddy": ld}, {"ldz": ld}, {"lddz": ld}):
        assert status(ctx, ctx.lib.gdy_execute_act_grad, ctypes.byref(act_grad(**a)), None) == UNSUPPORTED
    # rows and columns past 32 bits
    assert run_epilogue(ctx, [gemm(m=ld, trans_a=1, lda=ld, ldc=96)], [gdy.EpilogueDesc()]) == UNSUPPORTED
    assert run_epilogue(ctx, [gemm(n=ld, ldb=ld, ldc=ld)], [gdy.EpilogueDesc()]) == UNSUPPORTED
    assert run_epilogue(ctx, [gemm(k=ld, lda=ld)], [gdy.EpilogueDesc()]) == UNSUPPORTED


@pytest.mark.parametrize("stride", [1 << 45, 1 << 61, (1 << 61) + 64 * 128, 1 << 62, (1 << 63) - 1])
def test_batch_strides_past_every_offset(ctx, stride):
    """Strides between a member's items that leave 64-bit byte offsets are refused, as an epilogue's are; the
    largest allowed ones with the most items still compare as ranges."""
    good = {"batch": 3, "stride_a": 64 * 128, "stride_b": 128 * 96, "stride_c": 64 * 96}
    zero = gdy.EpilogueDesc()
    for field in ("stride_a", "stride_b", "stride_c"):
        g = gemm(**dict(good, **{field: stride}))
        add = gemm(**dict(good, **{field: stride}), op=gdy.ADD, k=0, lda=96)
        for x in (g, add):
            assert run_epilogue(ctx, [x], [zero]) == UNSUPPORTED
            assert status(ctx, ctx.lib.gdy_execute, (gdy.GemmDesc * 1)(x), 1, gdy.SELECTOR, 0, None, None) == UNSUPPORTED
        single = gemm(**{field: stride})  # ignored without a batch
        assert run_epilogue(ctx, [single], [zero]) == OK
    far = {"stride_a": 1 << 44, "a": 1 << 46, "batch": 3, "stride_c": 64 * 96, "stride_b": 0}
    assert run_epilogue(ctx, [gemm(**far)], [zero]) == OK
    most = {"m": 1, "n": 1, "k": 1, "lda": 1, "ldb": 1, "ldc": 1, "batch": (1 << 31) - (1 << 23), "stride_a": 1 << 44, "a": 8 << 40}
    assert run_epilogue(ctx, [gemm(**dict(most, stride_c=1))], [zero]) == OK
    # (C behind A's start: inside what A's items span)
    assert run_epilogue(ctx, [gemm(**dict(most, stride_c=1, c=9 << 40))], [zero]) == ALIAS


def test_members_of_more_work_items_than_workgroups(ctx):
    """A launch holds fewer than 2^32 threads; members of more work items loop over them, by an index of 31 bits."""
    ints = [(ctypes.c_int32 * 1)() for _ in range(4)]
    limit = ((1 << 32) - 1) // 512
    for op, k in ((gdy.GEMM, 3), (gdy.ADD, 0)):
        def member(q, batch):
            return gemm(m=1, n=1, k=k, op=op, lda=3, ldb=1, ldc=1, batch=batch, stride_a=3, stride_b=0, stride_c=1,
                        a=(4 * q + 1) << 42, b=(4 * q + 2) << 42, c=(4 * q + 3) << 42)
        for count, batch in ((1, 100), (1, limit - 7), (1, 1 << 26), (2, 1 << 22), (2, 1 << 23), (16, 1 << 20)):
            g = (gdy.GemmDesc * count)(*[member(q, batch) for q in range(count)])
            items = (ctypes.c_int64 * count)()
            assert ctx.lib.gdy_dispatch_map(ctx.h, g, count, gdy.DEFAULT if count == 1 else gdy.GO, count, 0, 1, *ints,
                                            items) == OK, ctx.last_error()
            # grid, gemm_of_wg, first_item, item_stride of workgroup 0
            share = limit // count // 8 * 8
            assert items[0] == batch and ints[0][0] <= limit and ints[3][0] >= min(batch, share), (op, count, batch)
            assert ints[1][0] == 0 and ints[2][0] == 0
        for batch, want in (((1 << 31) - 1 - limit, OK), ((1 << 31) - limit, UNSUPPORTED), ((1 << 31) - 1, UNSUPPORTED)):
            g = (gdy.GemmDesc * 1)(member(0, batch))
            assert status(ctx, ctx.lib.gdy_execute, g, 1, gdy.SELECTOR, 0, None, None) == want
            assert run_epilogue(ctx, list(g), [gdy.EpilogueDesc()]) == want


def test_null_arguments(ctx):
    assert ctx.lib.gdy_execute_grouped(None, None, None, None) == INVALID
    assert ctx.lib.gdy_execute_grouped(ctx.h, None, None, None) == INVALID
    assert ctx.lib.gdy_execute_act_grad(None, None, None) == INVALID
    assert ctx.lib.gdy_execute_act_grad(ctx.h, None, None) == INVALID


# ---- the kernels' code -------------------------------------------------------------
def device_code(tmp_path, unit):
    """(disassembly, notes) of a unit's device code."""
    obj = os.path.join(waits.BUILD, unit + ".o")
    tools = [os.path.join(waits.LLVM, t) for t in ("llvm-objcopy", "clang-offload-bundler", "llvm-objdump", "llvm-readelf")]
    if not os.path.exists(obj) or not all(shutil.which(t) for t in tools):
        pytest.skip("no built kernel objects or LLVM tools")
    fat, dev = str(tmp_path / "fat"), str(tmp_path / "dev.o")
    subprocess.run([tools[0], f"--dump-section=.hip_fatbin={fat}", obj, os.devnull], check=True)
    subprocess.run([tools[1], "--unbundle", "--type=o", f"--input={fat}", f"--output={dev}",
                    "--targets=hipv4-amdgcn-amd-amdhsa--gfx950"], check=True)
    return [subprocess.run([tools[q], *args, dev], check=True, capture_output=True, text=True).stdout
            for q, args in ((2, ["-d", "--no-show-raw-insn"]), (3, ["--notes"]))]


def check_code(unit, text, notes):
    assert not re.search(r"\bv_pk_(add|mul|fma)_f32\b", text)
    scratch = [int(x) for x in re.findall(r"\.private_segment_fixed_size:\s*(\d+)", notes)]
    assert len(scratch) > 0 and set(scratch) == {0}, (unit, scratch)


@pytest.mark.parametrize("unit", [f"kernels_{f}_{dt}" for f in ("ep", "ep1", "group") for dt in ("bf16", "f16", "fp8", "f32")])
def test_wait_states_and_no_scratch(tmp_path, unit):
    """As test_copy_wait_states, for the kernels of epilogues and grouped products."""
    text, notes = device_code(tmp_path, unit)
    assert waits.check_copies(text) > 50
    check_code(unit, text, notes)


@pytest.mark.parametrize("unit", ["kernels_skinny", "kernels_act"])
def test_no_scratch(tmp_path, unit):
    """The kernels of few rows and of activation gradients, which copy nothing to LDS."""
    check_code(unit, *device_code(tmp_path, unit))
