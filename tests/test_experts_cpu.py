"""Routing, scatter, combine, quantisation and products of 8-bit integers without a GPU: the
binding's structures against the C compiler's, tensors that disagree, every refusal of the
library on a host-only context, and the kernels' code."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2409_02227_amd import gdy
from tests import test_copy_wait_states as waits
from tests.test_operators_cpu import check_code, device_code, status

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, UNSUPPORTED, ALIAS, TOO_MANY = 0, 1, 2, 3, 4
BF, I32, I8 = torch.bfloat16, torch.int32, torch.int8


@pytest.fixture(scope="module")
def ctx():
    c = gdy.Context(-1)
    yield c
    c.close()


def test_layouts_equal_the_c_compilers(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    structs = {"gdy_route": gdy.RouteDesc, "gdy_scatter": gdy.ScatterDesc, "gdy_combine": gdy.CombineDesc,
               "gdy_quantize": gdy.QuantizeDesc, "gdy_integer": gdy.IntegerDesc}
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "gdy.h"', "int main(void) {"]
    for cname, py in structs.items():
        lines.append(f'  printf("{cname} size %zu\\n", sizeof({cname}));')
        lines += [f'  printf("{cname} {f} %zu\\n", offsetof({cname}, {f}));' for f, _ in py._fields_]
    lines += ['  printf("const top_k %d\\n", GDY_MAX_TOP_K);', '  printf("const alone %d\\n", GDY_ROUTE_ALONE);',
              "  return 0;", "}"]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines) + "\n")
    exe = tmp_path / "layout"
    subprocess.run([cc, "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split("\n")
    got = {(a, b): int(c) for a, b, c in (l.split() for l in out if l)}
    assert got[("const", "top_k")] == gdy.MAX_TOP_K and got[("const", "alone")] == gdy.ROUTE_ALONE
    for cname, py in structs.items():
        assert got[(cname, "size")] == ctypes.sizeof(py), cname
        for f, _ in py._fields_:
            assert got[(cname, f)] == getattr(py, f).offset, (cname, f)


# ---- the binding --------------------------------------------------------------
def z(*shape, dtype=BF):
    return torch.zeros(*shape, dtype=dtype)


def test_route_shapes():
    d = gdy.Route(z(5, 3, dtype=torch.int64), z(5, 3, dtype=I32), z(9, dtype=I32)).desc()
    assert (d.tokens, d.top_k, d.experts, d.ld_ids, d.id_bytes) == (5, 3, 8, 3, 8)
    d = gdy.Route(z(5, 8, dtype=I32)[:, :2], z(5, 2, dtype=I32), z(1, dtype=I32)).desc()
    assert (d.tokens, d.top_k, d.experts, d.ld_ids, d.id_bytes) == (5, 2, 0, 8, 4)
    for bad in (gdy.Route(z(5, 3), z(5, 3, dtype=I32), z(9, dtype=I32)),
                gdy.Route(z(5, 3, dtype=I32), z(5, 2, dtype=I32), z(9, dtype=I32)),
                gdy.Route(z(5, 3, dtype=I32), z(5, 3, dtype=torch.int64), z(9, dtype=I32)),
                gdy.Route(z(5, 3, dtype=I32), z(5, 4, dtype=I32)[:, :3], z(9, dtype=I32)),
                gdy.Route(z(5, 3, dtype=I32), z(5, 3, dtype=I32), z(9, dtype=torch.int64)),
                gdy.Route(z(1, 3, dtype=I32).expand(5, 3), z(5, 3, dtype=I32), z(9, dtype=I32)),
                gdy.Route(z(5, dtype=I32), z(5, 1, dtype=I32), z(9, dtype=I32))):
        with pytest.raises(ValueError):
            bad.desc()


def test_scatter_and_combine_shapes():
    x, out, slots = z(5, 16), z(12, 20)[:, :16], z(5, 3, dtype=I32)
    w, dw = z(5, 3, dtype=torch.float32), z(5, 3, dtype=torch.float32)
    d = gdy.Scatter(x, slots, out, w, z(12, 16), dw).desc()
    assert (d.tokens, d.rows, d.n, d.top_k, d.type, d.ldx, d.ldo, d.ldz, d.weights_type) == \
        (5, 12, 16, 3, gdy.BF16, 16, 20, 16, gdy.F32)
    assert gdy.Scatter(x, slots, out, z(5, 3)).desc().weights_type == gdy.BF16
    f8 = z(5, 16, dtype=torch.float8_e4m3fn)
    assert gdy.Scatter(f8, slots, z(12, 16, dtype=torch.float8_e4m3fn)).desc().type == gdy.FP8_E4M3
    row = z(1, 16).expand(5, 16)
    for bad in (gdy.Scatter(x, slots[:4], out), gdy.Scatter(x, slots, z(12, 15)), gdy.Scatter(x, slots, out.float()),
                gdy.Scatter(x, slots, out, w[:, :2]), gdy.Scatter(x, slots, out, z(5, 3, dtype=torch.float16)),
                gdy.Scatter(x, slots, out, w, None, dw), gdy.Scatter(x, slots, out, w, out, None),
                gdy.Scatter(x, slots, out, None, z(12, 16), dw), gdy.Scatter(x, slots, out, w, z(11, 16), dw),
                gdy.Scatter(x, slots, out, w, z(12, 16), dw.bfloat16()), gdy.Scatter(row, slots, out),
                gdy.Scatter(x, slots, z(1, 16).expand(12, 16)), gdy.Scatter(x.int(), slots, out.int()),
                gdy.Scatter(x, slots.long(), out), gdy.Scatter(x, z(3, 5, dtype=I32).t(), out),
                gdy.Scatter(z(16, 5).t(), slots, out), gdy.Scatter(x.byte(), slots, out.byte())):
        with pytest.raises(ValueError):
            bad.desc()
    y = z(5, 24)[:, :16]
    d = gdy.Combine(out, slots, y, w, x).desc()
    assert (d.tokens, d.rows, d.n, d.top_k, d.ldy, d.ldz, d.ldr) == (5, 12, 16, 3, 24, 20, 16)
    for bad in (gdy.Combine(out, slots, y[:4]), gdy.Combine(z(12, 15), slots, y), gdy.Combine(out.float(), slots, y),
                gdy.Combine(out, slots, y, residual=x[:4]), gdy.Combine(out, slots, y, residual=x.float()),
                gdy.Combine(out, slots, y, residual=row), gdy.Combine(out, slots, y, w.t()),
                gdy.Combine(out, slots, row)):
        with pytest.raises(ValueError):
            bad.desc()


def test_quantize_shapes():
    x, q, s, slots = z(5, 16), z(5, 20, dtype=I8)[:, :16], z(5, dtype=torch.float32), z(5, 2, dtype=I32)
    d = gdy.Quantize(x, q, s).desc()
    assert (d.rows, d.n, d.top_k, d.out_rows, d.ldq, d.slots) == (5, 16, 0, 0, 20, None)
    d = gdy.Quantize(x, z(12, 16, dtype=I8), z(12, dtype=torch.float32), slots).desc()
    assert (d.top_k, d.out_rows) == (2, 12) and d.slots
    none = gdy.Quantize(x[:0], z(12, 16, dtype=I8), z(12, dtype=torch.float32), slots[:0]).desc()
    assert (none.rows, none.top_k, none.out_rows, none.slots) == (0, 0, 0, None)
    for bad in (gdy.Quantize(x, z(6, 16, dtype=I8), z(6, dtype=torch.float32)), gdy.Quantize(x, q.byte(), s),
                gdy.Quantize(x, q, s[:4]), gdy.Quantize(x, q, s.double()), gdy.Quantize(x, z(5, 15, dtype=I8), s),
                gdy.Quantize(x, q, s, slots[:4]), gdy.Quantize(x.int(), q, s)):
        with pytest.raises(ValueError):
            bad.desc()


def test_int8_shapes():
    a, b, c = z(10, 16, dtype=I8), z(8, 16, dtype=I8), z(10, 8)
    rs, cs, off = z(10, dtype=torch.float32), z(8, dtype=torch.float32), z(4, dtype=I32)
    d, e = gdy.Int8(a, b, c, rs, cs, trans_b=1, epilogue=gdy.Epilogue(z(8), "silu", z(10, 8))).descs()
    assert (d.rows, d.n, d.k, d.lda, d.ldb, d.ldc, d.trans_b, d.c_type, d.offsets) == (10, 8, 16, 16, 16, 8, 1, gdy.BF16, None)
    assert (e.act, e.ldr) == (gdy.ACT_SILU, 8)
    d, _ = gdy.Int8(a, z(3, 16, 8, dtype=I8), c.float(), rs, z(3, 8, dtype=torch.float32), off).descs()
    assert (d.groups, d.stride_b, d.stride_col_scales, d.ldb, d.c_type) == (3, 128, 8, 8, gdy.F32)
    assert gdy.Int8(a, z(3, 16, 8, dtype=I8), c, rs, cs, off).descs()[0].stride_col_scales == 0
    for bad in (gdy.Int8(a, b, c), gdy.Int8(a, b.byte(), c, trans_b=1), gdy.Int8(a.byte(), b, c, trans_b=1),
                gdy.Int8(a, b, c[:9], trans_b=1), gdy.Int8(a, b, c.double(), trans_b=1),
                gdy.Int8(a, b, c, rs[:9], trans_b=1), gdy.Int8(a, b, c, rs, cs.bfloat16(), trans_b=1),
                gdy.Int8(a, b, c, rs, z(16, dtype=torch.float32)[::2], trans_b=1), gdy.Int8(a, b, c, offsets=off, trans_b=1),
                gdy.Int8(a, b, c, rs, z(3, 8, dtype=torch.float32), trans_b=1),
                gdy.Int8(a, z(1, 16, dtype=I8).expand(8, 16), c, trans_b=1),
                gdy.Int8(a, z(2, 8, 16, dtype=I8), c, offsets=off, trans_b=1)):
        with pytest.raises(ValueError):
            bad.descs()


def test_tensors_of_another_device_and_streams(monkeypatch):
    """No operand of the host or of another device reaches the library; without a stream a call runs on
    the current stream of the context's device."""
    import types
    seen = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: seen.append((name, [a.value for a in args if isinstance(a, ctypes.c_void_p)])) or 0

    class Elsewhere:
        def __init__(self, t, at):
            self.t, self.at, self.device = t, at, f"cuda:{at}"

        def get_device(self):
            return self.at

        def __getattr__(self, name):
            return getattr(self.t, name)

        def __getitem__(self, i):
            return Elsewhere(self.t[i], self.at)

    monkeypatch.setattr(torch.cuda, "current_stream",
                        lambda device=None: types.SimpleNamespace(cuda_stream=100 + (0 if device is None else device)))
    ctx = object.__new__(gdy.Context)
    ctx.h, ctx.lib, ctx.device = None, Library(), 3
    f32 = torch.float32
    slots = z(5, 2, dtype=I32)
    calls = {"route": (gdy.Route, dict(ids=slots.clone(), slots=slots, offsets=z(5, dtype=I32))),
             "scatter": (gdy.Scatter, dict(x=z(5, 8), slots=slots, out=z(10, 8), weights=z(5, 2, dtype=f32), z=z(10, 8),
                                           weight_grad=z(5, 2, dtype=f32))),
             "combine": (gdy.Combine, dict(z=z(10, 8), slots=slots, y=z(5, 8), weights=z(5, 2, dtype=f32), residual=z(5, 8))),
             "quantize": (gdy.Quantize, dict(x=z(5, 8), q=z(10, 8, dtype=I8), scales=z(10, dtype=f32), slots=slots)),
             "int8": (gdy.Int8, dict(a=z(5, 8, dtype=I8), b=z(2, 8, 4, dtype=I8), c=z(5, 4), row_scales=z(5, dtype=f32),
                                     col_scales=z(4, dtype=f32), offsets=z(3, dtype=I32)))}
    for name, (cls, args) in calls.items():
        call = getattr(ctx, "execute_" + name)
        here = {k: Elsewhere(v, 3) for k, v in args.items()}
        call(cls(**here))
        call(cls(**here), stream=7)
        for change in args:
            for t in (args[change], Elsewhere(args[change], 0)):
                with pytest.raises(ValueError, match="cuda:3"):
                    call(cls(**dict(here, **{change: t})))
    here = {k: Elsewhere(v, 3) for k, v in calls["int8"][1].items()}
    for field in ("bias", "residual"):
        e = gdy.Epilogue(**{field: z(4) if field == "bias" else z(5, 4)})
        with pytest.raises(ValueError, match="cuda:3"):
            ctx.execute_int8(gdy.Int8(**here, epilogue=e))
    assert [n for n, _ in seen] == [f"gdy_execute_{n}" for n in ("route", "scatter", "combine", "quantize", "integer")
                                    for _ in range(2)]
    assert [v[-1] for _, v in seen] == [103, 7] * 5


# ---- the library's refusals -------------------------------------------------------
BASE = 1 << 32  # addresses that nothing reads on a host-only context


def at(i):
    return BASE + (i << 28)


def filled(d, base, kw):
    for k, v in dict(base, **kw).items():
        setattr(d, k, v)
    return d


ROUTE = dict(tokens=100, top_k=2, experts=16, ids=at(0), ld_ids=2, id_bytes=8, slots=at(1), offsets=at(2))


@pytest.mark.parametrize("kw,want", [
    ({}, OK), ({"tokens": -1}, INVALID), ({"experts": -1}, INVALID), ({"top_k": 0}, INVALID), ({"top_k": 65}, INVALID),
    ({"top_k": 64, "ld_ids": 64}, OK), ({"experts": 4097}, TOO_MANY), ({"experts": 4096}, OK), ({"experts": 0}, OK),
    ({"id_bytes": 4}, OK), ({"id_bytes": 2}, INVALID), ({"reserved": 1}, INVALID), ({"ld_ids": 1}, INVALID),
    ({"ld_ids": 1 << 44, "slots": 1 << 60, "offsets": 1 << 61}, OK), ({"ld_ids": (1 << 44) + 1}, INVALID),
    ({"ids": None}, INVALID), ({"slots": None}, INVALID), ({"offsets": None}, INVALID), ({"offsets": at(2) + 2}, INVALID),
    ({"slots": at(1) + 2}, INVALID), ({"ids": at(0) + 4}, INVALID), ({"ids": at(0) + 4, "id_bytes": 4}, OK),
    ({"tokens": 0, "ids": None, "slots": None}, OK), ({"tokens": 0, "offsets": None}, INVALID),
    ({"tokens": 1 << 23}, OK), ({"tokens": (1 << 23) + 1}, UNSUPPORTED), ({"tokens": (1 << 63) - 1}, UNSUPPORTED),
    ({"slots": at(0)}, ALIAS), ({"slots": at(0) + 1596}, ALIAS), ({"slots": at(0) + 1600}, OK),
    ({"offsets": at(1) + 796}, ALIAS), ({"offsets": at(0)}, ALIAS), ({"offsets": at(1) - 64}, ALIAS),
    ({"offsets": at(1) - 68}, OK),
])
def test_route_checks(ctx, kw, want):
    assert status(ctx, ctx.lib.gdy_execute_route, ctypes.byref(filled(gdy.RouteDesc(), ROUTE, kw)), None) == want


SCATTER = dict(tokens=100, rows=150, n=96, top_k=2, type=gdy.BF16, slots=at(0), x=at(1), ldx=96, weights=at(2),
               weights_type=gdy.F32, out=at(3), ldo=96, z=at(4), ldz=96, weight_grad=at(5))


@pytest.mark.parametrize("kw,want", [
    ({}, OK), ({"weights": None, "weight_grad": None}, OK), ({"weight_grad": None, "z": None}, OK),
    ({"tokens": -1}, INVALID), ({"rows": -1}, INVALID), ({"n": -1}, INVALID), ({"top_k": 0}, INVALID), ({"top_k": 65}, INVALID),
    ({"tokens": (1 << 31) - 4096}, UNSUPPORTED), ({"rows": 1 << 31}, UNSUPPORTED), ({"n": 1 << 29, "ldx": 1 << 29}, UNSUPPORTED),
    ({"type": gdy.FP8_E4M3}, UNSUPPORTED), ({"type": gdy.FP8_E4M3, "weights": None, "weight_grad": None}, OK),
    ({"type": 0}, UNSUPPORTED), ({"type": 5}, UNSUPPORTED), ({"reserved": 1}, INVALID), ({"weights": None}, INVALID),
    ({"weights_type": gdy.BF16}, OK), ({"weights_type": gdy.F16}, UNSUPPORTED), ({"weights": None, "weight_grad": None,
                                                                                 "weights_type": 9}, OK),
    ({"slots": None}, INVALID), ({"slots": at(0) + 2}, INVALID), ({"x": None}, INVALID), ({"out": None}, INVALID),
    ({"z": None}, INVALID), ({"ldx": 95}, INVALID), ({"ldo": 95}, INVALID), ({"ldz": 95}, INVALID),
    ({"ldx": 1 << 61}, INVALID), ({"ldo": (1 << 63) - 1}, INVALID), ({"ldz": 95, "weight_grad": None}, OK),
    ({"ldx": 1 << 44, "slots": 1 << 61, "weights": 2 << 61, "out": 3 << 61, "z": 4 << 61, "weight_grad": 5 << 61}, OK),
    ({"x": at(1) + 1}, UNSUPPORTED), ({"out": at(3) + 1}, UNSUPPORTED), ({"z": at(4) + 1}, UNSUPPORTED),
    ({"weights": at(2) + 2}, UNSUPPORTED), ({"weights": at(2) + 2, "weights_type": gdy.BF16}, OK),
    ({"weight_grad": at(5) + 2}, UNSUPPORTED),
    ({"out": at(1)}, ALIAS), ({"out": at(4)}, ALIAS), ({"out": at(0)}, ALIAS), ({"out": at(2)}, ALIAS),
    ({"out": at(5)}, ALIAS), ({"weight_grad": at(2)}, ALIAS), ({"weight_grad": at(1)}, ALIAS), ({"x": at(4)}, OK),
    ({"out": at(1) + 2 * 96 * 100 - 2}, ALIAS), ({"out": at(1) + 2 * 96 * 100}, OK),
    ({"tokens": 0, "slots": None, "x": None}, OK), ({"rows": 0, "x": None, "out": None, "z": None}, OK),
    ({"n": 0, "x": None, "out": None, "z": None}, OK), ({"n": 0, "slots": None}, INVALID),
])
def test_scatter_checks(ctx, kw, want):
    assert status(ctx, ctx.lib.gdy_execute_scatter, ctypes.byref(filled(gdy.ScatterDesc(), SCATTER, kw)), None) == want


COMBINE = dict(tokens=100, rows=150, n=96, top_k=2, type=gdy.BF16, slots=at(0), z=at(1), ldz=96, weights=at(2),
               weights_type=gdy.F32, residual=at(3), ldr=96, y=at(4), ldy=96)


@pytest.mark.parametrize("kw,want", [
    ({}, OK), ({"weights": None}, OK), ({"residual": None}, OK), ({"residual": at(4)}, OK),
    ({"residual": at(4), "ldr": 100}, ALIAS), ({"residual": at(4) + 2}, ALIAS), ({"residual": at(1)}, OK),
    ({"y": at(1)}, ALIAS), ({"y": at(0)}, ALIAS), ({"y": at(2)}, ALIAS),
    ({"tokens": -1}, INVALID), ({"rows": -1}, INVALID), ({"n": -1}, INVALID), ({"top_k": 0}, INVALID), ({"top_k": 65}, INVALID),
    ({"type": gdy.FP8_E4M3}, UNSUPPORTED), ({"type": 5}, UNSUPPORTED), ({"type": gdy.F32}, OK), ({"reserved": 2}, INVALID),
    ({"weights_type": gdy.F16}, UNSUPPORTED), ({"weights": at(2) + 2}, UNSUPPORTED), ({"slots": None}, INVALID),
    ({"slots": at(0) + 1}, INVALID), ({"z": None}, INVALID), ({"y": None}, INVALID), ({"z": None, "rows": 0}, OK),
    ({"ldz": 95}, INVALID), ({"ldr": 95}, INVALID), ({"ldy": 95}, INVALID), ({"ldy": 1 << 45}, INVALID),
    ({"ldr": 95, "residual": None}, OK), ({"ldz": 0, "rows": 0}, OK),
    ({"z": at(1) + 1}, UNSUPPORTED), ({"y": at(4) + 1}, UNSUPPORTED), ({"residual": at(3) + 1}, UNSUPPORTED),
    ({"tokens": 0, "slots": None, "y": None}, OK), ({"n": 0, "slots": None, "y": None}, OK),
    ({"tokens": 1 << 31}, UNSUPPORTED), ({"rows": (1 << 31) - 4096}, UNSUPPORTED),
])
def test_combine_checks(ctx, kw, want):
    assert status(ctx, ctx.lib.gdy_execute_combine, ctypes.byref(filled(gdy.CombineDesc(), COMBINE, kw)), None) == want


QUANTIZE = dict(rows=100, n=96, type=gdy.BF16, top_k=2, x=at(0), ldx=96, slots=at(1), out_rows=150, q=at(2), ldq=96,
                scales=at(3))
PLAIN = dict(slots=None, top_k=0, out_rows=0)


@pytest.mark.parametrize("kw,want", [
    ({}, OK), (PLAIN, OK), (dict(PLAIN, top_k=1), INVALID), (dict(PLAIN, out_rows=100), INVALID),
    ({"rows": -1}, INVALID), ({"n": -1}, INVALID), ({"out_rows": -1}, INVALID), ({"top_k": 0}, INVALID), ({"top_k": 65}, INVALID),
    ({"type": gdy.FP8_E4M3}, UNSUPPORTED), ({"type": gdy.F32}, OK), ({"type": 6}, UNSUPPORTED),
    ({"x": None}, INVALID), ({"q": None}, INVALID), ({"scales": None}, INVALID), ({"scales": at(3) + 2}, INVALID),
    ({"slots": at(1) + 2}, INVALID), ({"ldx": 95}, INVALID), ({"ldq": 95}, INVALID), ({"ldq": 1 << 45}, INVALID),
    ({"x": at(0) + 1}, UNSUPPORTED), ({"q": at(2) + 1}, OK),
    ({"q": at(0)}, ALIAS), ({"q": at(1)}, ALIAS), ({"q": at(3)}, ALIAS), ({"scales": at(0)}, ALIAS), ({"scales": at(1)}, ALIAS),
    ({"scales": at(2) + 96 * 150 - 4}, ALIAS), ({"scales": at(2) + 96 * 150}, OK),
    (dict(PLAIN, scales=at(2) + 96 * 100), OK), ({"rows": 0, "x": None, "q": None, "scales": None}, OK),
    ({"out_rows": 0, "q": None, "scales": None}, OK), ({"n": 0, "x": None, "q": None}, OK),
    ({"rows": (1 << 31) - 4096}, UNSUPPORTED), ({"out_rows": 1 << 31}, UNSUPPORTED), ({"n": 1 << 28, "ldx": 1 << 28}, UNSUPPORTED),
])
def test_quantize_checks(ctx, kw, want):
    assert status(ctx, ctx.lib.gdy_execute_quantize, ctypes.byref(filled(gdy.QuantizeDesc(), QUANTIZE, kw)), None) == want


# Rows of 2^40 bytes: offsets of 2^23 of them end below 2^63, of one more at 2^63 and past it.  The second of two rows
# of 2^44 elements lies inside 64 bits whatever the type.
LAST, PAST = 1 << 23, (1 << 23) + 1


@pytest.mark.parametrize("op,kw,want", [
    ("route", {"tokens": 1 << 20, "ld_ids": 1 << 40}, OK),
    ("route", {"tokens": (1 << 20) + 1, "ld_ids": 1 << 40}, UNSUPPORTED),
    ("route", {"tokens": (1 << 20) + 1, "ld_ids": 1 << 40, "id_bytes": 4}, OK),
    ("route", {"tokens": 1 << 23, "ld_ids": 1 << 44}, UNSUPPORTED),
    ("scatter", {"tokens": LAST, "ldx": 1 << 39}, OK), ("scatter", {"tokens": PAST, "ldx": 1 << 39}, UNSUPPORTED),
    ("scatter", {"rows": LAST, "ldo": 1 << 39}, OK), ("scatter", {"rows": PAST, "ldo": 1 << 39}, UNSUPPORTED),
    ("scatter", {"rows": LAST, "ldz": 1 << 39}, OK), ("scatter", {"rows": PAST, "ldz": 1 << 39}, UNSUPPORTED),
    ("scatter", {"rows": PAST, "ldz": 1 << 39, "z": None, "weight_grad": None}, OK),
    ("scatter", {"tokens": PAST, "ldx": 1 << 38, "type": gdy.F32}, UNSUPPORTED),
    ("scatter", {"tokens": (1 << 31) - 4097, "top_k": 1, "ldx": 1 << 44}, UNSUPPORTED), ("scatter", {"tokens": 2, "ldx": 1 << 44}, OK),
    ("combine", {"tokens": LAST, "ldy": 1 << 39}, OK), ("combine", {"tokens": PAST, "ldy": 1 << 39}, UNSUPPORTED),
    ("combine", {"rows": LAST, "ldz": 1 << 39}, OK), ("combine", {"rows": PAST, "ldz": 1 << 39}, UNSUPPORTED),
    ("combine", {"tokens": LAST, "ldr": 1 << 39}, OK), ("combine", {"tokens": PAST, "ldr": 1 << 39}, UNSUPPORTED),
    ("combine", {"tokens": PAST, "ldr": 1 << 39, "residual": None}, OK), ("combine", {"rows": 0, "ldz": 1 << 62}, OK),
    ("quantize", {"rows": LAST, "ldx": 1 << 39}, OK), ("quantize", {"rows": PAST, "ldx": 1 << 39}, UNSUPPORTED),
    ("quantize", {"out_rows": LAST, "ldq": 1 << 40}, OK), ("quantize", {"out_rows": PAST, "ldq": 1 << 40}, UNSUPPORTED),
    ("quantize", dict(PLAIN, rows=PAST, ldq=1 << 40), UNSUPPORTED), ("quantize", {"rows": PAST, "ldx": 1 << 39, "n": 0}, OK),
])
def test_matrices_past_64_bit_offsets(ctx, op, kw, want):
    """Where the last row's byte offset would not fit a signed 64-bit product the call is refused, however few of the
    rows are named."""
    base, struct = {"route": (ROUTE, gdy.RouteDesc), "scatter": (SCATTER, gdy.ScatterDesc), "combine": (COMBINE, gdy.CombineDesc),
                    "quantize": (QUANTIZE, gdy.QuantizeDesc)}[op]
    d = filled(struct(), base, kw)
    far = {"ldx": "x", "ldo": "out", "ldz": "z", "ldy": "y", "ldr": "residual", "ldq": "q", "ld_ids": "ids"}
    apart = [name for ld, name in far.items() if ld in kw]
    for i, (name, kind) in enumerate(struct._fields_):  # 2^40 bytes for each operand, the one with rows far apart last
        if kind is ctypes.c_void_p and getattr(d, name):
            setattr(d, name, 1 << 50 if name in apart else (i + 1) << 40)
    assert status(ctx, getattr(ctx.lib, "gdy_execute_" + op), ctypes.byref(d), None) == want


INTEGER = dict(rows=64, n=96, k=128, c_type=gdy.BF16, trans_b=0, groups=4, offsets=at(0), a=at(1), lda=128, b=at(2), ldb=96,
               stride_b=128 * 96, row_scales=at(3), col_scales=at(4), stride_col_scales=96, c=at(5), ldc=96)
DENSE = dict(offsets=None, groups=0, stride_b=0, stride_col_scales=0)
BIAS = dict(act=gdy.ACT_SILU, bias=at(6), bias_type=gdy.F32, stride_bias=96, residual=at(7), ldr=96)


@pytest.mark.parametrize("kw,ep,want", [
    ({}, None, OK), (DENSE, None, OK), ({}, {}, OK), (DENSE, {}, OK), (dict(DENSE, groups=-5, stride_b=-1), None, OK),  # ignored
    ({"rows": -1}, None, INVALID), ({"n": -1}, None, INVALID), ({"k": -1}, None, INVALID), ({"groups": -1}, None, INVALID),
    ({"groups": 4097}, None, TOO_MANY), ({"groups": 4096}, None, OK), ({"groups": 0}, None, OK),
    ({"c_type": gdy.F16}, None, OK), ({"c_type": gdy.F32}, None, OK), ({"c_type": gdy.FP8_E4M3}, None, UNSUPPORTED),
    ({"c_type": 5}, None, UNSUPPORTED), ({"trans_b": 2}, None, INVALID), ({"trans_b": 1, "ldb": 128}, None, OK),
    ({"trans_b": 1, "ldb": 127}, None, INVALID), ({"reserved": 1}, None, INVALID),
    ({"k": 131071, "lda": 131071}, None, OK), ({"k": 131072, "lda": 131072}, None, UNSUPPORTED),
    ({"offsets": at(0) + 2}, None, INVALID), ({"row_scales": at(3) + 2}, None, INVALID),
    ({"col_scales": at(4) + 1}, None, INVALID), ({"row_scales": None, "col_scales": None}, None, OK),
    ({"a": None}, None, INVALID), ({"b": None}, None, INVALID), ({"c": None}, None, INVALID), ({"lda": 127}, None, INVALID),
    ({"ldb": 95}, None, INVALID), ({"ldc": 95}, None, INVALID), ({"a": at(1) + 1, "b": at(2) + 3}, None, OK),
    ({"c": at(5) + 1}, None, UNSUPPORTED), ({"stride_b": -1}, None, INVALID), ({"stride_b": 0}, None, OK),
    ({"stride_b": 1 << 45}, None, UNSUPPORTED), ({"stride_col_scales": 0}, None, OK), ({"stride_col_scales": 95}, None, INVALID),
    ({"stride_col_scales": -96}, None, INVALID), ({"stride_col_scales": 1 << 45}, None, UNSUPPORTED),
    ({"col_scales": None, "stride_col_scales": 5}, None, OK),
    ({"c": at(1)}, None, ALIAS), ({"c": at(2)}, None, ALIAS), ({"c": at(2) + 4 * 128 * 96 - 2}, None, ALIAS),
    ({"c": at(2) + 4 * 128 * 96}, None, OK), ({"c": at(3)}, None, ALIAS), ({"c": at(4) + 4 * 3 * 96}, None, ALIAS),
    ({"c": at(0)}, None, ALIAS), ({"k": 0, "a": None, "b": None}, None, OK), ({"n": 0, "c": None}, None, OK),
    ({"rows": 0, "c": None}, None, OK), ({"rows": (1 << 31) - 4096, "a": 1 << 40}, None, UNSUPPORTED),
    ({"rows": 1 << 25, "a": 1 << 42, "c": 1 << 43, "row_scales": 1 << 44}, None, OK), ({"lda": 1 << 23}, None, UNSUPPORTED),
    ({"ldb": 1 << 24, "b": 1 << 45}, None, UNSUPPORTED), ({"ldc": 1 << 22}, None, UNSUPPORTED),
    ({"lda": (1 << 63) - 1}, None, UNSUPPORTED), ({"ldc": (1 << 63) - 1}, None, UNSUPPORTED),
    # epilogues: forward, without saved values
    ({}, {"grad": 1}, UNSUPPORTED), ({}, {"aux": at(8), "ldaux": 96}, UNSUPPORTED), ({}, {"bias_grad": at(8)}, UNSUPPORTED),
    ({}, {"act": 5}, INVALID), ({}, {"bias_type": gdy.F16}, UNSUPPORTED), ({}, {"bias_type": gdy.BF16}, OK),
    ({}, {"ldr": 95}, INVALID), ({}, {"stride_bias": -1}, INVALID), ({}, {"residual": at(5)}, OK),
    ({}, {"residual": at(5), "ldr": 100}, ALIAS), ({}, {"bias": at(5)}, ALIAS), ({}, {"ldr": 1 << 23}, UNSUPPORTED),
    ({}, {"reserved": 1}, INVALID), ({}, {"residual": at(7) + 1}, UNSUPPORTED),
])
def test_integer_checks(ctx, kw, ep, want):
    e = None if ep is None else ctypes.byref(filled(gdy.EpilogueDesc(), BIAS, ep))
    assert status(ctx, ctx.lib.gdy_execute_integer, ctypes.byref(filled(gdy.IntegerDesc(), INTEGER, kw)), e, None) == want


def test_null_arguments(ctx):
    for name in ("route", "scatter", "combine", "quantize"):
        fn = getattr(ctx.lib, "gdy_execute_" + name)
        assert fn(None, None, None) == INVALID and fn(ctx.h, None, None) == INVALID
    assert ctx.lib.gdy_execute_integer(None, None, None, None) == INVALID
    assert ctx.lib.gdy_execute_integer(ctx.h, None, None, None) == INVALID


# ---- the kernels' code -------------------------------------------------------------
@pytest.mark.parametrize("unit", [f"kernels_integer_{dt}" for dt in ("bf16", "f16", "f32")])
def test_wait_states_and_no_scratch(tmp_path, unit):
    text, notes = device_code(tmp_path, unit)
    assert waits.check_copies(text) > 50
    check_code(unit, text, notes)


@pytest.mark.parametrize("unit", ["kernels_experts", "kernels_quantize"])
def test_no_scratch(tmp_path, unit):
    check_code(unit, *device_code(tmp_path, unit))


def test_integer_tile(ctx):
    tile = lambda kw: ctx.int8_tile(filled(gdy.IntegerDesc(), INTEGER, kw))  # noqa: E731
    big = dict(DENSE, rows=8192, n=8192, k=8192, lda=8192, ldb=8192, ldc=8192, a=1 << 42, b=1 << 43, c=1 << 44)
    assert tile(big) == (256, 256)
    assert tile(dict(big, a=(1 << 42) + 1)) == (128, 128)  # operands that take no copies
    assert tile(dict(DENSE, rows=1, k=2048, lda=2048, trans_b=1, ldb=2048)) == (16, 16)
    assert tile({}) == (32, 64)
    for nothing in ({"groups": 0}, {"rows": 0}, {"n": 0}):
        assert tile(nothing) == (0, 0)
    with pytest.raises(gdy.GdyError):
        tile({"k": -1})
    r, c, d = ctypes.c_int32(), ctypes.c_int32(), filled(gdy.IntegerDesc(), INTEGER, {})
    r, c, d = ctypes.byref(r), ctypes.byref(c), ctypes.byref(d)
    fn = ctx.lib.gdy_integer_tile
    assert fn(None, d, r, c) == INVALID and fn(ctx.h, None, r, c) == INVALID
    assert fn(ctx.h, d, None, c) == INVALID and fn(ctx.h, d, r, None) == INVALID
