"""Every kernel of the grouped products against 64-bit references, each at a size whose tile is
asserted: 256 x 256 tiles, whole and as halves, 128-row ones of the same kernel, and the smaller tiles
with operands by copies and by registers, for each type and layout, forward and backward."""
import pytest

import paper_2409_02227_amd  # noqa: F401  (sets GPU_MAX_HW_QUEUES before HIP starts)

torch = pytest.importorskip("torch")

from paper_2409_02227_amd import gdy  # noqa: E402
from tests.test_gpu_grouped import TABLE, OverK, Rows, run  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    c = gdy.Context(0, table=TABLE)
    yield c
    c.close()


K = 464  # whole 16-byte chunks of every type, no whole K tiles
# groups a row past whole tiles, empty, of whole tiles, of less than half a tile; rows of no group at both ends
SPLIT = (3, 1029, 0, 640, 257, 600)


def offsets(sizes):
    out = [sizes[0]]
    for s in sizes[1:]:
        out.append(out[-1] + s)
    return out


def halves(sizes, n, cus=256, xcds=8):
    """(whole 256 x 256 tiles, halved ones): each XCD's last ones are halved where they fill half its CUs at most."""
    total = sum(-(-s // 256) for s in sizes[1:]) * -(-n // 256)
    per = -(-total // xcds)
    rest = per % (cus // xcds)
    split = 2 * rest <= cus // xcds
    whole = sum(min(max(total - x * per, 0), per - rest if split else per) for x in range(xcds))
    return whole, total - whole


def check_rows(ctx, tile, *args, **kw):
    x = Rows(*args, **kw)
    assert ctx.grouped_tile(x.product) == tile, x.label
    run(ctx, x)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "fp8"])
@pytest.mark.parametrize("tb", [0, 1])
def test_whole_tiles_of_256_rows(ctx, dtype, tb):
    """No tile is halved: each writes its row of sums and a row of zeros."""
    assert halves(SPLIT, 4080) == (13 * 16, 0)
    check_rows(ctx, (256, 256), dtype, 2560, offsets(SPLIT), 4080, K, tb, ("gelu", "silu")[tb], bias=("groups", "shared")[tb],
               residual=True, aux=True, sums=("groups", "shared")[tb], scales=dtype == "fp8")


@pytest.mark.parametrize("dtype,tb,act", [("bf16", 1, "gelu"), ("f16", 0, "gelu_tanh"), ("fp8", 1, "silu"), ("bf16", 0, "relu")])
def test_whole_tiles_of_256_rows_backward(ctx, dtype, tb, act):
    check_rows(ctx, (256, 256), dtype, 2560, offsets(SPLIT), 4080, K, tb, act, grad=True, residual=tb == 0,
               sums=("shared", "groups")[tb], seed=1)


def test_whole_tiles_of_256_rows_linear(ctx):
    """Scales and a bias alone, which leave as plain tiles do."""
    check_rows(ctx, (256, 256), "fp8", 2560, offsets(SPLIT), 4080, K, 1, bias="groups", scales=True, seed=2)
    check_rows(ctx, (256, 256), "bf16", 2560, offsets(SPLIT), 4080, K, 0, seed=2)


@pytest.mark.parametrize("dtype,tb,grad", [("bf16", 0, False), ("f16", 1, True)])
def test_whole_and_halved_tiles_together(ctx, dtype, tb, grad):
    """(Rows of no group make the sizes that the host sees larger.)"""
    sizes = (5, 1100, 1, 0, 2000, 300, 129)
    whole, half = halves(sizes, 4080)
    assert whole >= 256 and half >= 16, (whole, half)
    check_rows(ctx, (256, 256), dtype, 5200, offsets(sizes), 4080, 208, tb, "silu", grad=grad, bias="groups", aux=not grad,
               sums="groups")


@pytest.mark.parametrize("dtype,tb", [("bf16", 1), ("f16", 0), ("fp8", 0)])
def test_halved_tiles(ctx, dtype, tb):
    """Most rows are in no group: few tiles, all of them halves, some with rows in the first alone."""
    sizes = (700, 128, 0, 257, 300, 4)
    whole, half = halves(sizes, 4080)
    assert whole == 0 and half == 6 * 16
    check_rows(ctx, (256, 256), dtype, 2560, offsets(sizes), 4080, K, tb, "gelu", residual=True, aux=True, sums="groups")


@pytest.mark.parametrize("dtype,tb,grad", [("bf16", 0, False), ("f16", 1, False), ("fp8", 1, False), ("fp8", 0, True),
                                           ("bf16", 1, True), ("f16", 0, True)])
def test_tiles_of_128_rows_on_the_wide_kernel(ctx, dtype, tb, grad):
    check_rows(ctx, (128, 256), dtype, 1500, offsets((0, 513, 129, 0, 128, 700)), 4080, K, tb, "gelu_tanh", grad=grad,
               bias="groups", residual=True, aux=not grad, sums=("groups", "shared")[tb], scales=dtype == "fp8")


SMALL = [("bf16", (128, 128), 800, 4080), ("bf16", (64, 128), 500, 4080), ("bf16", (32, 128), 400, 4080),
         ("bf16", (32, 64), 300, 496), ("f32", (128, 128), 1600, 2032), ("f32", (64, 128), 500, 3008),
         ("f32", (32, 128), 1600, 496), ("f32", (32, 64), 700, 496)]


@pytest.mark.parametrize("dtype,tile,rows,n", [(dt,) + s[1:] for s in SMALL for dt in
                                               (("bf16", "f16", "fp8") if s[0] == "bf16" else ("f32",))])
@pytest.mark.parametrize("tb", [0, 1])
@pytest.mark.parametrize("pad", [0, 1])
def test_smaller_tiles(ctx, dtype, tile, rows, n, tb, pad):
    """Copies (pad 0) and registers (pad 1), forward with sums by group and backward with shared ones."""
    q = rows // 8
    sizes = (2, 3 * q + 1, 0, 128 if rows > 400 else 64, q, rows - 2 - 4 * q - 1 - (128 if rows > 400 else 64) - 7)
    check_rows(ctx, tile, dtype, rows, offsets(sizes), n, K, tb, ("silu", "gelu")[pad], bias="groups", residual=True,
               aux=True, sums="groups", pad=pad, scales=dtype == "fp8")
    check_rows(ctx, tile, dtype, rows, offsets(sizes), n, K, tb, ("gelu_tanh", "relu")[tb], grad=True, sums="shared",
               pad=pad, seed=1)
    check_rows(ctx, tile, dtype, rows, offsets(sizes), n, K, tb, bias="shared", pad=pad, seed=2)


@pytest.mark.parametrize("dtype,tile,groups,k,n,pad", [
    ("bf16", 256, 7, 1520, 1264, 0), ("f16", 256, 7, 1520, 1264, 0), ("fp8", 256, 7, 1520, 1264, 16),
    ("bf16", 128, 4, 1040, 2032, 0), ("f16", 128, 4, 1040, 2032, 8), ("fp8", 128, 4, 1040, 2032, 0), ("f32", 128, 4, 1040, 2032, 0),
    ("bf16", 128, 4, 1041, 2031, 1), ("f16", 128, 4, 1041, 2031, 1), ("fp8", 128, 4, 1041, 2031, 1), ("f32", 128, 4, 1041, 2031, 1),
    ("bf16", 64, 4, 520, 784, 0), ("f16", 64, 4, 520, 784, 1), ("fp8", 64, 4, 528, 784, 0), ("fp8", 64, 4, 520, 783, 1),
    ("f32", 64, 4, 520, 784, 0)])
@pytest.mark.parametrize("residual", [None, "own", "c"])
def test_over_k(ctx, dtype, tile, groups, k, n, pad, residual):
    """One row, none, whole K tiles and a row past them in a group."""
    sizes = (6, 1, 0, 256, 129, 65, 0, 90)[:groups + 1]
    x = OverK(dtype, sum(sizes) + 9, offsets(sizes), k, n, residual, pad, scales=dtype == "fp8")
    assert ctx.grouped_tile(x.product) == (tile, tile), x.label
    run(ctx, x)


def test_tiles_of_nothing_and_refusals(ctx):
    x = Rows("bf16", 0, [0, 0, 0], 70, 64)
    assert ctx.grouped_tile(x.product) == (0, 0)
    d = x.product.descs()[0]
    d.trans_b = 2
    with pytest.raises(gdy.GdyError):
        ctx.grouped_tile(d)
