"""Submissions of so many small items that a workgroup for each would pass the 2^32 threads
of a launch."""
import pytest

import paper_2409_02227_amd  # noqa: F401  (sets GPU_MAX_HW_QUEUES before HIP starts)

torch = pytest.importorskip("torch")

from paper_2409_02227_amd import gdy  # noqa: E402
from tests.test_gpu_epilogue import TABLE  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    c = gdy.Context(0, table=TABLE)
    yield c
    c.close()


def descriptors(count):
    return (gdy.GemmDesc * count)(), (gdy.EpilogueDesc * count)()


def test_zero_sums_of_more_items_than_workgroups(ctx):
    """Members without rows: (2^24 + 5) items of one column (256 threads each), and beside them a few of 70
    columns, whose sums are zeros; what lies around stays."""
    items = (1 << 24) + 5
    out = torch.full((items + 2,), 7.0, device="cuda")
    few = torch.full((3, 72), 7.0, device="cuda")
    g, e = descriptors(2)
    for x, n, batch in ((g[0], 1, items), (g[1], 70, 3)):
        x.m, x.n, x.k, x.batch, x.stride_c = 0, n, 8, batch, n
        x.a_type = x.b_type = x.c_type = gdy.BF16
        x.scale_a = x.scale_b = 1.0
    e[0].bias_grad, e[0].stride_bias_grad = out[1:].data_ptr(), 1
    e[1].bias_grad, e[1].stride_bias_grad = few.data_ptr(), 72
    ctx.execute_descs(g, 2, gdy.SELECTOR, 0, None, e)
    torch.cuda.synchronize()
    assert float(out[0]) == 7.0 and float(out[-1]) == 7.0
    assert int(torch.count_nonzero(out[1:-1])) == 0
    assert int(torch.count_nonzero(few[:, :70])) == 0 and bool((few[:, 70:] == 7.0).all())


def small(gen, *shape):
    """Whole numbers whose sums here are exact in bf16."""
    return torch.randint(-2, 3, shape, generator=gen, device="cuda").to(torch.bfloat16)


GRID = ((1 << 32) - 1) // 512  # workgroups of 512 threads


@pytest.mark.parametrize("layout", ["nt", "nn"])
@pytest.mark.parametrize("members", [1, 2])
def test_few_rows_of_more_items_than_workgroups(ctx, layout, members):
    """Single tokens against a shared weight: a column tile each."""
    gen = torch.Generator("cuda").manual_seed(members)
    n, k, items = 16 if layout == "nt" else 64, 8, GRID // members + 9
    gemms, want = [], []
    for _ in range(members):
        a, b, bias = small(gen, items, 1, k), small(gen, k, n), small(gen, n)
        c = torch.full((items, 1, n), float("nan"), dtype=torch.bfloat16, device="cuda")
        want.append(torch.relu((a.view(items, k).float() @ b.float() + bias.float())).to(torch.bfloat16).view(items, 1, n))
        gemms.append(gdy.Gemm(a, b.t().contiguous() if layout == "nt" else b, c, trans_b=int(layout == "nt"),
                              epilogue=gdy.Epilogue(bias, "relu")))
    ctx.execute(gemms)
    torch.cuda.synchronize()
    for g, w in zip(gemms, want):
        assert torch.equal(g.c, w)


@pytest.mark.parametrize("kind", ["plain", "epilogue", "add"])
def test_tiles_of_more_items_than_workgroups(ctx, kind):
    """1 x 1 items of unaligned operands, a tile each, as many as 2^32 threads at 256 a workgroup."""
    gen = torch.Generator("cuda").manual_seed(3)
    items = (1 << 24) + 9
    c = torch.full((items, 1, 1), float("nan"), dtype=torch.bfloat16, device="cuda")
    if kind == "add":
        a, b = small(gen, items, 1, 1), small(gen, items, 1, 1)
        ctx.execute([gdy.Add(a, b, c)])
        want = a + b
    else:
        a, b, bias = small(gen, items, 1, 3), small(gen, 3, 1), small(gen, 1)
        ctx.execute([gdy.Gemm(a, b, c, epilogue=gdy.Epilogue(bias, "relu") if kind == "epilogue" else None)])
        want = a.view(items, 3).float() @ b.float()
        if kind == "epilogue":
            want = torch.relu(want + bias.float())
        want = want.to(torch.bfloat16).view(items, 1, 1)
    torch.cuda.synchronize()
    assert torch.equal(c, want)
