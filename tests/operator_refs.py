"""Plain 64-bit references of epilogues, grouped products and activation
gradients, and bounds on how far a kernel may be from them.

A bound counts, for C = round(f(z) + R) with z = scale * sum_k a b + bias:
* the rounding into C's type: half a step, eps / 2 of the value (fp16: at least
  half its smallest subnormal, 2^-25);
* the fp32 sum of K products in any order, (K + 4) * 2^-24 of S = sum |a b| +
  |bias|, times the largest slope of an activation (below 1.2);
* fp8 products: the matrix instruction aligns the products that it adds to the largest
  of them and drops what lies more than 13 bits below that one's leading bit (2^16 - 2^16
  + 2^s gives 2^s for s >= 3 and 0 below), so each of K products loses less than 2^-13
  of the largest: K * 2^-13 * max |a| max |b|;
* the activation in fp32, 2^-17 of its value and 2^-30: the exponential's argument
  reaches 20 in steps of 2^-24 and carries three roundings, 20 * 4 * 2^-24 < 2^-17;
  where it is larger the value is below 2^-30;
* a slope, whose terms are below 1.2: 2^-17 of the value it multiplies;
* one more fp32 rounding of every term that is added."""
import math

import torch

OUT = {"bf16": torch.bfloat16, "f16": torch.float16, "fp8": torch.bfloat16, "f32": torch.float32}
IN = {"bf16": torch.bfloat16, "f16": torch.float16, "fp8": torch.float8_e4m3fn, "f32": torch.float32}
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
EPS32 = 2.0 ** -24


def half_step(t):
    return torch.finfo(t).eps / 2


def tiny(t):
    return 2.0 ** -25 if t == torch.float16 else 2.0 ** -126


def value(z, act):
    if act == "relu":
        return torch.clamp(z, min=0.0)
    if act == "gelu":
        return z * torch.special.ndtr(z)
    if act == "gelu_tanh":
        return z * torch.sigmoid(math.sqrt(8 / math.pi) * (z + 0.044715 * z ** 3))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def slope(z, act):
    if act == "none":
        return torch.ones_like(z)
    if act == "relu":
        return (z > 0).to(z.dtype)
    z = z.clone().requires_grad_(True)  # of the definition above
    return torch.autograd.grad(value(z, act).sum(), z)[0]


def product(a, b, scale=1.0, bias=None, fp8=False):
    """(z, the error of its fp32 sum) of op(A) (m x k) and op(B) (k x n), in 64 bits."""
    a, b = a.double().cpu(), b.double().cpu()
    k = a.shape[1]
    z, s = a @ b * scale, a.abs() @ b.abs() * abs(scale)
    if bias is not None:
        z, s = z + bias.double().cpu(), s + bias.double().cpu().abs()
    err = (k + 4) * EPS32 * s
    if fp8 and k:
        err = err + k * 2.0 ** -13 * abs(scale) * a.abs().amax(1)[:, None] * b.abs().amax(0)[None, :]
    return z, err


class Expected:
    """What an epilogue gives for sums z that are off by err: C, its unrounded
    error, the written aux and the column sums, each with a bound."""

    def __init__(self, z, err, out_type, act="none", residual=None, aux=None, grad=False):
        self.aux, self.aux_bound = z, half_step(out_type) * z.abs() + 2 * err + tiny(out_type)
        if grad:
            f = z if act == "none" else z * slope(aux.double().cpu(), act)
            e = 1.2 * err + (2.0 ** -17 * z.abs() + 2.0 ** -30 if act != "none" else 0.0)
        else:
            f = value(z, act)
            e = 1.2 * err + (2.0 ** -17 * f.abs() + 2.0 ** -30 if act != "none" else 0.0)
        if residual is not None:
            r = residual.double().cpu()
            f, e = f + r, e + 2 * EPS32 * (f.abs() + r.abs())
        e = e + 2 * EPS32 * f.abs()
        self.c, self.raw_err = f, e
        self.c_bound = half_step(out_type) * f.abs() + (1 + half_step(out_type)) * e + tiny(out_type)

    def sums(self, rows=slice(None)):
        f, e = self.c[rows], self.raw_err[rows]
        return f.sum(0), e.sum(0) + (f.shape[0] + 4) * EPS32 * f.abs().sum(0)


def close(got, ref, bound, label):
    got = got.detach().double().cpu()
    bad = ~((got - ref).abs() <= bound)
    assert not bad.any(), (label, int(bad.sum()), bad.nonzero()[0].tolist(), got[bad][:3].tolist(),
                           ref[bad][:3].tolist(), bound[bad][:3].tolist() if torch.is_tensor(bound) else bound)


def padded(rows, cols, dtype, pad=0, fill=None, items=0, guard=2, device="cuda"):
    """(view rows x cols, whole buffer): rows `pad` elements longer, `guard` more rows
    behind the last, everything NaN (or `fill`)."""
    shape = (items, rows + guard, cols + pad) if items else (rows + guard, cols + pad)
    whole = torch.full(shape, float("nan") if fill is None else fill, dtype=dtype, device=device)
    return whole[..., :rows, :cols], whole


def untouched(view, whole, label):
    """Nothing was written outside the view (NaN before)."""
    mask = torch.zeros(whole.shape, dtype=torch.bool, device=whole.device)
    mask[..., :view.shape[-2], :view.shape[-1]] = True
    assert torch.isnan(whole.float()[~mask]).all().item(), f"{label}: wrote outside the output"


def operand(gen, rows, cols, dtype, pad=0, items=0, scale=1.0):
    """A matrix of the type on the GPU, rows padded with NaN."""
    shape = (items, rows, cols) if items else (rows, cols)
    x = (torch.rand(shape, generator=gen) * 2 - 1) * scale
    full = torch.full(shape[:-1] + (cols + pad,), float("nan"), dtype=torch.float32)
    full[..., :cols] = x
    return full.to(IN[dtype]).cuda()[..., :cols]
