"""Cases of the operators around a linear layer: GEMMs with an epilogue (bias,
activation, residual, saved pre-activation, activation and bias gradients),
products grouped by expert with row counts that only the device knows, and
the activation and bias gradient that no product precedes.

A case is a dict of plain values.

"op": "linear".  X is m x k, the weight k x n ("nn") or n x k ("nt").
  Forward: z = X W + bias, y = act(z) + residual, z kept where "aux".
  "backward": from dY (m x n), the weight, the pre-activation Z (m x k) that
  X = act(Z) came from, and X: dZ = (dY W^T) * act'(Z), its column sums, and
  dW = X^T dY, as one submission.  "batch" > 1: that many of them, strided.
"op": "experts".  The same over rows sorted by expert; "rows" of them belong
  to the "groups" experts, "tail" further rows to none.  "skew": how uneven
  the experts are, "holes": every third expert has no row.
"op": "act_grad".  dz = dy * act'(z) and its column sums, per group where
  "groups" > 0.
"pad" widens every row pitch by that many elements; "dtype" is the input type.
"""
import functools
import math
import os
import random

import torch

own = False

TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "fp8": torch.float8_e4m3fn, "f32": torch.float32}
OUT = {"bf16": torch.bfloat16, "f16": torch.float16, "fp8": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "fp8": 1, "f32": 4}
OUT_SIZE = {"bf16": 2, "f16": 2, "fp8": 2, "f32": 4}


def linear(name, dtype, m, n, k, layout="nn", act="none", bias=True, residual=False, aux=False, backward=False,
           batch=0, pad=0):
    return {"name": name, "op": "linear", "dtype": dtype, "m": m, "n": n, "k": k, "layout": layout, "act": act,
            "bias": bias, "residual": residual, "aux": aux, "backward": backward, "batch": batch, "pad": pad}


def experts(name, dtype, rows, groups, n, k, layout="nn", act="none", bias=False, aux=False, backward=False,
            skew=0.5, holes=False, tail=0, pad=0):
    return {"name": name, "op": "experts", "dtype": dtype, "rows": rows, "groups": groups, "n": n, "k": k,
            "layout": layout, "act": act, "bias": bias, "aux": aux, "backward": backward, "skew": skew,
            "holes": holes, "tail": tail, "pad": pad}


def act_grad(name, dtype, rows, n, act, groups=0, skew=0.5, holes=False, tail=0, pad=0):
    return {"name": name, "op": "act_grad", "dtype": dtype, "rows": rows, "n": n, "act": act, "groups": groups,
            "skew": skew, "holes": holes, "tail": tail, "pad": pad}


def listed():
    return [
        # one token through one linear layer: what a call costs, and a weight read once
        linear("linear_token_bf16", "bf16", 1, 2048, 2048, "nt", "silu"),
        # the FFN's first product in a tensor-sliced layer's training forward pass, z kept
        linear("linear_ffn_up_bf16", "bf16", 512, 6144, 12288, "nn", "gelu_tanh", aux=True),
        # the FFN's second product over a long prompt, onto the residual stream
        linear("linear_ffn_down_bf16", "bf16", 8192, 4096, 8192, "nt", residual=True),
        # backward through a linear layer and the activation before it, 2048 tokens
        linear("linear_backward_bf16", "bf16", 2048, 4096, 4096, "nn", "gelu", backward=True),
        # sizes that nothing divides, rows packed without any alignment
        linear("linear_odd_f16", "f16", 509, 2047, 1021, "nn", "relu", residual=True),
        # a decoding step: 32 sequences, two experts each
        experts("experts_decode_bf16", "bf16", 64, 16, 2048, 2048, "nt", "silu", skew=0.5),
        # a prompt through the experts' first product, training forward
        experts("experts_prefill_bf16", "bf16", 8192, 16, 4096, 2048, "nn", "gelu_tanh", bias=True, aux=True),
        # backward of the experts' products: input and weight gradients, bias gradients
        experts("experts_backward_bf16", "bf16", 8192, 8, 2048, 4096, "nn", "silu", backward=True, skew=1.0),
        # serving in fp8, a weight scale for each expert
        experts("experts_fp8", "fp8", 4096, 32, 4096, 4096, "nt", "silu", skew=0.8),
        # few rows, experts without any, odd sizes, rows of no expert behind the last
        experts("experts_ragged_f16", "f16", 777, 9, 1001, 515, "nn", "relu", bias=True, holes=True, tail=19),
        # backward through an activation that no product precedes, and the bias below it
        act_grad("act_grad_bf16", "bf16", 8192, 4096, "gelu"),
        # bias gradients of experts, full precision
        act_grad("act_grad_experts_f32", "f32", 2900, 1536, "silu", groups=16, tail=100),
    ]


def spread(rng, lo, hi, step=1):
    """A size between lo and hi, even over its logarithm, on multiples of step."""
    x = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(int(round(x / step)) * step, step)


MOST = 5e11  # flops of a drawn case, below the largest listed one's
MOST_BYTES = 4e8


def draw(rng):
    while True:
        c = draw_any(rng)
        w = work(c)
        if w["flops"] <= MOST / (6 if c["dtype"] == "f32" else 1) and w["bytes"] <= MOST_BYTES:
            return c


def draw_any(rng):
    kind = rng.choice(["linear", "linear", "linear_backward", "experts", "experts", "experts_backward", "act_grad"])
    pad = rng.choice([0, 0, 0, 16])
    acts = ["none", "relu", "gelu", "gelu_tanh", "silu"]
    step = rng.choice([256, 64, 64, 8, 1])
    if step == 1:
        pad = 0
    if kind == "act_grad":
        groups = rng.choice([0, 0, 1, 8, 64])
        return act_grad(None, rng.choice(["bf16", "f16", "f32"]), spread(rng, 1, 16384), spread(rng, 64, 8192, step),
                        rng.choice(acts), groups, rng.choice([0.0, 0.5, 1.5]), groups > 3 and rng.random() < 0.3,
                        rng.choice([0, 0, 37]) if groups else 0, pad)
    size = 1500 if step == 1 else 16384
    n, k = spread(rng, 64, size, step), spread(rng, 64, size, step)
    layout, act = rng.choice(["nn", "nt"]), rng.choice(acts)
    if kind.startswith("linear"):
        back = kind == "linear_backward"
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"] if back else ["bf16", "bf16", "f16", "fp8", "f32"])
        batch = rng.choice([0, 0, 0, 3]) if not back else 0
        return linear(None, dtype, spread(rng, 1, 8192), n, k, layout, act, rng.random() < 0.7,
                      not back and rng.random() < 0.4, not back and rng.random() < 0.3, back, batch, pad)
    back = kind == "experts_backward"
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"] if back else ["bf16", "bf16", "f16", "fp8", "f32"])
    groups = rng.choice([1, 4, 8, 16, 60, 128])
    top = 4096 if step > 1 else size
    n, k = min(n, top), min(k, top)
    return experts(None, dtype, spread(rng, 1, 16384), groups, n, k, layout, act, rng.random() < 0.4,
                   not back and rng.random() < 0.3, back, rng.choice([0.0, 0.5, 1.5]),
                   groups > 3 and rng.random() < 0.3, rng.choice([0, 0, 37]), pad)


def counts(c):
    """Rows of each expert: a power law over them, every third one empty where
    the case has holes, whole rows by largest remainder.  From the case alone."""
    e = c["groups"]
    w = [0.0 if c["holes"] and i % 3 == 1 else (i + 1.0) ** -c["skew"] for i in range(e)]
    total = sum(w)
    share = [c["rows"] * x / total for x in w]
    out = [int(s) for s in share]
    order = sorted(range(e), key=lambda i: out[i] - share[i])
    for i in order[:c["rows"] - sum(out)]:
        out[i] += 1
    return out


def placed_counts(c, seed):
    """The experts' counts in an order that the seed gives."""
    out = counts(c)
    random.Random(seed).shuffle(out)
    return out


# ---- inputs ------------------------------------------------------------------
def tensor(gen, c, shape, kind, dtype=None):
    """A matrix (or strided batch) with padded rows.  Activations and gradients
    are uniform in [-1, 1], weights normal with deviation 1 / sqrt(k) so that z is
    of the size that activations see, pre-activations normal, fp8 codes uniform."""
    dtype = dtype or c["dtype"]
    shape = shape[:-1] + (shape[-1] + c["pad"],)
    if dtype == "fp8":
        x = (torch.rand(shape, generator=gen, device="cuda") * 2 - 1) * 448.0
    elif kind == "weight":
        x = torch.randn(shape, generator=gen, device="cuda") * (2.0 / math.sqrt(c["k"]))
    elif kind == "pre":
        x = torch.randn(shape, generator=gen, device="cuda") * 1.5
    else:
        x = torch.rand(shape, generator=gen, device="cuda") * 2 - 1
    return x.to(TORCH[dtype])[..., :shape[-1] - c["pad"]]


def inputs(c, seed):
    """What a program has in hand, from the seed alone."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    out = {}
    ctype = "bf16" if c["dtype"] == "fp8" else c["dtype"]
    if c["op"] == "act_grad":
        total = c["rows"] + c["tail"]
        out["dy"] = tensor(gen, c, (total, c["n"]), "act")
        out["z"] = tensor(gen, c, (total, c["n"]), "pre") if c["act"] != "none" else None
        if c["groups"]:
            out["counts"] = placed_counts(c, seed)
        return out
    n, k = c["n"], c["k"]
    grouped = c["op"] == "experts"
    if grouped:
        out["counts"] = placed_counts(c, seed)
        m, items = c["rows"] + c["tail"], (c["groups"],)
        lead = ()
    else:
        m = c["m"]
        items = lead = (c["batch"],) if c["batch"] else ()
    out["w"] = tensor(gen, c, items + ((k, n) if c["layout"] == "nn" else (n, k)), "weight")
    out["x"] = tensor(gen, c, lead + (m, k), "act")
    if c["backward"]:
        out["dy"] = tensor(gen, c, lead + (m, n), "act")
        out["z"] = tensor(gen, c, lead + (m, k), "pre")
    else:
        rand = torch.randn((c["groups"], n) if grouped else (n,), generator=gen, device="cuda")
        out["bias"] = rand.to(TORCH[ctype]) if c["bias"] else None
        out["residual"] = tensor(gen, c, lead + (m, n), "act", ctype) if c.get("residual") else None
    # fp8 scales: codes up to 448 stand for activations up to 1 and weights up to 2 / sqrt(k)
    out["scale_x"], out["scale_w"] = 1.0, 1.0
    if c["dtype"] == "fp8":
        out["scale_x"] = float(torch.tensor(1.0 / 448, dtype=torch.float32))
        out["scale_w"] = float(torch.tensor(3.5 / math.sqrt(k) / 448, dtype=torch.float32))
        if grouped:
            out["scales"] = torch.rand(c["groups"], generator=gen, device="cuda") + 0.5
    return out


@functools.lru_cache(maxsize=1)
def context():
    """The handle a program creates once and keeps."""
    from paper_2409_02227_amd import gdy
    table = os.path.join(os.path.dirname(os.path.abspath(gdy.__file__)), "tables", "gfx950.table")
    return gdy.Context(0, table=table)


def empty(c, shape, fp32=False):
    """An output buffer with the case's row pitch.  Zeros: rows of no expert stay so."""
    dtype = torch.float32 if fp32 else OUT[c["dtype"]]
    return torch.zeros(shape[:-1] + (shape[-1] + c["pad"],), dtype=dtype, device="cuda")[..., :shape[-1]]


def prepare(c, seed):
    x = inputs(c, seed)
    s = {"case": c, "in": x, "offsets": None}
    if "counts" in x:
        off = [0]
        for q in x["counts"]:
            off.append(off[-1] + q)
        s["bounds"] = list(zip(off[:-1], off[1:]))
        s["offsets"] = torch.tensor(off, dtype=torch.int32, device="cuda")
    if c["op"] == "act_grad":
        s["dz"] = empty(c, tuple(x["dy"].shape))
        s["db"] = torch.zeros((c["groups"], c["n"]) if c["groups"] else (c["n"],), device="cuda")
    elif c["backward"]:
        s["dz"] = empty(c, tuple(x["x"].shape))
        s["dw"] = empty(c, tuple(x["w"].shape))
        s["db"] = torch.zeros(((c["groups"],) if c["op"] == "experts" else ()) + (c["k"],), device="cuda")
    else:
        shape = tuple(x["x"].shape[:-1]) + (c["n"],)
        s["y"] = empty(c, shape)
        s["aux"] = empty(c, shape) if c["aux"] else None
    if own:
        prepare_own(s)
    return s


def prepare_own(s):
    """The descriptors that a program fills in once for its buffers."""
    from paper_2409_02227_amd import gdy
    c, x = s["case"], s["in"]
    s["ctx"] = context()
    s["mode"] = gdy.SELECTOR
    nt = int(c.get("layout") == "nt")
    s["stream"] = gdy.ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    if c["op"] == "act_grad":
        s["desc"] = gdy.ActGrad(x["dy"], x["z"], s["dz"] if c["act"] != "none" else None, s["db"], act=c["act"],
                                offsets=s["offsets"]).desc()
        return
    # a weight gradient has the weight's layout: X^T dY, or dY^T X
    wa, wb = ((x["dy"], x["x"]) if nt else (x["x"], x["dy"])) if c["backward"] else (None, None)
    if c["backward"]:
        ep = gdy.Epilogue(act=c["act"], aux=x["z"], grad=True, bias_grad=s["db"])
    else:
        ep = gdy.Epilogue(bias=x["bias"], act=c["act"], residual=x["residual"], aux=s["aux"])
    if c["op"] == "linear":
        if c["backward"]:
            gemms = [gdy.Gemm(x["dy"], x["w"], s["dz"], 0, 1 - nt, epilogue=ep), gdy.Gemm(wa, wb, s["dw"], 1, 0)]
        else:
            gemms = [gdy.Gemm(x["x"], x["w"], s["y"], 0, nt, x["scale_x"], x["scale_w"], epilogue=ep)]
        s["n"] = len(gemms)
        s["descs"], s["epilogues"] = gdy.descs(gemms), gdy.epilogue_descs(gemms)
    elif c["backward"]:
        s["grouped"] = [gdy.Grouped(x["dy"], x["w"], s["dz"], s["offsets"], trans_b=1 - nt, epilogue=ep).descs(),
                        gdy.Grouped(wa, wb, s["dw"], s["offsets"], over="k").descs()]
    else:
        s["grouped"] = [gdy.Grouped(x["x"], x["w"], s["y"], s["offsets"], trans_b=nt, scale_a=x["scale_x"],
                                    scale_b=x["scale_w"], scales=x.get("scales"), epilogue=ep).descs()]


# ---- one pass ------------------------------------------------------------------
def outputs(s):
    c = s["case"]
    if c["op"] == "act_grad":
        return [s["dz"], s["db"]] if c["act"] != "none" else [s["db"]]
    if c["backward"]:
        return [s["dz"], s["db"], s["dw"]]
    return [s["y"]] + ([s["aux"]] if s["aux"] is not None else [])


def run(s):
    c = s["case"]
    if not own:
        {"linear": plain_linear, "experts": plain_experts, "act_grad": plain_act_grad}[c["op"]](c, s)
    elif c["op"] == "linear":
        s["ctx"].execute_descs(s["descs"], s["n"], s["mode"], 0, s["stream"], s["epilogues"])
    elif c["op"] == "experts":
        for d, e in s["grouped"]:
            s["ctx"].execute_grouped_descs(d, e, s["stream"])
    else:
        s["ctx"].execute_act_grad_desc(s["desc"], s["stream"])
    return outputs(s)


def apply_act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu":
        return z * (0.5 * torch.erfc(z * -math.sqrt(0.5)))
    if act == "gelu_tanh":  # (1 + tanh u) / 2 is the logistic function of 2u, without its cancellation
        return z / (1.0 + torch.exp(-math.sqrt(8.0 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * torch.erfc(z * -math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if act == "gelu_tanh":
        p = 1.0 / (1.0 + torch.exp(-math.sqrt(8.0 / math.pi) * (z + 0.044715 * z * z * z)))
        return p * (1.0 + z * (1.0 - p) * math.sqrt(8.0 / math.pi) * (1.0 + 3 * 0.044715 * z * z))
    if act == "silu":
        p = 1.0 / (1.0 + torch.exp(-z))
        return p * (1.0 + z * (1.0 - p))
    return torch.ones_like(z)


def plain_forward(c, x, w, scale, bias, residual, y, aux):
    """One product with its epilogue into the buffers y and aux."""
    w = w.float()
    z = torch.mm(x.float(), w.t() if c["layout"] == "nt" else w)
    if scale is not None:
        z = z * scale
    if bias is not None:
        z = z + bias.float()
    if aux is not None:
        aux.copy_(z)
    z = apply_act(z, c["act"])
    if residual is not None:
        z = z + residual.float()
    y.copy_(z)


def plain_backward(c, x, w, dy, z, dz, db, dw):
    w, dy = w.float(), dy.float()
    g = torch.mm(dy, w if c["layout"] == "nt" else w.t()) * act_slope(z.float(), c["act"])
    dz.copy_(g)
    db.copy_(g.sum(0))
    dw.copy_(torch.mm(dy.t(), x.float()) if c["layout"] == "nt" else torch.mm(x.float().t(), dy))


def plain_linear(c, s):
    x = s["in"]
    if c["backward"]:
        plain_backward(c, x["x"], x["w"], x["dy"], x["z"], s["dz"], s["db"], s["dw"])
        return
    scale = x["scale_x"] * x["scale_w"] if c["dtype"] == "fp8" else None
    if not c["batch"]:
        plain_forward(c, x["x"], x["w"], scale, x["bias"], x["residual"], s["y"], s["aux"])
        return
    for i in range(c["batch"]):
        plain_forward(c, x["x"][i], x["w"][i], scale, x["bias"], None if x["residual"] is None else x["residual"][i],
                      s["y"][i], None if s["aux"] is None else s["aux"][i])


def plain_experts(c, s):
    x = s["in"]
    for e, (lo, hi) in enumerate(s["bounds"]):
        if c["backward"]:
            plain_backward(c, x["x"][lo:hi], x["w"][e], x["dy"][lo:hi], x["z"][lo:hi], s["dz"][lo:hi], s["db"][e],
                           s["dw"][e])
        elif hi > lo:
            scale = x["scale_x"] * x["scale_w"] * x["scales"][e] if c["dtype"] == "fp8" else None
            plain_forward(c, x["x"][lo:hi], x["w"][e], scale, None if x["bias"] is None else x["bias"][e], None,
                          s["y"][lo:hi], None if s["aux"] is None else s["aux"][lo:hi])


def plain_act_grad(c, s):
    x = s["in"]
    used = c["rows"]
    g = x["dy"][:used].float()
    if c["act"] != "none":
        g = g * act_slope(x["z"][:used].float(), c["act"])
        s["dz"][:used].copy_(g)
    if not c["groups"]:
        s["db"].copy_(g.sum(0))
        return
    for e, (lo, hi) in enumerate(s["bounds"]):
        s["db"][e].copy_(g[lo:hi].sum(0))


def work(c):
    es, os_ = SIZE[c["dtype"]], OUT_SIZE[c["dtype"]]
    if c["op"] == "act_grad":
        e = max(c["groups"], 1)
        per = 1 if c["act"] == "none" else 3
        return {"bytes": per * c["rows"] * c["n"] * es + e * c["n"] * 4, "flops": (12 if per > 1 else 1) * c["rows"] * c["n"]}
    n, k = c["n"], c["k"]
    if c["op"] == "linear":
        items = max(c["batch"], 1)
        m, live, groups = c["m"] * items, items, 1
    else:
        m, live, groups = c["rows"], sum(1 for q in counts(c) if q), c["groups"]
    if c["backward"]:  # dY, X, Z, W read; dZ, dW and the bias gradients written
        dw = (live if c["op"] == "linear" else groups) * n * k * os_
        return {"bytes": (m * n + m * k + live * n * k) * es + 2 * m * k * os_ + dw + groups * k * 4,
                "flops": 4 * m * n * k}
    extra = 1 + int(bool(c.get("residual"))) + int(c["aux"])
    bias = (live if c["op"] == "experts" else 1) * n * os_ if c["bias"] else 0
    return {"bytes": (m * k + live * n * k) * es + extra * m * n * os_ + bias, "flops": 2 * m * n * k}


# ---- the definitions in 64 bits --------------------------------------------------
def f64(z, act):
    """(f(z), f'(z)) in double precision."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        on = (z > 0).double()
        return z * on, on
    if act == "gelu":
        phi = torch.special.ndtr(z)
        return z * phi, phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        p = torch.sigmoid(z)
        return z * p, p + z * p * torch.sigmoid(-z)
    t = torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))  # gelu_tanh
    inner = math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z ** 2)
    return z * (1 + t) / 2, (1 + t) / 2 + z * (1 - t ** 2) * inner / 2


def exact(c, seed):
    x = inputs(c, seed)
    x = {k: v.double() if isinstance(v, torch.Tensor) else v for k, v in x.items()}
    parts = [(0, c["rows"])] if c["op"] == "act_grad" else None
    if "counts" in x:
        parts, lo = [], 0
        for q in x["counts"]:
            parts.append((lo, lo + q))
            lo += q
    if c["op"] == "act_grad":
        dz = torch.zeros_like(x["dy"])
        dz[:c["rows"]] = x["dy"][:c["rows"]]
        if x["z"] is not None:
            dz = dz * f64(x["z"], c["act"])[1]
        db = torch.stack([dz[a:b].sum(0) for a, b in parts])
        db = db if c["groups"] else db[0]
        return [dz, db] if c["act"] != "none" else [db]
    # one list of (rows of X and dY, weight, bias, ...) problems
    w = x["w"] if c["layout"] == "nn" else x["w"].transpose(-1, -2)
    scale = x["scale_x"] * x["scale_w"]
    if c["backward"]:
        problems = [(slice(a, b), w[e]) for e, (a, b) in enumerate(parts)] if parts else [(slice(None), w)]
        dz, db, dw = torch.zeros_like(x["x"]), [], []
        for rows, we in problems:
            g = (x["dy"][rows] @ we.t()) * f64(x["z"][rows], c["act"])[1]
            dz[rows] = g
            db.append(g.sum(0))
            d = x["x"][rows].t() @ x["dy"][rows]
            dw.append(d if c["layout"] == "nn" else d.t())
        return [dz, torch.stack(db), torch.stack(dw)] if parts else [dz, db[0], dw[0]]
    y = torch.zeros(x["x"].shape[:-1] + (c["n"],), dtype=torch.float64, device="cuda")
    aux = torch.zeros_like(y)
    count = c["groups"] if parts else max(c["batch"], 1)
    for e in range(count):
        at = slice(*parts[e]) if parts else (e if c["batch"] else slice(None))
        z = x["x"][at] @ (w[e] if parts or c["batch"] else w) * scale
        if "scales" in x:
            z = z * x["scales"][e]
        if x["bias"] is not None:
            z = z + (x["bias"][e] if parts else x["bias"])
        aux[at] = z
        y[at] = f64(z, c["act"])[0]
        if x["residual"] is not None:
            y[at] += x["residual"][at]
    return [y, aux] if c["aux"] else [y]
