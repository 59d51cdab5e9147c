"""Cases of the operators around a mixture of experts and of 8-bit linear layers:
tokens sorted by expert, their rows taken to the experts and back (with the
gradients of both), rows quantised to 8-bit integers, and products of 8-bit
integers with a scale for each token and each channel, dense and by expert.

A case is a dict of plain values.

"op": "route".  From the expert ids of each token (tokens x top_k, "ids" 32 or 64
  bits; a share "drop" of them -1: pairs that no expert here takes) the bounds of
  each expert's rows and every pair's row (-1: none), pairs in their order.
"op": "dispatch".  Each token's row to its pairs' rows.  "backward": the gradient
  of "combine": every row weighted, and the products' sums for the weights.
"op": "combine".  The weighted sum of each token's rows ("weights" false: their
  sum, the gradient of "dispatch"), onto a residual where "residual".
"op": "linear8".  y = act(xs q(x) ws W + bias) + residual, x quantised by row (xs = max
  |x| / 127, q the nearest whole number; "quantize" false: it is in 8 bits already), W 8-bit with a scale for each column,
  k x n ("nn") or n x k ("nt").
"op": "experts8".  The same for the rows that tokens are taken to, by expert.
"skew": how uneven the experts are.  "pad" widens every row pitch by that many
elements; "dtype" is the activations' type.
"""
import functools
import math
import os

import torch

own = False

TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}


def route(name, tokens, top_k, experts, ids=64, drop=0.0, skew=0.5):
    return {"name": name, "op": "route", "tokens": tokens, "top_k": top_k, "experts": experts, "ids": ids,
            "drop": drop, "skew": skew}


def dispatch(name, dtype, tokens, top_k, experts, n, backward=False, drop=0.0, skew=0.5, pad=0):
    return {"name": name, "op": "dispatch", "dtype": dtype, "tokens": tokens, "top_k": top_k, "experts": experts,
            "n": n, "backward": backward, "drop": drop, "skew": skew, "pad": pad}


def combine(name, dtype, tokens, top_k, experts, n, weights=True, residual=False, drop=0.0, skew=0.5, pad=0):
    return {"name": name, "op": "combine", "dtype": dtype, "tokens": tokens, "top_k": top_k, "experts": experts,
            "n": n, "weights": weights, "residual": residual, "drop": drop, "skew": skew, "pad": pad}


def linear8(name, dtype, m, n, k, layout="nt", act="none", bias=False, residual=False, quantize=True, pad=0):
    return {"name": name, "op": "linear8", "dtype": dtype, "m": m, "n": n, "k": k, "layout": layout, "act": act,
            "bias": bias, "residual": residual, "quantize": quantize, "pad": pad}


def experts8(name, dtype, tokens, top_k, experts, n, k, layout="nt", act="none", bias=False, drop=0.0, skew=0.5, pad=0):
    return {"name": name, "op": "experts8", "dtype": dtype, "tokens": tokens, "top_k": top_k, "experts": experts,
            "n": n, "k": k, "layout": layout, "act": act, "bias": bias, "drop": drop, "skew": skew, "pad": pad}


def listed():
    return [
        # a decoding step of 32 sequences, two experts each: what a call costs
        route("route_decode", 32, 2, 16),
        # a batch of prompts or a training step, eight experts a token, some pairs on other GPUs
        route("route_prefill", 16384, 8, 128, ids=32, drop=0.1),
        # a training step's rows to their experts
        dispatch("dispatch_bf16", "bf16", 8192, 2, 16, 4096),
        # backward through the weighted sum: rows' gradients and the router's
        dispatch("combine_backward_bf16", "bf16", 8192, 2, 16, 4096, backward=True),
        # a decoding step's rows back onto the residual stream
        combine("combine_decode_bf16", "bf16", 32, 2, 16, 2048, residual=True),
        # a long batch back onto the residual stream, eight rows a token
        combine("combine_prefill_bf16", "bf16", 8192, 8, 64, 2048, residual=True),
        # sizes that nothing divides, pairs without a row, the gradient of taking rows to experts
        combine("dispatch_backward_odd_f16", "f16", 777, 3, 9, 1001, weights=False, drop=0.2),
        # one token through one 8-bit linear layer: what a call costs, and a weight read once
        linear8("linear8_token_bf16", "bf16", 1, 2048, 2048, act="silu", quantize=False),
        # a long prompt through an 8-bit layer, onto the residual stream
        linear8("linear8_prompt_bf16", "bf16", 4096, 8192, 8192, bias=True, residual=True),
        # sizes that nothing divides, rows packed without any alignment
        linear8("linear8_odd_f16", "f16", 509, 2047, 1021, layout="nn", act="relu", bias=True),
        # a decoding step: 32 sequences, two 8-bit experts each
        experts8("experts8_decode_bf16", "bf16", 32, 2, 16, 2048, 2048, act="silu"),
        # a prompt through 8-bit experts
        experts8("experts8_prefill_bf16", "bf16", 4096, 2, 16, 4096, 2048, act="silu", bias=True, skew=0.8),
    ]


def spread(rng, lo, hi, step=1):
    """A size between lo and hi, even over its logarithm, on multiples of step."""
    x = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(int(round(x / step)) * step, step)


MOST = 5e11  # operations of a drawn case, below the largest listed one's
MOST_BYTES = 3e8


def too_large(c):
    """Whether the plain form would take more memory than it should: pairs x experts
    comparisons, or every expert padded to the most popular one's rows."""
    if c["op"] == "route":
        return c["tokens"] * c["top_k"] * c["experts"] > 2e7
    if c["op"] == "experts8":
        p = [math.exp(v) for v in popularity(c)]
        most = c["tokens"] * min(1.0, c["top_k"] * max(p) / sum(p))
        return c["experts"] * most > 262144
    return False


def draw(rng):
    while True:
        c = draw_any(rng)
        w = work(c)
        if w["flops"] <= MOST and w["bytes"] <= MOST_BYTES and not too_large(c):
            return c


def draw_any(rng):
    kind = rng.choice(["route", "dispatch", "dispatch_grad", "combine", "linear8", "linear8", "experts8", "experts8"])
    experts, top_k = rng.choice([4, 8, 16, 60, 128, 256]), rng.choice([1, 2, 3, 4, 8])
    top_k = min(top_k, experts)
    drop, skew = rng.choice([0.0, 0.0, 0.25]), rng.choice([0.0, 0.5, 1.5])
    tokens = spread(rng, 1, 16384)
    if kind == "route":
        return route(None, tokens, top_k, experts, rng.choice([32, 64]), drop, skew)
    step = rng.choice([256, 64, 64, 8, 1])
    pad = rng.choice([0, 0, 0, 16]) if step > 1 else 0
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind.startswith("dispatch"):
        return dispatch(None, dtype, tokens, top_k, experts, spread(rng, 64, 8192, step), kind == "dispatch_grad", drop,
                        skew, pad)
    if kind == "combine":
        return combine(None, dtype, tokens, top_k, experts, spread(rng, 64, 8192, step), rng.random() < 0.6,
                       rng.random() < 0.5, drop, skew, pad)
    top = 1500 if step == 1 else 16384
    n, k = spread(rng, 64, top, step), spread(rng, 64, top, step)
    layout, act = rng.choice(["nt", "nt", "nn"]), rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"])
    if kind == "linear8":
        return linear8(None, dtype, spread(rng, 1, 8192), n, k, layout, act, rng.random() < 0.5, rng.random() < 0.5,
                       rng.random() < 0.6, pad)
    n, k = min(n, 4096 if step > 1 else top), min(k, 4096 if step > 1 else top)
    return experts8(None, dtype, spread(rng, 1, 8192), top_k, experts, n, k, layout, act, rng.random() < 0.4, drop,
                    skew, pad)


# ---- inputs ------------------------------------------------------------------
def popularity(c):
    """How much likelier each expert is, in logarithms: a power law over them."""
    return [-c["skew"] * math.log(i + 1.0) for i in range(c["experts"])]


def chosen(c, gen):
    """Expert ids (tokens x top_k, int64): each token's top_k distinct experts by their
    popularity and a draw of its own; a share of them none."""
    u = torch.rand((c["tokens"], c["experts"]), generator=gen, device="cuda").clamp_(1e-9, 1 - 1e-7)
    score = torch.tensor(popularity(c), device="cuda") - torch.log(-torch.log(u))
    ids = score.topk(c["top_k"], dim=1).indices
    gone = torch.rand(ids.shape, generator=gen, device="cuda") < c["drop"]
    return torch.where(gone, torch.full_like(ids, -1), ids)


def sorted_rows(ids, experts):
    """(slots, offsets, rows in use) of the ids: pairs stably sorted by expert."""
    flat = ids.reshape(-1)
    order = torch.where(flat < 0, experts, flat).argsort(stable=True)
    slots = torch.empty_like(flat)
    slots[order] = torch.arange(flat.numel(), device=flat.device)
    slots = torch.where(flat < 0, -1, slots).reshape(ids.shape).to(torch.int32)
    counts = torch.bincount(flat[flat >= 0], minlength=experts)
    offsets = torch.zeros(experts + 1, dtype=torch.int32, device=flat.device)
    offsets[1:] = counts.cumsum(0)
    return slots.contiguous(), offsets, counts


def padded(x, pad):
    """The values with `pad` more elements between rows."""
    if not pad:
        return x.contiguous()
    out = torch.zeros(x.shape[:-1] + (x.shape[-1] + pad,), dtype=x.dtype, device=x.device)
    out[..., :x.shape[-1]] = x
    return out[..., :x.shape[-1]]


def activations(gen, c, rows, n):
    """Rows of normal values, a few columns ten times the others, as layers see them."""
    x = torch.randn((rows, n), generator=gen, device="cuda")
    x[:, ::97] *= 10.0
    return padded(x.to(TORCH[c["dtype"]]), c["pad"])


def codes(gen, c, shape):
    """8-bit values of normal ones, the largest of each about 127."""
    x = torch.randn(shape, generator=gen, device="cuda") * 36.0
    return padded(x.round_().clamp_(-127, 127).to(torch.int8), c["pad"])


def inputs(c, seed):
    """What a program has in hand, from the seed alone."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = {}
    if c["op"] != "linear8":
        ids = chosen(c, gen)
        if c["op"] == "route":
            return {"ids": ids.to(torch.int64 if c["ids"] == 64 else torch.int32).contiguous()}
        x["slots"], x["offsets"], x["counts"] = sorted_rows(ids, c["experts"])
        pairs = c["tokens"] * c["top_k"]
    if c["op"] in ("dispatch", "combine"):
        if c["op"] == "dispatch":
            x["x"] = activations(gen, c, c["tokens"], c["n"])
        if c["op"] == "combine" or c["backward"]:
            x["z"] = activations(gen, c, pairs, c["n"])
        if c["op"] == "combine" and c["residual"]:
            x["residual"] = activations(gen, c, c["tokens"], c["n"])
        if c.get("weights") or c.get("backward"):
            w = torch.rand((c["tokens"], c["top_k"]), generator=gen, device="cuda") + 0.05
            x["weights"] = w / w.sum(1, keepdim=True)
        return x
    n, k = c["n"], c["k"]
    rows = c["m"] if c["op"] == "linear8" else c["tokens"]
    lead = () if c["op"] == "linear8" else (c["experts"],)
    if c["op"] == "linear8" and not c["quantize"]:
        x["q"] = codes(gen, c, (rows, k))
        x["scales"] = (torch.rand(rows, generator=gen, device="cuda") + 0.5) / 64
    else:
        x["x"] = activations(gen, c, rows, k)
    x["w"] = codes(gen, c, lead + ((k, n) if c["layout"] == "nn" else (n, k)))
    # products of unit deviation: codes of deviation 36
    x["w_scales"] = (torch.rand(lead + (n,), generator=gen, device="cuda") + 0.5) / (36.0 * math.sqrt(k))
    x["bias"] = torch.randn(lead + (n,), generator=gen, device="cuda").to(TORCH[c["dtype"]]) if c["bias"] else None
    x["residual"] = activations(gen, c, rows, n) if c.get("residual") else None
    return x


@functools.lru_cache(maxsize=1)
def context():
    """The handle a program creates once and keeps."""
    from paper_2409_02227_amd import gdy
    table = os.path.join(os.path.dirname(os.path.abspath(gdy.__file__)), "tables", "gfx950.table")
    return gdy.Context(0, table=table)


def empty(c, rows, n, dtype=None):
    """An output buffer with the case's row pitch.  Zeros: rows of no token stay so."""
    return torch.zeros((rows, n + c["pad"]), dtype=dtype or TORCH[c["dtype"]], device="cuda")[:, :n]


def prepare(c, seed):
    x = inputs(c, seed)
    s = {"case": c, "in": x}
    if c["op"] == "route":
        s["slots"] = torch.zeros(x["ids"].shape, dtype=torch.int32, device="cuda")
        s["offsets"] = torch.zeros(c["experts"] + 1, dtype=torch.int32, device="cuda")
    elif c["op"] == "dispatch":
        s["out"] = empty(c, c["tokens"] * c["top_k"], c["n"])
        s["dw"] = torch.zeros(c["tokens"], c["top_k"], device="cuda") if c["backward"] else None
    elif c["op"] == "combine":
        s["y"] = empty(c, c["tokens"], c["n"])
    else:
        rows = c["m"] if c["op"] == "linear8" else c["tokens"] * c["top_k"]
        s["y"] = empty(c, rows, c["n"])
        if "x" in x:
            s["q"] = empty(c, rows, c["k"], torch.int8)
            s["scales"] = torch.zeros(rows, device="cuda")
        if c["op"] == "experts8":  # the plain form's places of sorted rows among padded experts
            most = max(int(x["counts"].max()), 1)
            row = torch.arange(rows, device="cuda")
            e = torch.searchsorted(x["offsets"][1:].long().contiguous(), row, right=True)
            s["used"] = int(x["offsets"][-1])
            e = e[:s["used"]]
            s["place"] = e * most + row[:s["used"]] - x["offsets"].long()[e]
            s["most"] = most
    if own:
        prepare_own(s)
    return s


def prepare_own(s):
    """The descriptors that a program fills in once for its buffers."""
    from paper_2409_02227_amd import gdy
    c, x = s["case"], s["in"]
    s["ctx"] = context()
    s["stream"] = gdy.ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    if c["op"] == "route":
        s["desc"] = gdy.Route(x["ids"], s["slots"], s["offsets"]).desc()
    elif c["op"] == "dispatch":
        s["desc"] = gdy.Scatter(x["x"], x["slots"], s["out"], weights=x.get("weights"), z=x.get("z"),
                                weight_grad=s["dw"]).desc()
    elif c["op"] == "combine":
        s["desc"] = gdy.Combine(x["z"], x["slots"], s["y"], weights=x.get("weights"),
                                residual=x.get("residual")).desc()
    else:
        q, scales = (x["q"], x["scales"]) if "q" in x else (s["q"], s["scales"])
        s["quantize"] = gdy.Quantize(x["x"], q, scales, slots=x.get("slots")).desc() if "x" in x else None
        ep = gdy.Epilogue(bias=x["bias"], act=c["act"], residual=x["residual"])
        s["product"] = gdy.Int8(q, x["w"], s["y"], scales, x["w_scales"], offsets=x.get("offsets"),
                                trans_b=int(c["layout"] == "nt"), epilogue=ep).descs()


# ---- one pass ------------------------------------------------------------------
def outputs(s):
    op = s["case"]["op"]
    if op == "route":
        return [s["slots"], s["offsets"]]
    if op == "dispatch":
        return [s["out"]] + ([s["dw"]] if s["dw"] is not None else [])
    if op == "combine":
        return [s["y"]]
    return [s["y"]] + ([s["scales"]] if "scales" in s else [])


def run(s):
    op = s["case"]["op"]
    if not own:
        {"route": plain_route, "dispatch": plain_dispatch, "combine": plain_combine, "linear8": plain_linear8,
         "experts8": plain_experts8}[op](s["case"], s)
    elif op == "route":
        s["ctx"].execute_route_desc(s["desc"], s["stream"])
    elif op == "dispatch":
        s["ctx"].execute_scatter_desc(s["desc"], s["stream"])
    elif op == "combine":
        s["ctx"].execute_combine_desc(s["desc"], s["stream"])
    else:
        if s["quantize"] is not None:
            s["ctx"].execute_quantize_desc(s["quantize"], s["stream"])
        s["ctx"].execute_int8_descs(*s["product"], s["stream"])
    return outputs(s)


def plain_route(c, s):
    flat = s["in"]["ids"].reshape(-1)
    mine = torch.arange(c["experts"], device="cuda", dtype=flat.dtype)[:, None] == flat[None, :]
    upto = mine.cumsum(1, dtype=torch.int32)  # pairs of each expert so far, this one among them
    s["offsets"][1:] = upto[:, -1].cumsum(0)
    expert = flat.clamp(min=0).long()
    at = s["offsets"].long()[expert] + upto[expert, torch.arange(flat.numel(), device="cuda")] - 1
    s["slots"].copy_(torch.where(flat < 0, -1, at).reshape(s["slots"].shape))


def pairs_of(slots):
    """(the pairs that have a row, their rows, their tokens)."""
    flat = slots.reshape(-1).long()
    pair = (flat >= 0).nonzero()[:, 0]
    return pair, flat[pair], pair // slots.shape[1]


def plain_dispatch(c, s):
    x = s["in"]
    pair, row, token = pairs_of(x["slots"])
    if not c["backward"]:
        s["out"][row] = x["x"][token]
        return
    g = x["x"][token].float()
    s["out"][row] = (g * x["weights"].reshape(-1)[pair, None]).to(s["out"].dtype)
    s["dw"].zero_()
    s["dw"].view(-1)[pair] = (g * x["z"][row].float()).sum(1)


def plain_combine(c, s):
    x = s["in"]
    slots = x["slots"].long()
    rows = x["z"][slots.clamp(min=0)].float()  # tokens x top_k x n
    w = (slots >= 0).float()
    if c["weights"]:
        w = w * x["weights"]
    y = (rows * w[:, :, None]).sum(1)
    if c["residual"]:
        y = y + x["residual"].float()
    s["y"].copy_(y)


def quantized(x):
    """(8-bit values as fp32, scales) of rows: scale = max |x| / 127, values the nearest
    whole numbers (64 bits: a value next to a half must not cross it)."""
    x = x.double()
    most = x.abs().amax(1)
    over = torch.where(most > 0, most, torch.ones_like(most))
    return torch.round(x * 127.0 / over[:, None]).float(), most.float() / 127.0


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


def plain_linear8(c, s):
    x = s["in"]
    if "q" in x:
        q, scales = x["q"].float(), x["scales"]
    else:
        q, scales = quantized(x["x"])
        s["scales"].copy_(scales)
    w = x["w"].float()
    z = torch.mm(q, w.t() if c["layout"] == "nt" else w) * scales[:, None] * x["w_scales"]
    if x["bias"] is not None:
        z = z + x["bias"].float()
    z = apply_act(z, c["act"])
    if x["residual"] is not None:
        z = z + x["residual"].float()
    s["y"].copy_(z)


def plain_experts8(c, s):
    x = s["in"]
    pair, row, token = pairs_of(x["slots"])
    q, scales = quantized(x["x"])
    s["scales"][row] = scales[token]
    # the rows of every expert padded to the longest one's: one batched product
    a = torch.zeros((c["experts"] * s["most"], c["k"]), device="cuda")
    place = s["place"][row]
    a[place] = q[token]
    w = x["w"].float()
    w = w.transpose(1, 2).contiguous() if c["layout"] == "nt" else w.contiguous()
    z = torch.bmm(a.view(c["experts"], s["most"], c["k"]), w) * x["w_scales"][:, None]
    z = z.view(-1, c["n"])[s["place"]] * s["scales"][:s["used"], None]
    if x["bias"] is not None:
        z = z + x["bias"].float()[s["place"] // s["most"]]
    s["y"][:s["used"]] = apply_act(z, c["act"]).to(s["y"].dtype)


# ---- what a pass cannot do without ------------------------------------------------
def work(c):
    if c["op"] == "route":
        pairs = c["tokens"] * c["top_k"]
        return {"bytes": pairs * (c["ids"] // 8 + 4) + 4 * (c["experts"] + 1), "flops": 2 * pairs}
    if c["op"] == "linear8":
        m, n, k, es = c["m"], c["n"], c["k"], SIZE[c["dtype"]]
        a = m * k * (es if c["quantize"] else 1) + 4 * m
        side = (1 + int(c["residual"])) * m * n * es + (n * es if c["bias"] else 0)
        return {"bytes": a + n * k + 4 * n + side, "flops": 2 * m * n * k}
    es = SIZE[c["dtype"]]
    pairs = c["tokens"] * c["top_k"]
    rows = int(pairs * (1 - c["drop"]))
    if c["op"] == "dispatch":
        moved = c["tokens"] + (2 if c["backward"] else 1) * rows
        return {"bytes": moved * c["n"] * es + pairs * (4 + (8 if c["backward"] else 0)),
                "flops": (3 if c["backward"] else 1) * rows * c["n"]}
    if c["op"] == "combine":
        moved = rows + c["tokens"] * (1 + int(c["residual"]))
        return {"bytes": moved * c["n"] * es + pairs * (4 + (4 if c["weights"] else 0)), "flops": 2 * rows * c["n"]}
    n, k = c["n"], c["k"]
    live = min(c["experts"], rows)
    return {"bytes": c["tokens"] * k * es + live * (n * k + 4 * n + (n * es if c["bias"] else 0)) + rows * n * es + 4 * pairs
            + 4 * rows, "flops": 2 * rows * n * k}


# ---- the definitions in 64 bits --------------------------------------------------
def exact_act(z, act):
    if act == "relu":
        return torch.clamp(z, min=0.0)
    if act == "gelu":
        return z * torch.special.ndtr(z)
    if act == "gelu_tanh":
        return z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))) / 2
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def exact_rows(x):
    """The values that the 8-bit codes of each row stand for, over the row's scale, and the scales."""
    most = x.abs().max(1).values
    twice = 254 * x + most[:, None]  # the nearest whole number, ties to the even one
    steps = torch.floor(twice / (2 * most.clamp(min=1e-300)[:, None]))
    tie = (steps * (2 * most[:, None]) == twice) & (steps.remainder(2) == 1)
    return torch.where(tie, steps - 1, steps), most / 127


def exact(c, seed):
    x = inputs(c, seed)
    if c["op"] == "route":
        slots, offsets, _ = sorted_rows(x["ids"].long(), c["experts"])
        return [slots, offsets]
    x = {key: v.double() if isinstance(v, torch.Tensor) and v.dtype not in (torch.int32, torch.int64) else v
         for key, v in x.items()}
    if c["op"] in ("dispatch", "combine"):
        slots = x["slots"].long()
        pairs = c["tokens"] * c["top_k"]
        # tokens x rows as a list of links, one choice of every token after the other
        if c["op"] == "dispatch":
            out = torch.zeros((pairs, c["n"]), dtype=torch.float64, device="cuda")
            dw = torch.zeros((c["tokens"], c["top_k"]), dtype=torch.float64, device="cuda")
            for j in range(c["top_k"]):
                has = slots[:, j] >= 0
                at = slots[has, j]
                out[at] = x["x"][has] * (x["weights"][has, j, None] if c["backward"] else 1.0)
                if c["backward"]:
                    dw[has, j] = torch.linalg.vecdot(x["x"][has], x["z"][at])
            return [out, dw] if c["backward"] else [out]
        y = x["residual"].clone() if c["residual"] else torch.zeros((c["tokens"], c["n"]), dtype=torch.float64, device="cuda")
        for j in range(c["top_k"]):
            has = slots[:, j] >= 0
            y[has] += x["z"][slots[has, j]] * (x["weights"][has, j, None] if c["weights"] else 1.0)
        return [y]
    w = x["w"].transpose(-1, -2) if c["layout"] == "nt" else x["w"]
    q, scales = (x["q"], x["scales"]) if "q" in x else exact_rows(x["x"])
    if c["op"] == "linear8":
        z = (q * scales[:, None]) @ (w * x["w_scales"])
        z = exact_act(z if x["bias"] is None else z + x["bias"], c["act"])
        z = z if x["residual"] is None else z + x["residual"]
        return [z] if "q" in x else [z, scales]
    pairs = c["tokens"] * c["top_k"]
    y = torch.zeros((pairs, c["n"]), dtype=torch.float64, device="cuda")
    row_scales = torch.zeros(pairs, dtype=torch.float64, device="cuda")
    _, row, token = pairs_of(x["slots"])
    sorted_token = torch.zeros(pairs, dtype=torch.int64, device="cuda")
    sorted_token[row] = token
    row_scales[row] = scales[token]
    bounds = x["offsets"].tolist()
    for e in range(c["experts"]):
        lo, hi = bounds[e], bounds[e + 1]
        t = sorted_token[lo:hi]
        z = (q[t] * scales[t, None]) @ (w[e] * x["w_scales"][e])
        y[lo:hi] = exact_act(z if x["bias"] is None else z + x["bias"][e], c["act"])
    return [y, row_scales]
