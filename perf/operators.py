"""What a step of a model puts into the collectives and does with what they
deliver: the operators beside the synthesizer, as plain formulas and through
the library.

An expert-parallel layer spends its All-to-Alls on tokens that a router has
sent to experts; a tensor- or data-parallel one gathers operands and
gradients, the smaller the better.  The operators here are those ends:

  route      tokens to experts: softmax, top k, the slots in expert order
             (what the All-to-Allv's chunks are cut from), and the gradient
  mx         rows or columns to microscaled 4-bit floating point (blocks of 32
             E2M1 values with one power-of-two scale) and back
  linear     a product of two such operands; for one token, for prompts, and
             as a training step (forward, input and weight gradients)
  moe        a whole mixture-of-experts layer for a few tokens

`own` False: elementary torch operations in 32 bits, rounded once at the end.
`own` True: the calls a user of the library makes.
"""

from __future__ import annotations

import functools
import math

import torch

own = False

BLOCK = 32        # values that share a scale
PAD = 128         # stored rows end on whole multiples of this many values
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
MX_BYTES = 0.5 + 1 / BLOCK
VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ---- the cases ---------------------------------------------------------------

def _route(name, tokens, experts, topk, dtype, normalize, barred, train):
    c = {"op": "route", "tokens": tokens, "experts": experts, "topk": topk, "dtype": dtype,
         "normalize": normalize, "barred": barred, "train": train}
    return dict(c, name=name) if name else c


def _mx(name, rows, cols, dtype, both):
    c = {"op": "mx", "rows": rows, "cols": cols, "dtype": dtype, "both": both}
    return dict(c, name=name) if name else c


def _linear(name, m, n, k, dtype):
    c = {"op": "linear", "m": m, "n": n, "k": k, "dtype": dtype}
    return dict(c, name=name) if name else c


def _linear_train(name, m, n, k, dtype):
    c = {"op": "linear_train", "m": m, "n": n, "k": k, "dtype": dtype}
    return dict(c, name=name) if name else c


def _moe(name, tokens, experts, topk, hidden, inter, dtype, weights, masked):
    c = {"op": "moe", "tokens": tokens, "experts": experts, "topk": topk, "hidden": hidden, "inter": inter,
         "dtype": dtype, "weights": weights, "masked": masked}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of a decoder choosing among the experts of one 64-NPU group: latency only
        _route("route_1x64", 1, 64, 4, "f32", True, 0.0, False),
        # a training step's router, one expert for each of 256 NPUs
        _route("route_train_32768x256", 32768, 256, 8, "bf16", True, 0.0, True),
        # odd sizes, experts outside the token's process group barred, padding tokens, plain softmax weights
        _route("route_train_4099x61_barred", 4099, 61, 3, "f32", False, 0.3, True),
        # a small activation packed before it is sent, rows that end inside a block
        _mx("mx_333x1000", 333, 1000, "bf16", False),
        # a training activation packed along rows and columns for the forward and the weight gradient
        _mx("mx_both_16384x8192", 16384, 8192, "bf16", True),
        # one token through a 4-bit layer: the weights' bytes and the launches count
        _linear("linear_1x4096x4096", 1, 4096, 4096, "bf16"),
        # a decode batch through a wide layer
        _linear("linear_48x16384x5120", 48, 16384, 5120, "bf16"),
        # a prompt through a square layer: matrix-product bound
        _linear("linear_8192x8192x8192", 8192, 8192, 8192, "bf16"),
        # a training step of an odd-sized layer, every operand quantised along each axis it is contracted over
        _linear_train("linear_train_2040x1500x2080", 2040, 1500, 2080, "bf16"),
        # single-token decode, weights in 16 bits
        _moe("moe_1tok_64e_bf16", 1, 64, 4, 2048, 1024, "bf16", "same", False),
        # a decode batch with padding tokens, one expert for each of 128 NPUs, weights in 4 bits
        _moe("moe_16tok_128e_mx", 16, 128, 8, 4096, 1536, "bf16", "mx", True),
        # the largest decode batch, most experts in use, an odd inner size, weights in 16 bits
        _moe("moe_64tok_64e_bf16", 64, 64, 8, 2048, 1400, "bf16", "same", False),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over their logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("route", "mx", "linear", "linear_train", "moe"))
    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    if op == "route":
        experts = _spread(rng, 8, 256)
        return _route(None, _spread(rng, 1, 32768), experts, rng.randint(1, 8), dtype, rng.random() < 0.5,
                      rng.choice((0.0, 0.3)), rng.random() < 0.6)
    if op == "mx":
        return _mx(None, _spread(rng, 1, 16384), _spread(rng, 1, 8192), dtype, rng.random() < 0.5)
    if op == "linear":
        return _linear(None, _spread(rng, 1, 8192), _spread(rng, 64, 8192), _spread(rng, 64, 8192), dtype)
    if op == "linear_train":
        return _linear_train(None, _spread(rng, 16, 4096), _spread(rng, 64, 4096), _spread(rng, 64, 4096), dtype)
    mx = rng.random() < 0.5
    experts = _spread(rng, 8, 128)
    hidden = 8 * _spread(rng, 32, 512)
    return _moe(None, _spread(rng, 1, 64), experts, rng.randint(1, 8), hidden, 8 * _spread(rng, 16, 192),
                rng.choice(("bf16", "f16")), "mx" if mx else "same", rng.random() < 0.3)


# ---- microscaled 4-bit floating point, plain ------------------------------------

def _padded(k):
    return -(-k // PAD) * PAD


def _quantize(x):
    """(codes, scales) of the rows of x: scale 2^(floor(log2 max|block|) - 2), values rounded to the nearest E2M1
    value (ties to the even code) and held at 6 at most; a block with a value that is not finite has the scale NaN."""
    rows, k = x.shape
    kp = _padded(k)
    v = torch.zeros((rows, kp), dtype=torch.float32, device=x.device)
    v[:, :k] = x
    v = v.view(rows, kp // BLOCK, BLOCK)
    top = v.abs().amax(dim=-1, keepdim=True)
    bad = ~torch.isfinite(top)
    e = (torch.frexp(torch.where(bad, torch.ones_like(top), top)).exponent - 3).clamp(-127, 127)
    e = torch.where(top == 0, torch.full_like(e, -127), e)
    a = torch.ldexp(torch.ldexp(v.abs(), -torch.div(e, 2, rounding_mode="floor")), torch.div(e, 2, rounding_mode="floor") - e)
    a = torch.where(bad, torch.zeros_like(a), a)
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = (torch.round(a / step) * step).clamp(max=6.0)
    code = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8)
    code = code | (torch.signbit(v) & ~bad).to(torch.uint8) * 8
    code = code.view(rows, kp // 2, 2)
    scale = torch.where(bad, torch.full_like(e, 255), e + 127).to(torch.uint8)
    return code[..., 0] | (code[..., 1] << 4), scale.view(rows, kp // BLOCK)


def _dequantize(codes, scales, k):
    """The 32-bit values that codes and scales stand for, the first k of each row."""
    lead = codes.shape[:-1]
    table = torch.tensor(VALUES + tuple(-v for v in VALUES), dtype=torch.float32, device=codes.device)
    both = torch.stack((codes & 15, codes >> 4), dim=-1).to(torch.int32)
    v = table[both].view(*lead, -1, BLOCK)
    half = torch.div(scales.to(torch.int32) - 127, 2, rounding_mode="floor")
    v = torch.ldexp(torch.ldexp(v, half[..., None]), (scales.to(torch.int32) - 127 - half)[..., None])
    v = torch.where(scales[..., None] == 255, torch.full_like(v, math.nan), v)
    return v.view(*lead, -1)[..., :k]


def _values(x):
    """x as its microscaled form stands for it, in 32 bits."""
    return _dequantize(*_quantize(x), x.shape[1])


# ---- inputs ------------------------------------------------------------------------

def _normal(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def _activations(g, rows, cols, dtype):
    """Normal values with a spread of row sizes and a few channels that are far larger, as activations have."""
    x = torch.randn(rows, cols, generator=g, device="cuda")
    x *= torch.exp(0.5 * torch.randn(rows, 1, generator=g, device="cuda"))
    x *= torch.where(torch.rand(1, cols, generator=g, device="cuda") < 0.01, 20.0, 1.0)
    return x.to(dtype)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op, dtype = case["op"], DTYPES[case["dtype"]]
    s = {"case": dict(case)}
    if op == "route":
        t, e, k = case["tokens"], case["experts"], min(case["topk"], case["experts"])
        logits = torch.randn(t, e, generator=g, device="cuda") * 2
        s["mask"] = None
        if case["barred"]:  # experts outside a token's group, whole rows among them, and padding tokens
            logits[torch.rand(t, e, generator=g, device="cuda") < case["barred"]] = -math.inf
            logits[torch.rand(t, generator=g, device="cuda") < 0.02] = -math.inf
            s["mask"] = (torch.rand(t, generator=g, device="cuda") >= 0.05).to(torch.uint8)
        s["logits"] = logits.to(dtype)
        s["dweights"] = torch.randn(t, k, generator=g, device="cuda")
    elif op == "mx":
        s["x"] = _activations(g, case["rows"], case["cols"], dtype)
    elif op == "linear":
        s["x"] = _activations(g, case["m"], case["k"], dtype)
        s["w"] = _quantize(_normal(g, case["n"], case["k"], scale=case["k"] ** -0.5))
    elif op == "linear_train":
        s["x"] = _activations(g, case["m"], case["k"], dtype)
        s["w"] = _normal(g, case["n"], case["k"], dtype=dtype, scale=case["k"] ** -0.5)
        s["dy"] = _normal(g, case["m"], case["n"], dtype=dtype, scale=1e-3)
    else:
        t, e, h, i = case["tokens"], case["experts"], case["hidden"], case["inter"]
        s["x"] = _normal(g, t, h, dtype=dtype)
        s["router"] = _normal(g, e, h, dtype=dtype, scale=2 * h ** -0.5)
        s["mask"] = (torch.arange(t, device="cuda") < max(1, t - t // 4)).to(torch.uint8) if case["masked"] else None
        up, down = [], []
        for _ in range(e):
            u, d = _normal(g, 2 * i, h, scale=h ** -0.5), _normal(g, h, i, scale=i ** -0.5)
            up.append(_quantize(u) if case["weights"] == "mx" else u.to(dtype))
            down.append(_quantize(d) if case["weights"] == "mx" else d.to(dtype))
        if case["weights"] == "mx":
            s["up"] = tuple(torch.stack(p) for p in zip(*up))
            s["down"] = tuple(torch.stack(p) for p in zip(*down))
        else:
            s["up"], s["down"] = torch.stack(up), torch.stack(down)
    return s


# ---- plain forms ---------------------------------------------------------------------

def _pick(logits, k, normalize, mask):
    """weights, ids of the k largest logits of each row (ties to the lowest index); -1 and 0 where none is left."""
    l = logits.float()
    if mask is not None:
        l = torch.where(mask[:, None] != 0, l, torch.full_like(l, -math.inf))
    val, ids = torch.sort(l, dim=1, descending=True, stable=True)
    val, ids = val[:, :k], ids[:, :k]
    top = val[:, :1]
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    there = val > -math.inf
    w = torch.exp(val - top)
    total = (w if normalize else torch.exp(l - top)).sum(dim=1, keepdim=True)
    w = torch.where(there, w / torch.where(total == 0, torch.ones_like(total), total), torch.zeros_like(w))
    return w, torch.where(there, ids, torch.full_like(ids, -1)).to(torch.int32)


def _plain_route(s):
    c, logits, mask = s["case"], s["logits"], s["mask"]
    t, e = logits.shape
    k = min(c["topk"], e)
    w, ids = _pick(logits, k, c["normalize"], mask)
    flat = ids.reshape(-1).to(torch.int64)
    flat = torch.where(flat < 0, torch.full_like(flat, e), flat)
    place, slot = torch.sort(flat, stable=True)
    out = {"weights": w, "ids": ids,
           "counts": (flat[:, None] == torch.arange(e, device=flat.device)).sum(dim=0).to(torch.int32),
           "order": torch.where(place < e, slot, torch.full_like(slot, -1)).to(torch.int32)}
    if c["train"]:
        gw = s["dweights"] * w
        inner = gw.sum(dim=1, keepdim=True)
        spot = torch.where(ids < 0, torch.full_like(ids, e), ids).to(torch.int64)
        d = torch.zeros((t, e + 1), dtype=torch.float32, device=w.device)
        if c["normalize"]:
            d.scatter_(1, spot, gw - w * inner)
            d = d[:, :e]
        else:
            l = logits.float()
            if mask is not None:
                l = torch.where(mask[:, None] != 0, l, torch.full_like(l, -math.inf))
            top = l.amax(dim=1, keepdim=True)
            p = torch.exp(l - torch.where(torch.isinf(top), torch.zeros_like(top), top))
            total = p.sum(dim=1, keepdim=True)
            p = p / torch.where(total == 0, torch.ones_like(total), total)
            d.scatter_(1, spot, gw)
            d = d[:, :e] - p * inner
        out["dlogits"] = d.to(logits.dtype)
    return out


def _plain_mx(s):
    x = s["x"]
    out = {"rows": _values(x).to(x.dtype)}
    if s["case"]["both"]:
        out["cols"] = _values(x.t()).to(x.dtype)
    return out


def _plain_linear(s):
    x = s["x"]
    return (_values(x) @ _dequantize(*s["w"], x.shape[1]).t()).to(x.dtype)


def _plain_linear_train(s):
    x, w, dy = s["x"], s["w"], s["dy"]
    return {"y": (_values(x) @ _values(w).t()).to(x.dtype),
            "dx": (_values(dy) @ _values(w.t()).t()).to(x.dtype),
            "dw": _values(dy.t()) @ _values(x.t()).t()}


def _plain_moe(s):
    c, x, up, down = s["case"], s["x"].float(), s["up"], s["down"]
    t, e, h, i = c["tokens"], c["experts"], c["hidden"], c["inter"]
    k = min(c["topk"], e)
    w, ids = _pick(x @ s["router"].float().t(), k, True, s["mask"])
    there = ids >= 0
    slot = torch.where(there, ids, torch.zeros_like(ids)).to(torch.int64)
    full = (lambda p, n, at: _dequantize(p[0][at], p[1][at], n)) if c["weights"] == "mx" else (lambda p, n, at: p[at].float())
    if t * k < e:  # each slot's own weights
        at = slot.reshape(-1)
        rows = x.repeat_interleave(k, dim=0)[:, :, None]
        gate, lift = torch.bmm(full(up, h, at), rows)[:, :, 0].split(i, dim=1)
        y = torch.bmm(full(down, i, at), (gate / (1 + torch.exp(-gate)) * lift)[:, :, None])[:, :, 0].view(t, k, h)
        return (torch.where(there, w, torch.zeros_like(w))[:, :, None] * y).sum(dim=1).to(s["x"].dtype)
    every = torch.arange(e, device=x.device)  # all experts on all tokens
    gate, lift = torch.matmul(full(up, h, every), x.t()).transpose(1, 2).split(i, dim=2)
    y = torch.bmm(gate / (1 + torch.exp(-gate)) * lift, full(down, i, every).transpose(1, 2))
    mix = torch.zeros((t, e), dtype=torch.float32, device=x.device)
    mix.scatter_add_(1, slot, torch.where(there, w, torch.zeros_like(w)))
    return (mix.t()[:, :, None] * y).sum(dim=0).to(s["x"].dtype)


# ---- the library's calls -----------------------------------------------------------------

@functools.lru_cache(maxsize=None)
def _library():
    from paper_2606_07019_amd import operators
    return operators, operators.Operators(device=0)


def _own_route(s):
    c, logits, mask = s["case"], s["logits"], s["mask"]
    _, ops = _library()
    k = min(c["topk"], c["experts"])
    w, ids, counts, order = ops.route(logits, k, normalize=c["normalize"], mask=mask)
    out = {"weights": w, "ids": ids, "counts": counts, "order": order}
    if c["train"]:
        out["dlogits"] = ops.route_backward(logits, w, ids, s["dweights"], normalize=c["normalize"], mask=mask)
    return out


def _own_mx(s):
    x = s["x"]
    _, ops = _library()
    if not s["case"]["both"]:
        return {"rows": ops.dequantize(ops.quantize(x), x.dtype)}
    rows, cols = ops.quantize_both(x)
    return {"rows": ops.dequantize(rows, x.dtype), "cols": ops.dequantize(cols, x.dtype)}


def _own_linear(s):
    x = s["x"]
    lib, ops = _library()
    return ops.matmul(ops.quantize(x), lib.MX(s["w"][0], s["w"][1], x.shape[1]), x.dtype)


def _own_linear_train(s):
    x, w, dy = s["x"], s["w"], s["dy"]
    _, ops = _library()
    (xr, xc), (wr, wc), (dr, dc) = ops.quantize_both(x), ops.quantize_both(w), ops.quantize_both(dy)
    return {"y": ops.matmul(xr, wr, x.dtype), "dx": ops.matmul(dr, wc, x.dtype),
            "dw": ops.matmul(dc, xc, torch.float32)}


def _own_moe(s):
    c, up, down = s["case"], s["up"], s["down"]
    lib, ops = _library()
    if c["weights"] == "mx":
        up, down = lib.MX(up[0], up[1], c["hidden"]), lib.MX(down[0], down[1], c["inter"])
    return ops.moe_layer(s["x"], s["router"], up, down, min(c["topk"], c["experts"]), normalize=True, mask=s["mask"])


def run(state):
    return globals()[("_own_" if own else "_plain_") + state["case"]["op"]](state)


# ---- what a pass cannot do without ---------------------------------------------------------

def _experts_used(tokens, experts, k):
    """Expected number of different experts among the picks of that many tokens."""
    return experts * (1 - (1 - k / experts) ** tokens)


def work(case):
    op, b = case["op"], SIZE[case["dtype"]]
    if op == "route":
        t, e, k = case["tokens"], case["experts"], min(case["topk"], case["experts"])
        out = t * k * 12 + 4 * e + (t if case["barred"] else 0)
        # the normalised weights' gradient needs the picks alone
        train = (t * e * b * (1 if case["normalize"] else 2) + t * k * 12) if case["train"] else 0
        return {"bytes": t * e * b + out + train, "flops": t * e * (4 if case["train"] else 2)}
    if op == "mx":
        n = case["rows"] * case["cols"]
        sides = 2 if case["both"] else 1
        return {"bytes": n * (b + sides * (2 * MX_BYTES + b)), "flops": n * 4 * sides}
    if op == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": m * k * b + n * k * MX_BYTES + m * n * b, "flops": 2 * m * n * k}
    if op == "linear_train":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": (m * k + n * k + m * n) * b + (m * n + m * k) * b + n * k * 4, "flops": 6 * m * n * k}
    t, e, h, i = case["tokens"], case["experts"], case["hidden"], case["inter"]
    k = min(case["topk"], e)
    live = max(1, t - t // 4) if case["masked"] else t
    per = 3 * h * i * (MX_BYTES if case["weights"] == "mx" else b)
    return {"bytes": _experts_used(live, e, k) * per + e * h * b + 2 * t * h * b,
            "flops": live * (2 * e * h + k * 6 * h * i)}


# ---- the definitions in 64 bits -----------------------------------------------------------------

def _exact_values(x):
    """Microscaled values by their definition: each block against the eight magnitudes at its scale, in 64 bits."""
    x = x.double()
    rows, k = x.shape
    nb = -(-k // BLOCK)
    v = torch.zeros((rows, nb * BLOCK), dtype=torch.float64, device=x.device)
    v[:, :k] = x
    v = v.view(rows, nb, BLOCK)
    top = v.abs().amax(dim=-1, keepdim=True)
    exponent = torch.floor(torch.log2(torch.where(top > 0, top, torch.ones_like(top))))
    exponent = exponent - (torch.exp2(exponent) > top).double() * (top > 0) + (torch.exp2(exponent + 1) <= top).double()
    unit = torch.exp2(torch.clamp(exponent - 2, -127, 127))
    a = v.abs() / unit
    mags = torch.tensor(VALUES, dtype=torch.float64, device=x.device)
    mids = (mags[1:] + mags[:-1]) / 2
    up = torch.searchsorted(mids, a.contiguous(), right=False)   # ties to the lower of the two ...
    tie = (up < 7) & (a == mids[up.clamp(max=6)]) & (up % 2 == 1)  # ... unless its code is odd
    return (torch.sign(v) * mags[up + tie.long()] * unit).view(rows, nb * BLOCK)[:, :k]


def _exact_unpacked(codes, scales, k):
    mags = torch.tensor(VALUES, dtype=torch.float64, device=codes.device)
    c = torch.empty((codes.shape[0], codes.shape[1] * 2), dtype=torch.long, device=codes.device)
    c[:, 0::2], c[:, 1::2] = codes.long() % 16, codes.long() // 16
    v = mags[c % 8] * (1 - 2 * (c // 8)).double()
    return (v * torch.exp2(scales.double() - 127).repeat_interleave(BLOCK, dim=1))[:, :k]


def _exact_pick(l, k, normalize, mask):
    if mask is not None:
        l = l.masked_fill(mask[:, None] == 0, -math.inf)
    p = torch.nan_to_num(torch.softmax(l, dim=1), nan=0.0)
    ids = torch.argsort(l, dim=1, descending=True, stable=True)[:, :k]
    none = torch.gather(l, 1, ids) == -math.inf
    w = torch.gather(p, 1, ids).masked_fill(none, 0.0)
    if normalize:
        w = w / w.sum(dim=1, keepdim=True).clamp(min=1e-300)
    return w, ids.masked_fill(none, -1), p


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "route":
        l, k = s["logits"].double(), min(case["topk"], case["experts"])
        w, ids, p = _exact_pick(l, k, case["normalize"], s["mask"])
        out = {"weights": w, "ids": ids.int(), "counts": None, "order": None}
        if case["train"]:
            g = s["dweights"].double()
            picked = torch.zeros_like(l)
            grad = torch.zeros_like(l)
            for j in range(k):
                at = torch.nonzero(ids[:, j] >= 0)[:, 0]
                picked[at, ids[at, j]] = w[at, j]
                grad[at, ids[at, j]] = g[at, j]
            soft = picked if case["normalize"] else p
            out["dlogits"] = picked * grad - soft * (picked * grad).sum(dim=1, keepdim=True)
        return out
    if op == "mx":
        out = {"rows": _exact_values(s["x"])}
        if case["both"]:
            out["cols"] = _exact_values(s["x"].t())
        return out
    if op == "linear":
        return torch.matmul(_exact_values(s["x"]), _exact_unpacked(*s["w"], case["k"]).t().contiguous())
    if op == "linear_train":
        x, w, dy = s["x"], s["w"], s["dy"]
        return {"y": torch.matmul(_exact_values(x), _exact_values(w).t().contiguous()),
                "dx": torch.matmul(_exact_values(dy), _exact_values(w.t()).t().contiguous()),
                "dw": torch.matmul(_exact_values(dy.t()), _exact_values(x.t()).t().contiguous())}
    x = s["x"].double()
    i, k = case["inter"], min(case["topk"], case["experts"])
    w, ids, _ = _exact_pick(torch.matmul(x, s["router"].double().t().contiguous()), k, True, s["mask"])
    y = torch.zeros_like(x)
    for e in range(case["experts"]):
        t, j = torch.nonzero(ids == e, as_tuple=True)
        if t.numel() == 0:
            continue
        if case["weights"] == "mx":
            up = _exact_unpacked(s["up"][0][e], s["up"][1][e], case["hidden"])
            down = _exact_unpacked(s["down"][0][e], s["down"][1][e], i)
        else:
            up, down = s["up"][e].double(), s["down"][e].double()
        both = torch.matmul(x[t], up.t().contiguous())
        y[t] += w[t, j][:, None] * torch.matmul(torch.sigmoid(both[:, :i]) * both[:, :i] * both[:, i:], down.t().contiguous())
    return y
