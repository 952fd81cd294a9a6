"""The operators at the ends of a collective by their definitions, in 64-bit
numpy: microscaled 4-bit values, products of them, the router with its
gradient, and the mixture-of-experts layer.  Shares nothing with the library.
"""

from __future__ import annotations

import numpy as np

BLOCK, STEP = 32, 128
MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def mx_quantize(x: np.ndarray):
    """(codes, scales) of the rows of x, padded to whole steps of 128."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    pad = -(-cols // STEP) * STEP
    v = np.zeros((rows, pad))
    v[:, :cols] = x
    v = v.reshape(rows, pad // BLOCK, BLOCK)
    with np.errstate(invalid="ignore"):
        top = np.abs(v).max(axis=2)          # NaN where a block holds one
    bad = ~np.isfinite(top)
    exponent = np.frexp(np.where(bad | (top == 0), 1.0, top))[1] - 1   # floor(log2)
    e = np.maximum(exponent - 2, -127)
    scales = np.where(bad, 255, np.where(top == 0, 0, e + 127)).astype(np.uint8)
    unit = np.exp2(e.astype(np.float64))[..., None]
    a = np.abs(np.where(bad[..., None], 0.0, v)) / unit
    mids = (MAGNITUDES[1:] + MAGNITUDES[:-1]) / 2
    code = np.searchsorted(mids, a, side="left")       # a tie goes to the lower code ...
    tie = (code < 7) & (a == mids[np.minimum(code, 6)])
    code = code + (tie & (code % 2 == 1))              # ... unless that one is odd
    code = (code + 8 * (np.signbit(v) & ~bad[..., None])).astype(np.uint8).reshape(rows, pad)
    return code[:, 0::2] | (code[:, 1::2] << 4), scales


def mx_values(codes: np.ndarray, scales: np.ndarray, cols: int) -> np.ndarray:
    c = np.empty((codes.shape[0], codes.shape[1] * 2), np.int64)
    c[:, 0::2], c[:, 1::2] = codes & 15, codes >> 4
    v = MAGNITUDES[c % 8] * np.where(c >= 8, -1.0, 1.0)
    s = np.exp2(scales.astype(np.float64) - 127)
    s[scales == 255] = np.nan
    return (v * np.repeat(s, BLOCK, axis=1))[:, :cols]


def route(logits, topk: int, normalize: bool, mask=None):
    """(weights, ids, counts, order) in 64 bits."""
    l = np.array(logits, dtype=np.float64)
    tokens, experts = l.shape
    if mask is not None:
        l[np.asarray(mask) == 0] = -np.inf
    weights = np.zeros((tokens, topk))
    ids = np.full((tokens, topk), -1, np.int32)
    for t in range(tokens):
        key = np.where(np.isnan(l[t]), np.inf, l[t])
        picks = sorted(range(experts), key=lambda e: (not np.isnan(l[t, e]), -key[e], e))[:topk]
        picks = [e for e in picks if np.isnan(l[t, e]) or l[t, e] > -np.inf]
        if not picks:
            continue
        ids[t, :len(picks)] = picks
        with np.errstate(invalid="ignore"):
            p = np.exp(l[t] - l[t, picks[0]])
        weights[t, :len(picks)] = p[picks] / (p[picks].sum() if normalize else p[p == p].sum() if not np.isnan(l[t]).any() else np.nan)
    flat = ids.reshape(-1)
    counts = np.array([(flat == e).sum() for e in range(experts)], np.int32)
    order = np.full(tokens * topk, -1, np.int32)
    slots = [s for e in range(experts) for s in np.nonzero(flat == e)[0]]
    order[:len(slots)] = slots
    return weights, ids, counts, order


def route_backward(logits, ids, dweights, normalize: bool, mask=None):
    """Gradient of sum(dweights * weights) with respect to the logits, the picks held fixed."""
    l = np.array(logits, dtype=np.float64)
    if mask is not None:
        l[np.asarray(mask) == 0] = -np.inf
    d = np.zeros_like(l)
    for t in range(l.shape[0]):
        at = ids[t][ids[t] >= 0]
        if at.size == 0:
            continue
        g = np.asarray(dweights, np.float64)[t][ids[t] >= 0]
        p = np.exp(l[t] - l[t].max())
        if normalize:
            q = np.zeros_like(p)
            q[at] = p[at]
            p = q
        p /= p.sum()
        d[t] = -p * (g * p[at]).sum()
        d[t, at] += g * p[at]
    return d


def moe_layer(x, router, up, down, topk: int, normalize: bool, mask=None):
    """(y, bound): the layer in 64 bits, and for every output the sum of the
    magnitudes that are added up for it (what rounding errors scale with)."""
    x, router = np.asarray(x, np.float64), np.asarray(router, np.float64)
    w, ids, _, _ = route(x @ router.T, topk, normalize, mask)
    y, bound = np.zeros_like(x), np.zeros_like(x)
    for t in range(x.shape[0]):
        for j in range(topk):
            e = ids[t, j]
            if e < 0:
                continue
            u, d = np.asarray(up[e], np.float64), np.asarray(down[e], np.float64)
            i = d.shape[1]
            both, size = u @ x[t], np.abs(u) @ np.abs(x[t])
            gate, lift = both[:i], both[i:]
            s = 1 / (1 + np.exp(-gate))
            y[t] += w[t, j] * (d @ (gate * s * lift))
            # silu' is at most 1.1; the sums behind gate and lift are as large as `size`
            bound[t] += w[t, j] * (np.abs(d) @ (1.1 * size[:i] * np.abs(lift) + np.abs(gate * s) * size[i:] + np.abs(gate * s * lift)))
    return y, bound


# ---- 8-bit values with a scale for 128 of them, and what is made of them ----------

F8_BLOCK = 128
E4M3 = np.array([(m / 8) * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127])


def _f8_scale(top):
    """(exponents, bad) for blocks with those largest magnitudes."""
    bad = ~np.isfinite(top)
    e = np.full(top.shape, -127)
    for x in range(-126, 128):                      # the first with top <= 448 * 2^x
        e[top > 448.0 * 2.0 ** (x - 1)] = x
    return np.where(bad, 0, e), bad


def _f8_codes(v, e, bad):
    a = np.abs(np.where(bad, 0.0, v)) * 2.0 ** -e.astype(np.float64)
    mids = (E4M3[1:] + E4M3[:-1]) / 2
    code = np.searchsorted(mids, a, side="left")    # a tie goes to the lower code ...
    tie = (code < 126) & (a == mids[np.minimum(code, 125)])
    code = code + (tie & (code % 2 == 1))           # ... unless that one is odd
    return (code + 128 * (np.signbit(v) & ~bad)).astype(np.uint8)


def f8_quantize(x, tiles: bool = False):
    """(codes, scales) of the rows of x, as they are stored; with `tiles` 128 x 128 values share a scale."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    nb = -(-cols // F8_BLOCK)
    v = np.zeros((rows, nb * F8_BLOCK))
    v[:, :cols] = x
    v = v.reshape(rows, nb, F8_BLOCK)
    with np.errstate(invalid="ignore"):
        top = np.abs(v).max(axis=2, initial=0.0)    # NaN where a block holds one
        if tiles:
            for r in range(0, rows, F8_BLOCK):
                top[r:r + F8_BLOCK] = top[r:r + F8_BLOCK].max(axis=0)
    e, bad = _f8_scale(top)
    codes = _f8_codes(v, e[..., None], bad[..., None]).reshape(rows, -1)
    scales = np.zeros((rows, -(-nb // 4) * 4), np.uint8)
    scales[:, :nb] = np.where(bad, 255, e + 127)
    return codes, scales


def f8_values(codes, scales, cols: int):
    mags = np.append(E4M3, np.nan)
    v = mags[codes % 128] * np.where(codes >= 128, -1.0, 1.0)
    s = np.exp2(scales.astype(np.float64) - 127)
    s[scales == 255] = np.nan
    return (v * np.repeat(s, F8_BLOCK, axis=1)[:, :codes.shape[1]])[:, :cols]


def expert_blocks(counts, rows: int, block: int = 128):
    """(blocks before each expert, [(first row, rows, expert)]) for rows in expert order."""
    starts, out, at = [0], [], 0
    for e, c in enumerate(counts):
        n = min(max(int(c), 0), rows - at)
        out += [(at + i, min(block, n - i), e) for i in range(0, n, block)]
        at += n
        starts.append(len(out))
    return starts, out


def balance(logits, ids, mask=None):
    """(loss, counts, probs, rows) in 64 bits."""
    l, ids = np.array(logits, np.float64), np.asarray(ids)
    tokens, experts = l.shape
    if mask is not None:
        l[np.asarray(mask) == 0] = -np.inf
    probs, counts, rows = np.zeros(experts), np.zeros(experts, np.int32), 0
    for t in range(tokens):
        if not (np.isnan(l[t]).any() or (l[t] > -np.inf).any()):
            continue
        rows += 1
        with np.errstate(invalid="ignore"):
            p = np.exp(l[t] - l[t].max())
            probs += p / p.sum()
        for e in ids[t]:
            if 0 <= e < experts:
                counts[e] += 1
    probs /= max(rows, 1)
    loss = float((counts * probs).sum() * experts / counts.sum()) if counts.sum() else 0.0
    return loss, counts, probs, rows


def balance_backward(logits, counts, rows, dloss, dprobs=None, mask=None):
    """The gradient of dloss * loss + sum(dprobs * probs) with respect to the logits, the counts held fixed."""
    l, counts = np.array(logits, np.float64), np.asarray(counts, np.float64)
    if mask is not None:
        l[np.asarray(mask) == 0] = -np.inf
    v = dloss * counts * (l.shape[1] / counts.sum()) if counts.sum() else np.zeros(l.shape[1])
    v = v + (0.0 if dprobs is None else np.asarray(dprobs, np.float64))
    d = np.zeros_like(l)
    for t in range(l.shape[0]):
        if np.isnan(l[t]).any() or (l[t] > -np.inf).any():
            with np.errstate(invalid="ignore"):
                p = np.exp(l[t] - l[t].max())
                p /= p.sum()
            d[t] = p * (v - (v * p).sum()) / rows
    return d
