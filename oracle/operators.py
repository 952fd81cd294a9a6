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
