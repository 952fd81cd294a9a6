"""GPU: the operators at the ends of a collective against the 64-bit oracle.

Codes, scales, picks, counts and orders are whole numbers and must be equal.
Floating results carry bounds derived from their arithmetic: a sum of n
products in 32 bits is within (n + 2) 2^-24 of the sum of the products'
magnitudes, a result rounded to a type within half its last place.
"""

import numpy as np
import pytest

from oracle import operators as O

pytestmark = pytest.mark.gpu

ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}   # half a last place, relative
TINY = {"f32": 0.0, "bf16": 0.0, "f16": 2.0 ** -25}               # and below the normal numbers


def _torch():
    import torch
    return torch


def _type(name):
    t = _torch()
    return {"f32": t.float32, "bf16": t.bfloat16, "f16": t.float16}[name]


@pytest.fixture(scope="module")
def ops():
    from paper_2606_07019_amd.operators import Operators
    o = Operators(0)
    yield o
    o.close()


def _to(a, dtype="f32"):
    return _torch().from_numpy(np.ascontiguousarray(a)).to("cuda").to(_type(dtype))


def _np(t):
    return t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def _values(rng, rows, cols, dtype):
    """Values over the whole range of the type, ties, zeros, and blocks that are not finite, as the type holds them."""
    span = {"f32": 120, "bf16": 120, "f16": 12}[dtype]
    x = rng.normal(size=(rows, cols)) * np.exp2(rng.integers(-span, span, size=(rows, 1)))
    quarter = rng.integers(-32, 33, size=(rows, cols)) / 4.0     # on the codes and halfway between them
    x = np.where(rng.random((rows, 1)) < 0.4, quarter, x)
    x[rng.random((rows, cols)) < 0.02] = 0.0
    x[rng.random((rows, cols)) < 0.002] = np.inf
    x[rng.random((rows, cols)) < 0.002] = np.nan
    x[rng.random(rows) < 0.1] = 0.0
    if dtype != "f16":
        x[rng.random(rows) < 0.1] = -0.0
        small = rng.random(rows) < 0.1                           # below the normal numbers
        x[small] = (rng.integers(-127, 128, size=(int(small.sum()), cols))) * 2.0 ** -133
    return _to(x, dtype)


SHAPES = [(1, 1), (1, 32), (3, 31), (5, 33), (32, 128), (33, 129), (130, 257), (7, 1000), (300, 96), (128, 512)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_packing(ops, rows, cols, dtype):
    print(f"[operators] packing {rows}x{cols} {dtype}", flush=True)
    rng = np.random.default_rng(rows * 1000 + cols)
    x = _values(rng, rows, cols, dtype)
    for q, want in zip(ops.quantize_both(x), (_np(x), _np(x).T)):
        codes, scales = O.mx_quantize(want)
        np.testing.assert_array_equal(q.scales.cpu().numpy(), scales)
        np.testing.assert_array_equal(q.codes.cpu().numpy(), codes)
        for out in ("f32", "bf16"):                              # both hold every value
            np.testing.assert_array_equal(_np(ops.dequantize(q, _type(out))), O.mx_values(codes, scales, want.shape[1]))
    one = ops.quantize(x)
    both = ops.quantize_both(x)
    assert _torch().equal(one.codes, both[0].codes) and _torch().equal(one.scales, both[0].scales)
    cols_only = ops.quantize_columns(x)
    assert _torch().equal(cols_only.codes, both[1].codes) and _torch().equal(cols_only.scales, both[1].scales)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_packing_of_strided_and_unaligned_rows(ops, dtype):
    print(f"[operators] strided packing {dtype}", flush=True)
    rng = np.random.default_rng(3)
    whole = _values(rng, 70, 211, dtype)
    for x in (whole[:, 1:], whole[::2, 3:100], whole[5:6, 7:8], whole[:, 8:200]):
        for q, want in zip(ops.quantize_both(x), (_np(x), _np(x).T)):
            codes, scales = O.mx_quantize(want)
            np.testing.assert_array_equal(q.scales.cpu().numpy(), scales)
            np.testing.assert_array_equal(q.codes.cpu().numpy(), codes)


def test_unpacking_of_every_code_and_scale(ops):
    from paper_2606_07019_amd.operators import MX
    t = _torch()
    codes = np.tile(np.arange(256, dtype=np.uint8), (64, 1)).reshape(256, 64)
    scales = np.arange(1024, dtype=np.uint32).reshape(256, 4) // 4
    scales = scales.astype(np.uint8)
    q = MX(t.from_numpy(codes).cuda(), t.from_numpy(scales).cuda(), 128)
    want = O.mx_values(codes, scales, 128)
    with np.errstate(over="ignore"):                             # 2^127 times 2 and more passes the largest number
        for out in ("f32", "bf16"):
            np.testing.assert_array_equal(_np(ops.dequantize(q, _type(out))), want.astype(np.float32).astype(np.float64))
        np.testing.assert_array_equal(_np(ops.dequantize(q, t.float16)), want.astype(np.float16).astype(np.float64))


def _packed(rng, rows, cols, lo=120, hi=130):
    """Random packed rows and their values; what is stored behind a row is zero."""
    from paper_2606_07019_amd.operators import MX
    t = _torch()
    v = rng.choice(np.concatenate([O.MAGNITUDES, -O.MAGNITUDES]), size=(rows, cols))
    codes, _ = O.mx_quantize(np.concatenate([np.where(v == 0, 0, v), np.zeros((rows, 0))], axis=1) if cols else np.zeros((rows, 1)))
    pad = -(-cols // 128) * 128
    c = np.zeros((rows, pad), np.uint8)
    mags = np.searchsorted(O.MAGNITUDES, np.abs(v))
    c[:, :cols] = mags + 8 * (v < 0)
    codes = c[:, 0::2] | (c[:, 1::2] << 4)
    scales = np.zeros((rows, pad // 32), np.uint8)
    nb = -(-cols // 32)
    scales[:, :nb] = rng.integers(lo, hi + 1, size=(rows, nb))
    q = MX(t.from_numpy(codes).cuda(), t.from_numpy(scales).cuda(), cols)
    return q, O.mx_values(codes, scales, cols)


PRODUCTS = [(1, 1, 1), (1, 16, 128), (1, 17, 33), (3, 100, 129), (16, 64, 4096), (17, 40, 300), (33, 1000, 256), (48, 31, 1111),
            (64, 129, 640), (65, 1, 5), (65, 128, 128), (100, 130, 384), (129, 257, 700), (300, 520, 1025), (257, 64, 2048),
            (4100, 4200, 160)]


@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product_is_exact_on_whole_numbers(ops, m, n, k):
    # scale 2: all values are whole numbers up to 12, sums below 2^24
    print(f"[operators] product {m}x{n}x{k}, whole numbers", flush=True)
    rng = np.random.default_rng(m + 7 * n + 13 * k)
    a, av = _packed(rng, m, k, 128, 128)
    b, bv = _packed(rng, n, k, 128, 128)
    got = ops.matmul(a, b, _torch().float32)
    np.testing.assert_array_equal(_np(got), av @ bv.T)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m,n,k", PRODUCTS[:-1])
def test_product(ops, m, n, k, dtype):
    print(f"[operators] product {m}x{n}x{k} {dtype}", flush=True)
    rng = np.random.default_rng(m + 7 * n + 13 * k)
    a, av = _packed(rng, m, k)
    b, bv = _packed(rng, n, k, 116, 124)
    got, want = _np(ops.matmul(a, b, _type(dtype))), av @ bv.T
    bound = (k + 2) * 2.0 ** -24 * (np.abs(av) @ np.abs(bv).T) + ULP[dtype] * np.abs(want) * 1.01 + TINY[dtype]
    assert (np.abs(got - want) <= bound).all()


@pytest.mark.parametrize("m,n", [(5, 40), (200, 300)])
def test_product_of_blocks_that_are_not_numbers(ops, m, n):
    print(f"[operators] NaN blocks {m}x{n}", flush=True)
    rng = np.random.default_rng(5)
    a, av = _packed(rng, m, 320)
    b, bv = _packed(rng, n, 320)
    a.scales[m - 1, 3] = 255
    b.scales[2, 9] = 255
    got = _np(ops.matmul(a, b, _torch().bfloat16))
    nan = np.zeros((m, n), bool)
    nan[m - 1], nan[:, 2] = True, True
    np.testing.assert_array_equal(np.isnan(got), nan)


def test_product_into_a_view_and_of_nothing(ops):
    print("[operators] product into a view", flush=True)
    t = _torch()
    rng = np.random.default_rng(6)
    for m, n in ((20, 33), (140, 33)):
        a, av = _packed(rng, m, 64, 128, 128)
        b, bv = _packed(rng, n, 64, 128, 128)
        room = t.full((m, n + 8), 7.0, device="cuda")
        ops.matmul(a, b, t.float32, out=room[:, 3:3 + n])
        want = np.full((m, n + 8), 7.0)
        want[:, 3:3 + n] = av @ bv.T
        np.testing.assert_array_equal(_np(room), want)
    a, _ = _packed(rng, 0, 64)
    assert ops.matmul(a, b, t.float32).shape == (0, 33)
    a, _ = _packed(rng, 4, 0)
    b, _ = _packed(rng, 6, 0)
    assert (ops.matmul(a, b, t.bfloat16) == 0).all()


# ---- router ---------------------------------------------------------------------

ROUTES = [(1, 1, 1), (1, 64, 4), (2, 8, 8), (63, 61, 3), (64, 64, 8), (65, 65, 2), (200, 128, 8), (257, 200, 1), (130, 256, 32),
          (70, 300, 8), (129, 512, 6), (33, 1000, 5), (66, 1024, 32), (1000, 17, 17)]


def _logits(rng, tokens, experts, dtype, barred):
    l = rng.normal(size=(tokens, experts)) * 3
    l = np.where(rng.random((tokens, 1)) < 0.3, np.round(l), l)      # ties
    l[rng.random(tokens) < 0.1] = 0.0
    if barred:
        l[rng.random((tokens, experts)) < 0.4] = -np.inf
        l[rng.random(tokens) < 0.1] = -np.inf
    return _to(l, dtype)


@pytest.mark.parametrize("barred", [False, True])
@pytest.mark.parametrize("normalize", [True, False])
@pytest.mark.parametrize("tokens,experts,topk", ROUTES)
def test_route_and_its_gradient(ops, tokens, experts, topk, normalize, barred):
    t = _torch()
    for dtype in ("f32", "bf16", "f16"):
        print(f"[operators] route {tokens}x{experts} top {topk} {dtype} {normalize} {barred}", flush=True)
        rng = np.random.default_rng(tokens * 7 + experts)
        l = _logits(rng, tokens, experts, dtype, barred)
        mask = t.from_numpy((rng.random(tokens) > 0.2).astype(np.uint8)).cuda() if barred else None
        host = None if mask is None else mask.cpu().numpy()
        w, ids, counts, order = ops.route(l, topk, normalize=normalize, mask=mask)
        ww, wi, wc, wo = O.route(_np(l), topk, normalize, host)
        np.testing.assert_array_equal(ids.cpu().numpy(), wi)
        np.testing.assert_array_equal(counts.cpu().numpy(), wc)
        np.testing.assert_array_equal(order.cpu().numpy(), wo)
        # exp of a 32-bit difference d is off by |d| 2^-24 + 2^-22, sum and quotient by 2^-20 at most
        room = 2.0 ** -19
        assert (np.abs(_np(w) - ww) <= room * ww + 1e-30).all()
        g = t.from_numpy(rng.normal(size=(tokens, topk)).astype(np.float32)).cuda()
        d = _np(ops.route_backward(l, w, ids, g, normalize=normalize, mask=mask))
        want = O.route_backward(_np(l), wi, _np(g), normalize, host)
        size = np.abs(_np(g)).max(axis=1, keepdims=True) * 2
        assert (np.abs(d - want) <= room * size + ULP[dtype] * np.abs(want) * 1.01 + TINY[dtype]).all()


@pytest.mark.parametrize("normalize", [True, False])
def test_route_gradient_against_differences(ops, normalize):
    print("[operators] route gradient against differences", flush=True)
    rng = np.random.default_rng(11)
    l = rng.normal(size=(4, 9)).astype(np.float32)
    g = rng.normal(size=(4, 3)).astype(np.float32)
    w, ids, _, _ = ops.route(_to(l), 3, normalize=normalize)
    d = _np(ops.route_backward(_to(l), w, ids, _to(g), normalize=normalize))
    h = 1e-6
    for t in range(4):
        for e in range(9):
            f = []
            for s in (h, -h):
                m = l.astype(np.float64)
                m[t, e] += s
                f.append((O.route(m, 3, normalize)[0] * g).sum())
            assert abs((f[0] - f[1]) / (2 * h) - d[t, e]) < 1e-5   # 32-bit softmax: 2^-19 of |g| <= 3, and the differences' 1e-9


def test_route_not_a_number(ops):
    print("[operators] route with NaN", flush=True)
    l = np.zeros((2, 70))
    l[0, 66], l[0, 5], l[1, 3] = np.nan, 2.0, 1.0
    w, ids, counts, _ = ops.route(_to(l), 2)
    np.testing.assert_array_equal(ids.cpu().numpy(), [[66, 5], [3, 0]])
    assert np.isnan(_np(w)[0]).all() and np.isfinite(_np(w)[1]).all()


def test_route_strides_and_no_tokens(ops):
    print("[operators] route strided, empty", flush=True)
    t = _torch()
    rng = np.random.default_rng(8)
    room = _to(rng.normal(size=(80, 77)), "bf16")
    for l in (room[:, 1:66], room[::2, 3:5], room[7:8, :]):
        w, ids, counts, order = ops.route(l, 2, normalize=False)
        ww, wi, wc, wo = O.route(_np(l), 2, False)
        np.testing.assert_array_equal(ids.cpu().numpy(), wi)
        np.testing.assert_array_equal(order.cpu().numpy(), wo)
        d = _np(ops.route_backward(l, w, ids, t.ones_like(w), normalize=False))
        want = O.route_backward(_np(l), wi, np.ones(wi.shape), False)
        assert (np.abs(d - want) <= 2.0 ** -18 + ULP["bf16"] * np.abs(want) * 1.01).all()
    _, ids, counts, order = ops.route(_to(np.zeros((0, 12))), 3)
    assert ids.shape == (0, 3) and order.numel() == 0 and (counts == 0).all()


# ---- mixture-of-experts layer ------------------------------------------------------

LAYERS = [(1, 1, 1, 8, 8), (1, 8, 2, 256, 128), (1, 64, 4, 520, 200), (3, 4, 4, 33, 17), (16, 16, 2, 128, 136), (17, 5, 3, 384, 96),
          (64, 8, 8, 256, 72), (64, 40, 2, 96, 40), (100, 3, 2, 160, 64), (256, 70, 4, 64, 48), (200, 1, 1, 40, 24)]


@pytest.mark.parametrize("weights", ["same", "mx"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("tokens,experts,topk,hidden,inter", LAYERS)
def test_layer(ops, tokens, experts, topk, hidden, inter, dtype, weights):
    from paper_2606_07019_amd.operators import MX
    t = _torch()
    print(f"[operators] layer {tokens} of {experts}/{topk}, {hidden}x{inter} {dtype} {weights}", flush=True)
    rng = np.random.default_rng(tokens + experts)
    x = _to(rng.normal(size=(tokens, hidden)), dtype)
    router = _to(rng.normal(size=(experts, hidden)) * 2 / np.sqrt(hidden), dtype)
    up = rng.normal(size=(experts, 2 * inter, hidden)) / np.sqrt(hidden)
    down = rng.normal(size=(experts, hidden, inter)) / np.sqrt(inter)
    normalize = tokens % 2 == 1
    mask = t.from_numpy((rng.random(tokens) > 0.2).astype(np.uint8)).cuda() if tokens > 2 else None
    if weights == "mx":
        pairs = [[O.mx_quantize(p) for p in w] for w in (up, down)]
        packed = [MX(t.from_numpy(np.stack([c for c, _ in p])).cuda(), t.from_numpy(np.stack([s for _, s in p])).cuda(), n)
                  for p, n in zip(pairs, (hidden, inter))]
        values = [np.stack([O.mx_values(c, s, n) for c, s in p]) for p, n in zip(pairs, (hidden, inter))]
        got = ops.moe_layer(x, router, *packed, topk, normalize=normalize, mask=mask)
    else:
        tensors = [_to(up, dtype), _to(down, dtype)]
        values = [_np(v) for v in tensors]
        got = ops.moe_layer(x, router, *tensors, topk, normalize=normalize, mask=mask)
    want, size = O.moe_layer(_np(x), _np(router), *values, topk, normalize, None if mask is None else mask.cpu().numpy())
    # 32-bit sums over hidden and inner values, the weights' 2^-18 and the inner values' two parts (2^-17, 2^-28 at least)
    room = ((hidden + inter + topk) * 2.0 ** -24 + 2.0 ** -16) * size + 2.0 ** -24
    assert (np.abs(_np(got) - want) <= room + ULP[dtype] * np.abs(want) * 1.01 + TINY[dtype]).all()
    if mask is not None:
        assert (got[mask == 0] == 0).all()


def test_layer_with_large_inner_values(ops):
    # gate and up near 2^10: their product passes f16's largest number, the result does not
    print("[operators] large inner values", flush=True)
    rng = np.random.default_rng(2)
    x = _to(np.ones((2, 64)) * 32, "f16")
    up, down = _to(np.full((1, 32, 64), 0.5), "f16"), _to(rng.normal(size=(1, 64, 16)) * 2.0 ** -10, "f16")
    router = _to(np.zeros((1, 64)), "f16")
    got = _np(ops.moe_layer(x, router, up, down, 1))
    want, size = O.moe_layer(_np(x), _np(router), _np(up), _np(down), 1, True)
    assert np.abs(want).max() > 1000
    assert (np.abs(got - want) <= 2.0 ** -16 * size + ULP["f16"] * np.abs(want) * 1.01).all()


def test_layer_with_every_token_masked(ops):
    print("[operators] every token masked", flush=True)
    t = _torch()
    x = t.ones((5, 64), dtype=t.bfloat16, device="cuda")
    z = lambda *s: t.ones(s, dtype=t.bfloat16, device="cuda")   # noqa: E731
    y = ops.moe_layer(x, z(4, 64), z(4, 64, 64), z(4, 64, 32), 2, mask=t.zeros(5, dtype=t.uint8, device="cuda"))
    assert (y == 0).all()


def test_layer_of_strided_tokens(ops):
    print("[operators] strided tokens", flush=True)
    rng = np.random.default_rng(4)
    room = _to(rng.normal(size=(6, 140)), "bf16")
    router, up, down = (_to(rng.normal(size=s) * 0.2, "bf16") for s in ((4, 64), (4, 64, 64), (4, 64, 32)))
    for x in (room[:, 1:65], room[:, 8:72], room[::2, 4:68]):
        got = ops.moe_layer(x, router, up, down, 2)
        assert _torch().equal(got, ops.moe_layer(x.contiguous(), router, up, down, 2))


# ---- streams, graphs, refusals -------------------------------------------------------

def test_on_another_stream_and_in_a_graph(ops):
    print("[operators] stream and graph", flush=True)
    t = _torch()
    rng = np.random.default_rng(9)
    x = _to(rng.normal(size=(130, 256)), "bf16")
    w, _ = _packed(rng, 96, 256)
    router, up, down = (_to(rng.normal(size=s) * 0.1, "bf16") for s in ((8, 256), (8, 128, 256), (8, 256, 64)))

    def step(v):
        y = ops.matmul(ops.quantize(v), w, t.bfloat16)
        z = ops.moe_layer(v[:16], router, up, down, 2)
        return [y, z, *ops.route(v, 4)]

    want = [a.clone() for a in step(x)]
    side = t.cuda.Stream()
    side.wait_stream(t.cuda.current_stream())
    with t.cuda.stream(side):
        got = step(x)
    side.synchronize()
    assert all(t.equal(a, b) for a, b in zip(got, want))
    held = x.clone()
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        got = step(held)
    for k in range(4):
        y = _to(rng.normal(size=(130, 256)), "bf16")
        want = step(y)
        held.copy_(y)
        graph.replay()
        t.cuda.synchronize()
        assert all(t.equal(a, b) for a, b in zip(got, want)), k


def test_refusals(ops):
    from paper_2606_07019_amd import pccl as P
    from paper_2606_07019_amd.operators import MX
    t = _torch()
    print("[operators] refusals", flush=True)

    def status(fn, *a, **k):
        try:
            fn(*a, **k)
            return "OK"
        except P.PcclError as e:
            assert str(e).split(": ", 1)[1]
            return e.name[len("PCCL_"):]

    h = ops.h
    room = t.zeros(1 << 16, dtype=t.uint8, device="cuda")
    p = room.data_ptr()
    Q = P.pccl_mx_quantize
    assert status(Q, h, p, 7, 4, 4, 4, p, p) == "EINVAL"                   # type
    assert status(Q, h, None, 0, 4, 4, 4, p, p) == "EINVAL"
    assert status(Q, h, p + 1, 0, 4, 4, 4, p, p) == "EINVAL"
    assert status(Q, h, p, 0, 4, 4, 3, p, p) == "EINVAL"                   # stride below the row
    assert status(Q, h, p, 0, 4, 4, 4) == "EINVAL"                         # no output
    assert status(Q, h, p, 0, 4, 4, 4, p, None) == "EINVAL"
    assert status(Q, h, p, 0, 4, 4, 4, p + 8, p) == "EINVAL"
    assert status(Q, h, p, 0, 4, 4, 4, None, None, p, p + 2) == "EINVAL"
    assert status(Q, h, p, 0, 1 << 31, 4, 4, p, p) == "EUNSUPPORTED"
    assert status(Q, h, None, 0, 0, 4, 4, p, p) == "OK"
    D = P.pccl_mx_dequantize
    assert status(D, h, None, p, 4, 4, p, 0, 4) == "EINVAL"
    assert status(D, h, p, p, 4, 4, p, 0, 2) == "EINVAL"
    M = P.pccl_mx_matmul
    assert status(M, h, None, p, p, p, 4, 4, 4, p, 0, 4) == "EINVAL"
    assert status(M, h, p, p, p, p + 1, 4, 4, 4, p, 0, 4) == "EINVAL"
    assert status(M, h, p, p, p, p, 4, 4, 4, p, 0, 3) == "EINVAL"
    assert status(M, h, p, p, p, p, 4, 4, 1 << 31, p, 0, 4) == "EUNSUPPORTED"
    assert status(M, h, None, None, None, None, 0, 4, 4, None, 0, 4) == "OK"
    R = P.pccl_moe_route
    assert status(R, h, p, 0, 4, 0, 4, 1, 1, None, p, p, p, p) == "EINVAL"  # no experts
    assert status(R, h, p, 0, 4, 4, 4, 5, 1, None, p, p, p, p) == "EINVAL"  # more picks than experts
    assert status(R, h, p, 0, 4, 4, 4, 0, 1, None, p, p, p, p) == "EINVAL"
    assert status(R, h, p, 0, 4, 1025, 1025, 2, 1, None, p, p, p, p) == "EUNSUPPORTED"
    assert status(R, h, p, 0, 4, 64, 64, 33, 1, None, p, p, p, p) == "EUNSUPPORTED"
    assert status(R, h, p, 0, 1 << 30, 64, 64, 4, 1, None, p, p, p, p) == "EUNSUPPORTED"
    assert status(R, h, p, 0, 4, 4, 4, 2, 1, None, None, p, p, p) == "EINVAL"
    assert status(R, h, p, 0, 100, 4, 4, 2, 1, None, p, p, p, p) == "EINVAL"              # workspace missing
    assert status(R, h, p, 0, 100, 4, 4, 2, 1, None, p, p, p, p, p, 16) == "ENOMEM"
    assert status(R, h, p, 0, 100, 4, 4, 2, 1, None, p, p, p, p, p + 64, 4096) == "EINVAL"
    B = P.pccl_moe_route_backward
    assert status(B, h, None, 0, 4, 4, 4, 2, 0, None, p, p, p, p, 4) == "EINVAL"          # logits are read
    assert status(B, h, p, 0, 4, 4, 4, 2, 0, None, p, None, p, p, 4) == "EINVAL"
    L = P.pccl_moe_layer
    assert status(L, h, p, 0, 8, 2, 4, 2, 8, 8, 1, None, p, p, None, p, None, p, 8, p, 1 << 16) == "EINVAL"      # f32
    assert status(L, h, p, 1, 8, 257, 4, 2, 8, 8, 1, None, p, p, None, p, None, p, 8, p, 1 << 16) == "EUNSUPPORTED"
    assert status(L, h, p, 1, 8, 2, 4, 2, 8, 8, 1, None, p, p, p, p, None, p, 8, p, 1 << 16) == "EINVAL"         # one packed
    assert status(L, h, p, 1, 8, 2, 4, 2, 0, 8, 1, None, p, p, None, p, None, p, 8, p, 1 << 16) == "EINVAL"
    assert status(L, h, p, 1, 8, 2, 4, 2, 8, 8, 1, None, p, p, None, p, None, p, 8, p, 64) == "ENOMEM"
    assert status(L, h, None, 1, 8, 0, 4, 2, 8, 8, 1, None, p, p, None, p, None, None, 8) == "OK"
    # tensors
    x = t.zeros((4, 8), device="cuda")
    for bad in (lambda: ops.quantize(x.cpu()), lambda: ops.quantize(x.double()), lambda: ops.quantize(x.t()),
                lambda: ops.quantize(x[0]), lambda: ops.matmul(ops.quantize(x), ops.quantize(x[:, :4]), t.float32),
                lambda: ops.matmul(MX(room[:64].view(1, 64), room[:8].view(1, 8), 8), ops.quantize(x), t.float32),
                lambda: ops.route(x, 2, mask=t.ones(3, dtype=t.uint8, device="cuda")),
                lambda: ops.moe_layer(x, x, x, x, 1)):
        with pytest.raises(ValueError):
            bad()
