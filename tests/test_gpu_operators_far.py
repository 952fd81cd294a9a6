"""GPU: the operators at sizes and values further out: a long k that is shared
out, many tokens, experts with many tokens, rows that start anywhere, offsets
past 32 bits, values that are not finite.  Whole results must be equal;
floating ones carry the bounds that tests/test_gpu_operators.py derives.
"""

import numpy as np
import pytest

from oracle import operators as O
from test_gpu_operators import TINY, ULP, _logits, _np, _packed, _to, _torch, _type, ops  # noqa: F401

pytestmark = pytest.mark.gpu


# every number of steps that a wave of the few-row form holds, with whole and broken last ones; k shared out
# between workgroups, evenly and not; both forms of many rows next to them
LONG = [(1, 16, 1024), (5, 33, 1025), (16, 40, 2048), (17, 31, 2900), (33, 64, 3333), (20, 70, 5120), (49, 20, 5500), (64, 17, 7000),
        (8, 500, 8192), (64, 100, 8193), (7, 33, 20000), (1, 1, 65536), (65, 130, 4097), (200, 300, 5000), (129, 257, 9000)]


@pytest.mark.parametrize("m,n,k", LONG)
def test_product_with_a_long_k(ops, m, n, k):   # noqa: F811
    print(f"[operators] product {m}x{n}x{k}", flush=True)
    rng = np.random.default_rng(m + n + k)
    # scale 1: whole and half numbers up to 6, sums in quarters below 2^22
    a, av = _packed(rng, m, k, 127, 127)
    b, bv = _packed(rng, n, k, 127, 127)
    want = av @ bv.T
    assert (np.abs(av) @ np.abs(bv).T).max() < 2.0 ** 22
    np.testing.assert_array_equal(_np(ops.matmul(a, b, _torch().float32)), want)
    a, av = _packed(rng, m, k)
    b, bv = _packed(rng, n, k, 116, 124)
    want, size = av @ bv.T, np.abs(av) @ np.abs(bv).T
    for dtype in ("bf16", "f16"):
        got = _np(ops.matmul(a, b, _type(dtype)))
        with np.errstate(over="ignore"):
            held = np.abs(want) < 6e4 if dtype == "f16" else np.abs(want) < np.inf
        bound = (k + 2) * 2.0 ** -24 * size + ULP[dtype] * np.abs(want) * 1.01 + TINY[dtype]
        assert (np.abs(got - want) <= bound)[held].all()


def test_shared_out_product_of_not_numbers_into_a_view_and_in_a_graph(ops):   # noqa: F811
    print("[operators] shared-out product: NaN, view, graph", flush=True)
    t = _torch()
    rng = np.random.default_rng(1)
    m, n, k = 70, 90, 6100
    a, av = _packed(rng, m, k, 127, 127)
    b, bv = _packed(rng, n, k, 127, 127)
    room = t.full((m, n + 9), 5.0, device="cuda")
    ops.matmul(a, b, t.float32, out=room[:, 4:4 + n])
    want = np.full((m, n + 9), 5.0)
    want[:, 4:4 + n] = av @ bv.T
    np.testing.assert_array_equal(_np(room), want)
    graph = t.cuda.CUDAGraph()
    t.cuda.synchronize()
    with t.cuda.graph(graph):
        out = ops.matmul(a, b, t.float32)
    for i in range(4):
        other, ov = _packed(rng, m, k, 127, 127)
        a.codes.copy_(other.codes)
        eager = ops.matmul(other, b, t.float32)
        graph.replay()
        t.cuda.synchronize()
        assert t.equal(out, eager), i
        np.testing.assert_array_equal(_np(out), ov @ bv.T)
    a.scales[69, 190] = 255                                   # the last block of the last row
    got = _np(ops.matmul(a, b, t.bfloat16))
    np.testing.assert_array_equal(np.isnan(got), np.arange(m)[:, None].repeat(n, 1) == 69)


def test_shared_out_product_asks_for_its_workspace(ops):   # noqa: F811
    from paper_2606_07019_amd import pccl as P
    print("[operators] workspace of a shared-out product", flush=True)
    need = P.pccl_mx_matmul_workspace(ops.h, 70, 90, 6100)
    assert need >= 2 * 70 * 90 * 4 and P.pccl_mx_matmul_workspace(ops.h, 70, 90, 100) == 0
    p = _torch().zeros(1 << 20, dtype=_torch().uint8, device="cuda").data_ptr()
    for space, size, name in ((None, 0, "EINVAL"), (p, need - 1, "ENOMEM")):
        with pytest.raises(P.PcclError) as e:
            P.pccl_mx_matmul(ops.h, p, p, p, p, 70, 90, 6100, p, 0, 90, space, size)
        assert e.value.name == "PCCL_" + name


@pytest.mark.parametrize("tokens,experts,topk", [(32768, 5, 2), (32769, 64, 1), (40001, 24, 3), (70001, 3, 3)])
def test_route_many_tokens(ops, tokens, experts, topk):   # noqa: F811
    print(f"[operators] route {tokens}x{experts} top {topk}", flush=True)
    t = _torch()
    rng = np.random.default_rng(tokens)
    l = _logits(rng, tokens, experts, "bf16", True)
    mask = t.from_numpy((rng.random(tokens) > 0.2).astype(np.uint8)).cuda()
    for normalize in (True, False):
        w, ids, counts, order = ops.route(l, topk, normalize=normalize, mask=mask)
        ww, wi, wc, wo = O.route(_np(l), topk, normalize, mask.cpu().numpy())
        np.testing.assert_array_equal(ids.cpu().numpy(), wi)
        np.testing.assert_array_equal(counts.cpu().numpy(), wc)
        np.testing.assert_array_equal(order.cpu().numpy(), wo)
        assert (np.abs(_np(w) - ww) <= 2.0 ** -19 * ww + 1e-30).all()


# experts with more tokens than one, two and four tiles of 16; waves with tiles of their own (few blocks of k, many
# experts), with one and with four tiles of tokens; inner and hidden sizes that end within a step and a block
MANY = [(256, 2, 1, 72, 40), (150, 2, 2, 392, 136), (256, 3, 2, 1000, 296), (64, 128, 8, 512, 256), (256, 128, 8, 512, 256),
        (40, 128, 6, 520, 264), (256, 1, 1, 2056, 648), (5, 130, 20, 136, 1000)]


@pytest.mark.parametrize("weights", ["same", "mx"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("tokens,experts,topk,hidden,inter", MANY)
def test_layer_of_many(ops, tokens, experts, topk, hidden, inter, dtype, weights):   # noqa: F811
    from paper_2606_07019_amd.operators import MX
    t = _torch()
    print(f"[operators] layer {tokens} of {experts}/{topk}, {hidden}x{inter} {dtype} {weights}", flush=True)
    rng = np.random.default_rng(tokens + experts)
    x = _to(rng.normal(size=(tokens, hidden)), dtype)
    router = _to(rng.normal(size=(experts, hidden)) * 2 / np.sqrt(hidden), dtype)
    up, down = (_to(rng.normal(size=s).astype(np.float32) / np.sqrt(s[2]), dtype) for s in ((experts, 2 * inter, hidden), (experts, hidden, inter)))
    mask = t.from_numpy((rng.random(tokens) > 0.1).astype(np.uint8)).cuda()
    if weights == "mx":
        def pack(w):
            q = ops.quantize(w.view(-1, w.shape[2]))
            return MX(q.codes.view(experts, w.shape[1], -1), q.scales.view(experts, w.shape[1], -1), w.shape[2])
        args = [pack(up), pack(down)]
        values = [O.mx_values(q.codes.cpu().numpy().reshape(-1, q.codes.shape[2]), q.scales.cpu().numpy().reshape(-1, q.scales.shape[2]),
                              q.cols).reshape(experts, -1, q.cols) for q in args]
    else:
        args = [up, down]
        values = [_np(v) for v in args]
    got = _np(ops.moe_layer(x, router, *args, topk, mask=mask))
    want, size = O.moe_layer(_np(x), _np(router), *values, topk, True, mask.cpu().numpy())
    room = ((hidden + inter + topk) * 2.0 ** -24 + 2.0 ** -16) * size + 2.0 ** -24
    assert (np.abs(got - want) <= room + ULP[dtype] * np.abs(want) * 1.01 + TINY[dtype]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_layer_of_rows_that_start_anywhere(ops, dtype):   # noqa: F811
    print(f"[operators] layer, operands off alignment, {dtype}", flush=True)
    t = _torch()
    rng = np.random.default_rng(12)
    x, router, up, down = (_to(rng.normal(size=s) * 0.2, dtype) for s in ((21, 136), (6, 136), (6, 80, 136), (6, 136, 40)))

    def off(a):   # the same values, two bytes further on
        room = t.empty(a.numel() + 1, dtype=a.dtype, device="cuda")
        room[1:].copy_(a.reshape(-1))
        return room[1:].view(a.shape)

    want = ops.moe_layer(x, router, up, down, 2)
    for which in range(1, 16):
        got = ops.moe_layer(*(off(a) if which >> i & 1 else a for i, a in enumerate((x, router, up, down))), 2)
        assert t.equal(got, want), which   # the products are the same ones in the same order


@pytest.mark.parametrize("weights", ["same", "mx"])
def test_layer_keeps_infinities_and_nan_to_their_tokens(ops, weights):   # noqa: F811
    print(f"[operators] layer, tokens that are not finite, {weights}", flush=True)
    from paper_2606_07019_amd.operators import MX
    t = _torch()
    rng = np.random.default_rng(13)
    x, router, up, down = (_to(rng.normal(size=s) * 0.2, "bf16") for s in ((30, 160), (5, 160), (5, 96, 160), (5, 160, 48)))
    if weights == "mx":
        up, down = (MX(*(f.view(5, w.shape[1], -1) for f in ops.quantize(w.view(-1, w.shape[2]))[:2]), w.shape[2]) for w in (up, down))
    want = ops.moe_layer(x, router, up, down, 2)
    bad = x.clone()
    bad[3, 7], bad[11, 0], bad[29, 159] = float("inf"), float("nan"), float("-inf")
    got = ops.moe_layer(bad, router, up, down, 2)
    fine = t.ones(30, dtype=t.bool, device="cuda")
    fine[[3, 11, 29]] = False
    assert t.equal(got[fine], want[fine]) and t.isnan(got[11]).all()
    assert not t.isfinite(got[3]).any() and not t.isfinite(got[29]).any()
    mask = fine.to(t.uint8)                                   # masked tokens are not looked at
    got = ops.moe_layer(bad, router, up, down, 2, mask=mask)
    assert t.equal(got[fine], want[fine]) and (got[~fine] == 0).all()


# ---- offsets past 32 bits -----------------------------------------------------------

def test_packing_past_32_bit_offsets(ops):   # noqa: F811
    print("[operators] packing 70000x70000", flush=True)
    t = _torch()
    n = 70000
    x = t.empty((n, n), dtype=t.bfloat16, device="cuda").normal_()
    rows, cols = ops.quantize_both(x)
    one = ops.quantize(x)
    for q in (rows, one):
        end = ops.quantize(x[n - 300:])
        assert t.equal(q.codes[n - 300:], end.codes) and t.equal(q.scales[n - 300:], end.scales)
    end = ops.quantize(x[:, n - 300:].t().contiguous())
    assert t.equal(cols.codes[n - 300:], end.codes) and t.equal(cols.scales[n - 300:], end.scales)
    whole = ops.dequantize(one, t.bfloat16)
    from paper_2606_07019_amd.operators import MX
    assert t.equal(whole[n - 300:], ops.dequantize(MX(one.codes[n - 300:].contiguous(), one.scales[n - 300:].contiguous(), n), t.bfloat16))


def test_product_past_32_bit_offsets(ops):   # noqa: F811
    print("[operators] product 70000x70000x40", flush=True)
    from paper_2606_07019_amd.operators import MX
    t = _torch()
    rng = np.random.default_rng(14)
    n, k = 70000, 40
    a, av = _packed(rng, n, k, 127, 127)
    b, bv = _packed(rng, n, k, 127, 127)
    y = ops.matmul(a, b, t.bfloat16)
    for r in (slice(0, 200), slice(n - 200, n)):
        want = av[r] @ bv.T
        assert (np.abs(_np(y[r]) - want) <= ULP["bf16"] * np.abs(want)).all()
    few = MX(a.codes[n - 9:].contiguous(), a.scales[n - 9:].contiguous(), k)
    assert t.equal(ops.matmul(few, b, t.bfloat16), y[n - 9:])


def test_layer_past_32_bit_offsets(ops):   # noqa: F811
    print("[operators] layer of 1024 experts, 13 GB of weights", flush=True)
    t = _torch()
    rng = np.random.default_rng(15)
    experts, hidden, inter = 1024, 2048, 1024
    x = _to(np.abs(rng.normal(size=(4, hidden))) + 0.1, "bf16")
    router = t.full((experts, hidden), -0.01, dtype=t.bfloat16, device="cuda")
    router[-3:] = _to(rng.random((3, hidden)) * 0.01, "bf16")
    up = t.zeros((experts, 2 * inter, hidden), dtype=t.bfloat16, device="cuda")
    down = t.zeros((experts, hidden, inter), dtype=t.bfloat16, device="cuda")
    up[-3:].normal_(std=hidden ** -0.5)
    down[-3:].normal_(std=inter ** -0.5)
    got = ops.moe_layer(x, router, up, down, 2)
    assert (got != 0).any(dim=1).all()
    # the others' logits are negative and not picked: normalized, the last three alone give the same result
    want, size = O.moe_layer(_np(x), _np(router[-3:]), _np(up[-3:]), _np(down[-3:]), 2, True, None)
    room = ((hidden + inter + 2) * 2.0 ** -24 + 2.0 ** -16) * size + 2.0 ** -24
    assert (np.abs(_np(got) - want) <= room + ULP["bf16"] * np.abs(want) * 1.01).all()
