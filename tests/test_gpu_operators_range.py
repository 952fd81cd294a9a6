"""Inner values of an expert layer beyond the range that holds them, and types
that the operators do not take."""

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2606_07019_amd.operators import Operators
    o = Operators(0)
    yield o
    o.close()


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype,size", [("bfloat16", 2.0 ** 66), ("float16", 2.0 ** 13)])
def test_layer_beyond_the_inner_range_is_infinite(ops, dtype, size, packed):
    # gate = up = size: 2^132 passes 32 bits' largest number, 2^26 the 2^24 that f16's parts hold
    import torch
    print(f"[operators] inner values of {size}^2 {dtype} packed {packed}", flush=True)
    kind = getattr(torch, dtype)
    x = torch.full((3, 64), size / 64, dtype=kind, device="cuda")
    up = torch.ones((1, 64, 64), dtype=kind, device="cuda")
    down = torch.ones((1, 64, 32), dtype=kind, device="cuda")
    router = torch.zeros((1, 64), dtype=kind, device="cuda")
    if packed:
        from paper_2606_07019_amd.operators import MX
        up, down = (MX(q.codes[None], q.scales[None], q.cols) for q in (ops.quantize(up[0]), ops.quantize(down[0])))
    x[1] = 1.0 / 64                                              # another token's values stay what they are
    y = ops.moe_layer(x, router, up, down, 1)
    assert torch.isposinf(y[0]).all() and torch.isposinf(y[2]).all()
    assert torch.isfinite(y[1]).all()


def test_types_that_are_not_taken(ops):
    import torch
    q = ops.quantize(torch.ones((2, 32), device="cuda"))
    for bad in (torch.float64, torch.int32, None):
        with pytest.raises(ValueError):
            ops.dequantize(q, bad)
        with pytest.raises(ValueError):
            ops.matmul(q, q, bad)


@pytest.mark.parametrize("normalize", [True, False])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_an_infinite_logit_leaves_no_weights(ops, dtype, normalize):
    # infinity less infinity: the row's softmax is no number, its picks are what they are, and no other row knows
    import torch
    print(f"[operators] infinite logit {dtype} {normalize}", flush=True)
    l = torch.zeros((3, 70), dtype=getattr(torch, dtype), device="cuda")
    l[1, 66], l[1, 4], l[2, 5] = float("inf"), 3.0, 1.0
    w, ids, counts, _ = ops.route(l, 2, normalize=normalize)
    assert ids.tolist() == [[0, 1], [66, 4], [5, 0]]
    assert torch.isnan(w[1]).all() and torch.isfinite(w[[0, 2]]).all()
    d = ops.route_backward(l, w, ids, torch.ones_like(w), normalize=normalize)
    assert torch.isnan(d[1, [66, 4]]).all() and torch.isfinite(d[[0, 2]]).all()
