"""GPU: the operators under torch's automatic differentiation.  The router's
weights carry its gradient; what has no gradient says so where one is asked
for, and never returns a wrong one or none in silence."""

import numpy as np
import pytest

from oracle import operators as O
from test_gpu_operators import _logits, _np, _to, _torch, _type, ops  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("normalize", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("tokens,experts,topk", [(1, 8, 2), (130, 61, 3), (70, 300, 8)])
def test_router_learns(ops, tokens, experts, topk, dtype, normalize):   # noqa: F811
    print(f"[operators] autograd of route {tokens}x{experts} top {topk} {dtype} {normalize}", flush=True)
    t = _torch()
    rng = np.random.default_rng(tokens + experts)
    l = _logits(rng, tokens, experts, dtype, True).requires_grad_()
    mask = t.from_numpy((rng.random(tokens) > 0.2).astype(np.uint8)).cuda()
    g = _to(rng.normal(size=(tokens, topk)))
    w, ids, counts, order = ops.route(l, topk, normalize=normalize, mask=mask)
    assert w.requires_grad and not (ids.requires_grad or counts.requires_grad or order.requires_grad)
    with t.no_grad():
        plain = ops.route(l, topk, normalize=normalize, mask=mask)
    assert not plain[0].requires_grad
    for a, b in zip((w, ids, counts, order), plain):
        assert t.equal(a, b)
    (w * g).sum().backward()
    assert l.grad.dtype == l.dtype
    assert t.equal(l.grad, ops.route_backward(l.detach(), plain[0], ids, g, normalize=normalize, mask=mask))
    assert (np.abs(_np(l.grad)).max() > 0) == (np.abs(O.route_backward(_np(l.detach()), _np(ids), _np(g), normalize, _np(mask))).max() > 0)


def test_router_learns_through_what_computes_its_logits(ops):   # noqa: F811
    print("[operators] autograd through a router's product", flush=True)
    t = _torch()
    rng = np.random.default_rng(3)
    x, r = _to(rng.normal(size=(20, 32))), _to(rng.normal(size=(9, 32)) * 0.3).requires_grad_()
    w, ids, _, _ = ops.route((x @ r.t())[:, 1:], 2)
    w[:, 0].sum().backward()                                     # a gradient with strides and zeros
    logits = _np(x) @ _np(r.detach()).T
    d = O.route_backward(logits[:, 1:], _np(ids), np.tile([1.0, 0.0], (20, 1)), True)
    want = np.concatenate([np.zeros((20, 1)), d], axis=1).T @ _np(x)
    assert np.abs(want).max() > 0.1
    # 32-bit products of 32 values, a softmax of 2^-19 of |g| <= 1, sums over 20 tokens of |x| < 5
    assert (np.abs(_np(r.grad) - want) <= 20 * 5 * 2.0 ** -17).all()


def test_logits_changed_after_the_picks_are_noticed(ops):   # noqa: F811
    print("[operators] logits changed in place", flush=True)
    t = _torch()
    l = t.randn(4, 8, device="cuda").requires_grad_()
    z = l * 1.0
    w, *_ = ops.route(z, 2, normalize=False)
    z.add_(1.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        w.sum().backward()


def test_no_second_derivative_in_silence(ops):   # noqa: F811
    print("[operators] second derivative", flush=True)
    t = _torch()
    l = t.randn(4, 8, device="cuda").requires_grad_()
    w, *_ = ops.route(l, 2)
    d, = t.autograd.grad(w.square().sum(), l, create_graph=True)
    with pytest.raises(RuntimeError):
        d.square().sum().backward()


def test_layer_has_no_gradient_and_says_so(ops):   # noqa: F811
    print("[operators] layer asked for a gradient", flush=True)
    t = _torch()
    x, router, up, down = (t.randn(s, device="cuda").bfloat16() for s in ((3, 64), (4, 64), (4, 64, 64), (4, 64, 32)))
    want = ops.moe_layer(x, router, up, down, 2)
    assert not want.requires_grad
    for at in range(4):
        args = [a.clone().requires_grad_(i == at) for i, a in enumerate((x, router, up, down))]
        y = ops.moe_layer(*args, 2)
        assert t.equal(y, want)
        with pytest.raises(RuntimeError, match="no gradient"):
            y.float().sum().backward()
        with t.no_grad():
            assert not ops.moe_layer(*args, 2).requires_grad


def test_packed_values_have_no_gradient(ops):   # noqa: F811
    # codes and scales are whole numbers, of which torch knows no gradient
    print("[operators] packing asked for a gradient", flush=True)
    t = _torch()
    x = t.randn(8, 64, device="cuda", requires_grad=True)
    q = ops.quantize(x)
    assert not q.codes.requires_grad and not q.scales.requires_grad
    with pytest.raises(RuntimeError):
        ops.matmul(q, q, t.float32).sum().backward()
    with pytest.raises(RuntimeError):
        ops.dequantize(q, t.float32).sum().backward()
    with pytest.raises(ValueError):                              # nothing is written into a tensor that a gradient is asked of
        ops.matmul(q, q, t.float32, out=t.zeros(8, 8, device="cuda", requires_grad=True))


def test_a_product_into_a_tensor_that_a_gradient_needs_is_noticed(ops):   # noqa: F811
    print("[operators] product into a saved tensor", flush=True)
    t = _torch()
    q = ops.quantize(t.randn(8, 64, device="cuda"))
    a, saved = t.randn(8, 8, device="cuda", requires_grad=True), t.randn(8, 8, device="cuda")
    y = a * saved
    ops.matmul(q, q, t.float32, out=saved)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_forward_mode_is_refused(ops):   # noqa: F811
    print("[operators] forward mode", flush=True)
    t = _torch()
    import torch.autograd.forward_ad as fw
    l = t.randn(4, 8, device="cuda")
    with fw.dual_level(), pytest.raises(RuntimeError):
        ops.route(fw.make_dual(l, t.ones_like(l)), 2)


def test_batched_tensors_are_refused(ops):   # noqa: F811
    print("[operators] vmap", flush=True)
    t = _torch()
    x = t.randn(3, 4, 8, device="cuda")
    with pytest.raises(RuntimeError):
        t.vmap(lambda l: ops.route(l, 2)[0])(x)


def test_inference_tensors_are_taken(ops):   # noqa: F811
    print("[operators] inference mode", flush=True)
    t = _torch()
    with t.inference_mode():
        q = ops.quantize(t.randn(8, 64, device="cuda"))
        out = t.zeros(8, 8, device="cuda")
        assert ops.matmul(q, q, t.float32, out=out) is out
        want = ops.dequantize(q, t.float32)
        np.testing.assert_allclose(_np(out), _np(want) @ _np(want).T, atol=64 * 2.0 ** -20)
        w, ids, _, _ = ops.route(out, 2)
        assert ids.shape == (8, 2)


def test_layer_of_packed_weights_has_no_gradient_and_says_so(ops):   # noqa: F811
    print("[operators] layer of packed weights asked for a gradient", flush=True)
    from paper_2606_07019_amd.operators import MX
    t = _torch()
    x, router = t.randn(3, 64, device="cuda").bfloat16(), t.randn(4, 64, device="cuda").bfloat16()
    up, down = (MX(*(f.view(4, w.shape[1], -1) for f in ops.quantize(w.view(-1, w.shape[2]))[:2]), w.shape[2])
                for w in (t.randn(4, 64, 64, device="cuda"), t.randn(4, 64, 32, device="cuda")))
    want = ops.moe_layer(x, router, up, down, 2)
    y = ops.moe_layer(x.clone().requires_grad_(), router, up, down, 2)
    assert t.equal(y, want) and not want.requires_grad
    with pytest.raises(RuntimeError, match="no gradient"):
        y.float().sum().backward()
