"""The operators' own gradients, asked for a gradient of theirs, raise instead
of ending the graph in silence (CPU: no kernel runs, values do not matter)."""

import pytest

torch = pytest.importorskip("torch")

from paper_2606_07019_amd import operators as W  # noqa: E402
from paper_2606_07019_amd import pccl as P  # noqa: E402


@pytest.fixture
def ops(monkeypatch):
    o = W.Operators.__new__(W.Operators)
    o.device, o.h = torch.device("cpu"), None
    monkeypatch.setattr(W.Operators, "_call", lambda self, function, *args: None)
    monkeypatch.setattr(W.Operators, "_space", lambda self, ask, *sizes: (None, None, 0))
    monkeypatch.setattr(W.Operators, "_stream", lambda self: None)
    o._lib = P.load_library()
    return o


def _balance(ops, learned):
    i32 = torch.int32
    given = {"logits": torch.zeros(6, 8), "dloss": torch.ones(()), "dprobs": torch.ones(8)}
    given = {k: v.requires_grad_() if k == learned else v for k, v in given.items()}
    return lambda: ops.balance_loss_backward(given["logits"], torch.ones(8, dtype=i32), torch.ones((), dtype=i32), given["dloss"], given["dprobs"])


def _route(ops, learned):
    given = {"logits": torch.zeros(6, 8), "weights": torch.zeros(6, 2), "dweights": torch.ones(6, 2)}
    given = {k: v.requires_grad_() if k == learned else v for k, v in given.items()}
    return lambda: ops.route_backward(given["logits"], given["weights"], torch.zeros(6, 2, dtype=torch.int32), given["dweights"], normalize=False)


CALLS = [(_balance, n) for n in ("logits", "dloss", "dprobs")] + [(_route, n) for n in ("logits", "weights", "dweights")]


@pytest.mark.parametrize("make,learned", CALLS, ids=[f"{f.__name__[1:]}-{n}" for f, n in CALLS])
def test_a_gradient_of_a_gradient_raises(ops, make, learned):
    call = make(ops, learned)
    d = call()
    assert d.requires_grad
    with pytest.raises(RuntimeError, match="has no gradient"):
        d.sum().backward()
    with torch.no_grad():
        assert not call().requires_grad
    assert not make(ops, None)().requires_grad


@pytest.mark.parametrize("make", sorted({f for f, _ in CALLS}, key=lambda f: f.__name__))
def test_it_can_be_handed_on(ops, make):
    leaf = torch.zeros(6, 8, requires_grad=True)
    (leaf * 1).backward(gradient=make(ops, "logits")())          # as the part of a step that the caller makes
    assert leaf.grad.shape == (6, 8) and not leaf.grad.requires_grad


def test_recorded_gradients_are_as_they_were(ops):
    i32 = torch.int32
    l = torch.zeros(6, 8, requires_grad=True)
    loss, _, probs, _ = ops.balance_loss(l, torch.zeros(6, 2, dtype=i32))
    d, = torch.autograd.grad(loss + probs.sum(), l)
    assert d.shape == (6, 8) and not d.requires_grad
    w = ops.route(l, 2)[0]
    d, = torch.autograd.grad(w.sum(), l)
    assert d.shape == (6, 8) and not d.requires_grad


def test_forward_mode_is_refused(ops):
    from torch.autograd import forward_ad
    x = torch.zeros(6, 8)
    i32 = torch.int32
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(x, x)
        with pytest.raises(RuntimeError, match="forward-mode"):
            ops.balance_loss_backward(dual, torch.ones(8, dtype=i32), torch.ones((), dtype=i32), torch.ones(()))
        with pytest.raises(RuntimeError, match="forward-mode"):
            ops.route_backward(dual, x[:, :2].contiguous(), torch.zeros(6, 2, dtype=i32), x[:, :2].contiguous())
        assert not ops.balance_loss_backward(x, torch.ones(8, dtype=i32), torch.ones((), dtype=i32), None, torch.ones(8)).requires_grad
