"""GPU: a training step of an expert-parallel layer's own part from its router to
its gradients, eager, on another stream and captured; and what a captured step,
two contexts and automatic differentiation have to keep."""

import numpy as np
import pytest

from oracle import operators as O
from test_gpu_operators8 import _np, _to, _torch, ops  # noqa: F401

pytestmark = pytest.mark.gpu

TOKENS, EXPERTS, TOPK, HIDDEN, INTER = 700, 12, 3, 264, 200


def _inputs(seed):
    t = _torch()
    rng = np.random.default_rng(seed)
    x = _to(rng.normal(size=(TOKENS, HIDDEN)), "bf16")
    router = _to(rng.normal(size=(EXPERTS, HIDDEN)) * 2 / np.sqrt(HIDDEN), "bf16")
    w = _to(rng.normal(size=(EXPERTS, INTER, HIDDEN)) / np.sqrt(HIDDEN), "bf16")
    mask = t.from_numpy((rng.random(TOKENS) < 0.9).astype(np.uint8)).cuda()
    return x, router, w, _to(rng.normal(size=(TOKENS * TOPK, INTER)), "bf16"), mask


def _step(ops, x, router, w, dy, mask):   # noqa: F811
    """The layer's own part of a training step, as its user writes it; rows of no one are zeros."""
    t = _torch()
    logits = x @ router.t()
    weights, ids, counts, order = ops.route(logits, TOPK, mask=mask)
    loss, seen, probs, n = ops.balance_loss(logits, ids, mask=mask)
    dlogits = ops.balance_loss_backward(logits, seen, n, t.ones((), device="cuda"), mask=mask)
    groups = ops.expert_groups(counts, TOKENS * TOPK)
    rows = x[t.clamp(order, min=0).long() // TOPK]
    (xr, xc), (dr, dc) = ops.quantize8_both(rows, groups), ops.quantize8_both(dy, groups)
    wr, wc = ops.quantize8_tiles(w)
    y = ops.expert_matmul8(xr, wr, groups, t.bfloat16, out=t.zeros(TOKENS * TOPK, INTER, dtype=t.bfloat16, device="cuda"))
    dx = ops.expert_matmul8(dr, wc, groups, t.bfloat16, out=t.zeros(TOKENS * TOPK, HIDDEN, dtype=t.bfloat16, device="cuda"))
    dw = ops.expert_gradient8(dc, xc, groups, t.float32)
    return [weights, ids, counts, order, loss, seen, probs, n, dlogits, y, dx, dw]


def test_a_training_step(ops):   # noqa: F811
    print("[operators8] training step", flush=True)
    t = _torch()
    x, router, w, dy, mask = _inputs(1)
    weights, ids, counts, order, loss, seen, probs, n, dlogits, y, dx, dw = _step(ops, x, router, w, dy, mask)
    assert t.equal(counts, seen) and int(n) == int(mask.sum())
    used = int(counts.sum())
    assert used == TOPK * int(n) and (y[used:] == 0).all() and (dx[used:] == 0).all()
    start = [0, *np.cumsum(counts.cpu().numpy())]
    order = order.cpu().numpy()
    for e in range(EXPERTS):
        rows = order[start[e]:start[e + 1]]
        assert (ids.view(-1)[t.from_numpy(rows).cuda().long()] == e).all()
        v, g, m = _np(x)[rows // TOPK], _np(dy)[start[e]:start[e + 1]], _np(w)[e]
        # each factor is off by a sixteenth at most (half a step of four digits) where it is not far below its block's
        # largest; their errors have both signs, so that the norm is off by far less than both of them together
        for got, want in ((y[start[e]:start[e + 1]], v @ m.T), (dx[start[e]:start[e + 1]], g @ m), (dw[e], g.T @ v)):
            assert np.linalg.norm(_np(got) - want) <= 2 * 2.0 ** -4 * np.linalg.norm(want)
    wl, wc, wp, wr = O.balance(_np(x @ router.t()), ids.cpu().numpy(), mask.cpu().numpy())
    assert abs(float(loss) - wl) <= 1e-4 * wl and wr == int(n)


def test_on_another_stream_and_in_a_graph(ops):   # noqa: F811
    print("[operators8] stream and graph", flush=True)
    t = _torch()
    inputs = _inputs(2)
    want = [a.clone() for a in _step(ops, *inputs)]
    side = t.cuda.Stream()
    side.wait_stream(t.cuda.current_stream())
    with t.cuda.stream(side):
        got = _step(ops, *inputs)
    side.synchronize()
    assert all(t.equal(a, b) for a, b in zip(got, want))
    held = [a.clone() for a in inputs]
    graphs = []
    for _ in range(2):                                           # two graphs share no workspace
        graph = t.cuda.CUDAGraph()
        with t.cuda.graph(graph):
            got = _step(ops, *held)
        graphs.append((graph, got))
    for k in range(4):
        fresh = _inputs(3 + k)
        want = _step(ops, *fresh)
        for a, b in zip(held, fresh):
            a.copy_(b)
        for graph, _ in graphs:
            graph.replay()
        t.cuda.synchronize()
        for _, got in graphs:
            assert all(t.equal(a, b) for a, b in zip(got, want)), k


def test_results_do_not_change_from_run_to_run(ops):   # noqa: F811
    print("[operators8] run to run", flush=True)
    t = _torch()
    inputs = _inputs(9)
    want = [a.clone() for a in _step(ops, *inputs)]
    rng = np.random.default_rng(4)
    l = _to(rng.normal(size=(40000, 300)), "f32")                # many workgroups, joined by several
    ids = t.from_numpy(rng.integers(0, 300, (40000, 4)).astype(np.int32)).cuda()
    first = ops.balance_loss(l, ids)
    for _ in range(5):
        assert all(t.equal(a, b) for a, b in zip(_step(ops, *inputs), want))
        assert all(t.equal(a, b) for a, b in zip(ops.balance_loss(l, ids), first))


def test_a_captured_gradient_of_the_balance_loss(ops):   # noqa: F811
    print("[operators8] captured gradient", flush=True)
    t = _torch()
    rng = np.random.default_rng(5)
    held = _to(rng.normal(size=(300, 40)), "f32")
    ids = t.from_numpy(rng.integers(0, 40, (300, 2)).astype(np.int32)).cuda()

    def gradient(l):
        leaf = l.detach().requires_grad_()
        loss, _, probs, _ = ops.balance_loss(leaf, ids)
        return t.autograd.grad(loss * 3 + probs.square().sum(), leaf)[0]

    side = t.cuda.Stream()
    side.wait_stream(t.cuda.current_stream())
    with t.cuda.stream(side):
        gradient(held)
    t.cuda.current_stream().wait_stream(side)
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        got = gradient(held)
    for k in range(3):
        fresh = _to(rng.normal(size=(300, 40)), "f32")
        want = gradient(fresh)
        held.copy_(fresh)
        graph.replay()
        t.cuda.synchronize()
        assert t.equal(got, want), k


def test_products_bump_the_version_of_what_they_write(ops):   # noqa: F811
    print("[operators8] versions", flush=True)
    t = _torch()
    x = _to(np.random.default_rng(6).normal(size=(70, 128)), "bf16")
    q = ops.quantize8(x)
    out = t.zeros(70, 70, device="cuda")
    scale = t.ones(70, 70, device="cuda", requires_grad=True)
    loss = (scale * out).sum()
    ops.matmul8(q, q, t.float32, out=out)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    with t.inference_mode():
        ops.matmul8(q, q, t.float32, out=t.zeros(70, 70, device="cuda"))
    assert not ops.quantize8(x.float().requires_grad_()).codes.requires_grad


@pytest.mark.parametrize("experts", [8, 200, 600])
def test_gradient_of_a_joint_batch(ops, experts):   # noqa: F811
    """Counts and rows summed over ranks: more picks in all than 32 bits hold."""
    print(f"[operators8] joint batch, {experts} experts", flush=True)
    t = _torch()
    rng = np.random.default_rng(experts)
    logits = _to(rng.normal(size=(70, experts)) * 2, "f32")
    counts = rng.integers(0, 2 ** 31, size=experts).astype(np.int32)
    counts[:3] = 2 ** 31 - 1
    rows, dloss = 2 ** 30 + 7, 2.0 ** 30
    got = _np(ops.balance_loss_backward(logits, t.from_numpy(counts).cuda(), t.tensor(rows, dtype=t.int32, device="cuda"),
                                        t.full((), dloss, device="cuda")))
    assert counts.astype(np.int64).sum() > 2 ** 32
    want = O.balance_backward(_np(logits), counts, rows, dloss)
    p = np.exp(_np(logits))
    p /= p.sum(axis=1, keepdims=True)
    size = dloss * experts * counts / counts.astype(np.float64).sum()
    # as in tests/test_gpu_operators8.py: a probability's error, and the difference's, as large as its parts
    bound = p * (size + (p * size).sum(axis=1, keepdims=True)) / rows * (2.0 ** 5 + 2 * experts + 16) * 2.0 ** -24
    assert (np.abs(got - want) <= bound + 2.0 ** -24 * np.abs(want)).all()
    # and the halves of a batch, each with the counts and rows of both, have the gradient of the whole
    ids = t.from_numpy(rng.integers(0, experts, (70, 2)).astype(np.int32)).cuda()
    _, whole, _, n = ops.balance_loss(logits, ids)
    one = t.ones((), device="cuda")
    parts = [ops.balance_loss(logits[i:i + 35], ids[i:i + 35].contiguous()) for i in (0, 35)]
    joint, both = parts[0][1] + parts[1][1], parts[0][3] + parts[1][3]
    assert t.equal(joint, whole) and t.equal(both, n)
    halves = [ops.balance_loss_backward(logits[i:i + 35], joint, both, one) for i in (0, 35)]
    assert t.equal(t.cat(halves), ops.balance_loss_backward(logits, whole, n, one))


def test_two_streams_and_two_contexts_at_once(ops):   # noqa: F811
    """Calls with workspaces in flight together, with nothing waited for in between."""
    print("[operators8] two streams, two contexts", flush=True)
    from paper_2606_07019_amd.operators import Operators
    from test_gpu_operators8 import _packed
    t = _torch()
    rng = np.random.default_rng(10)
    many = [_packed(rng, rows, 9000, 116, 122)[0] for rows in (129, 257)]   # shared out over k
    few = [_packed(rng, rows, 20000, 116, 122)[0] for rows in (7, 3000)]
    l = _to(rng.normal(size=(5000, 300)), "f32")                 # many workgroups, joined
    ids = t.from_numpy(rng.integers(0, 300, (5000, 4)).astype(np.int32)).cuda()
    inputs = _inputs(11)

    def calls(o):
        return [o.matmul8(*many, t.float32), o.matmul8(*few, t.bfloat16), *o.balance_loss(l, ids), o.matmul8(*few, t.float32),
                o.matmul8(*many, t.bfloat16), *_step(o, *inputs)]

    want = [a.clone() for a in calls(ops)]
    other = Operators(0)
    for contexts in ((ops, ops), (ops, other), (other, other)):
        sides = [t.cuda.Stream() for _ in range(2)]
        got = []
        for side in sides:
            side.wait_stream(t.cuda.current_stream())
        for _ in range(4):
            for side, o in zip(sides, contexts):
                with t.cuda.stream(side):
                    got.append(calls(o))
        t.cuda.synchronize()
        for results in got:
            assert all(t.equal(a, b) for a, b in zip(results, want))
    other.close()
