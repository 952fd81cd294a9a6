"""GPU: products of 8-bit operands at the ends of the scales' range, up to 2^127
times 448 on one side and down to 2^-127 on the other, in every form of the
product.  A product's values are E4M3 codes times powers of two whatever their
size; results that lie within their type are numbers.

A result of 32 bits is within (k + 2) 2^-24 of the sum of its products'
magnitudes, but for operand values below 2^-126, which may be lost as a whole
where they do not meet a block of 2^120 or more; one of 16 bits as
tests/test_gpu_operators8.py derives it."""

import numpy as np
import pytest

from test_gpu_operators8 import _bound, _close, _np, _packed, _to, _torch, _type, ops  # noqa: F401

pytestmark = pytest.mark.gpu


def _ends(rng, m, n, k, zeros=0.3):
    """Operands whose blocks meet at 2^0: one far up, the other as far down, either way round, among ordinary ones."""
    from paper_2606_07019_amd.operators import F8
    from oracle import operators as O
    t = _torch()
    nb = -(-k // 128)
    d = rng.choice([0, 0, 0, 121, 127, -121, -127, 110], size=nb)
    d[nb - 1] = 125                                              # one at least
    pair = []
    for rows, sign in ((m, 1), (n, -1)):
        q, _ = _packed(rng, rows, k)
        c, s = q.codes.cpu().numpy(), np.zeros(tuple(q.scales.shape), np.uint8)
        c[rng.random(c.shape) < zeros] = 0
        s[:, :nb] = np.clip(127 + sign * d + rng.integers(-3, 4, size=(rows, nb)), 0, 254)
        pair.append((F8(t.from_numpy(c).cuda(), t.from_numpy(s).cuda(), k), O.f8_values(c, s, k)))
    return pair


def _exact_bound(av, bv):
    """How far a result of 32 bits may be from av bv^T."""
    lost = [np.where(np.abs(v) < 2.0 ** -126, np.abs(v), 0.0) for v in (av, bv)]
    near = [np.where(np.abs(v) < 448 * 2.0 ** 119, np.abs(v), 0.0) for v in (av, bv)]   # blocks of up to 2^119
    size = np.abs(av) @ np.abs(bv).T
    return (av.shape[1] + 2) * 2.0 ** -24 * size + lost[0] @ near[1].T + near[0] @ lost[1].T


# few rows of each number of sixteens, one part of k and several; tiles of 128 alone, two a compute unit and
# shared out over k; tiles of 256
SHAPES = [(1, 40, 300), (20, 33, 700), (45, 70, 2000), (64, 40, 640), (9, 33, 20000), (50, 20, 9000), (100, 130, 700), (129, 257, 5000),
          (2100, 2080, 300), (4000, 4096, 260)]


@pytest.mark.parametrize("m,n,k", SHAPES)
def test_product(ops, m, n, k):   # noqa: F811
    print(f"[operators8] ends, product {m}x{n}x{k}", flush=True)
    rng = np.random.default_rng(m + n + k)
    (a, av), (b, bv) = _ends(rng, m, n, k)
    want = av @ bv.T
    assert (np.abs(want) < 1e38).all() and np.abs(av).max() >= 2.0 ** 128   # past f32's and bf16's numbers
    _close(_np(ops.matmul8(a, b, _type("f32"))), want, _exact_bound(av, bv), "f32")
    if m * n * k < 10 ** 7:
        _close(_np(ops.matmul8(a, b, _type("bf16"))), want, _bound(a, av, b, bv, "bf16"), "bf16")


@pytest.mark.parametrize("m,n", [(10, 40), (140, 150)])
def test_product_beside_blocks_that_are_not_numbers(ops, m, n):   # noqa: F811
    print(f"[operators8] ends, NaN blocks {m}x{n}", flush=True)
    rng = np.random.default_rng(m)
    (a, av), (b, bv) = _ends(rng, m, n, 640)
    a.scales[m - 1, 3] = 255
    b.scales[2, 4] = 255
    a.codes[1, 600] = 127
    got = _np(ops.matmul8(a, b, _type("f32")))
    nan = np.zeros((m, n), bool)
    nan[m - 1], nan[:, 2], nan[1] = True, True, True
    np.testing.assert_array_equal(np.isnan(got), nan)
    bound = _exact_bound(av, bv)
    assert (np.abs(got - av @ bv.T)[~nan] <= bound[~nan] * (1 + 2.0 ** -24) + 2.0 ** -24 * np.abs(av @ bv.T)[~nan] * 1.01).all()


# experts in tiles of 128 and of 256
@pytest.mark.parametrize("counts,n,k", [([129, 0, 1, 300], 140, 300), ([640] * 16, 4096, 260)], ids=["128", "256"])
def test_experts_product(ops, counts, n, k):   # noqa: F811
    print(f"[operators8] ends, {len(counts)} experts, {n}x{k}", flush=True)
    from paper_2606_07019_amd.operators import F8
    t = _torch()
    rng = np.random.default_rng(n)
    rows, experts = sum(counts), len(counts)
    (a, av), (w, wv) = _ends(rng, rows, experts * n, k)
    g = ops.expert_groups(t.tensor(counts, dtype=t.int32, device="cuda"), rows)
    got = _np(ops.expert_matmul8(a, F8(w.codes.view(experts, n, -1), w.scales.view(experts, n, -1), k), g, t.float32))
    at = 0
    for e, c in enumerate(counts):
        x, y = av[at:at + c], wv[e * n:e * n + n]
        _close(got[at:at + c], x @ y.T, _exact_bound(x, y), "f32")
        at += c


# gradients in tiles of 128 and of 256
@pytest.mark.parametrize("counts,m,n", [([129, 0, 1, 300], 140, 260), ([200] * 16, 1024, 2048)], ids=["128", "256"])
def test_experts_gradient(ops, counts, m, n):   # noqa: F811
    print(f"[operators8] ends, gradient of {len(counts)} experts, {m}x{n}", flush=True)
    from paper_2606_07019_amd.operators import group_blocks
    t = _torch()
    rng = np.random.default_rng(m)
    rows, blocks = sum(counts), [-(-c // 128) for c in counts]
    (a, av), (b, bv) = _ends(rng, m, n, 128 * group_blocks(len(counts), rows))
    a.scales[:, 1], b.scales[:, 1] = 251, 3                      # of those that are used: the last one may not be
    av, bv = (_values8(q) for q in (a, b))
    g = ops.expert_groups(t.tensor(counts, dtype=t.int32, device="cuda"), rows)
    got = _np(ops.expert_gradient8(a, b, g, t.float32))
    at = 0
    for e, c in enumerate(blocks):
        x, y = av[:, 128 * at:128 * (at + c)], bv[:, 128 * at:128 * (at + c)]
        _close(got[e], x @ y.T, _exact_bound(x, y), "f32")
        at += c


def _values8(q):
    from oracle import operators as O
    return O.f8_values(q.codes.cpu().numpy(), q.scales.cpu().numpy(), q.cols)


@pytest.mark.parametrize("m", [8, 200])
def test_what_packing_makes_of_the_largest_numbers(ops, m):   # noqa: F811
    print(f"[operators8] ends, {m} rows of the largest numbers", flush=True)
    t = _torch()
    rng = np.random.default_rng(m)
    top = float(t.finfo(t.float32).max)
    x = rng.normal(size=(m, 300)) * 2.0 ** 124
    x[:, ::9] = top                                              # rounded to 2^128
    w = np.clip(rng.normal(size=(70, 300)), -2, 2) * 2.0 ** -20
    w[:, ::2] = 0.0
    a, b = ops.quantize8(_to(x)), ops.quantize8(_to(w))
    av, bv = _values8(a), _values8(b)
    assert np.isfinite(av).all() and av.max() == 2.0 ** 128
    _close(_np(ops.matmul8(a, b, t.float32)), av @ bv.T, _exact_bound(av, bv), "f32")
