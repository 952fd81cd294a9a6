"""GPU: the expert layer's inner values keep 32 bits, over the whole range of a
32-bit number, whatever type the tokens and the weights have.

Rounding y hides what is lost before it, so the layers here bring it out: by
cancellation, where every partial sum is exact and the result must be too; by
small inner values against large weights, with bounds that are relative alone;
and by large ones against weights of both signs.
"""

import numpy as np
import pytest

from oracle import operators as O
from test_gpu_operators import TINY, ULP, _np, _to, _torch, ops  # noqa: F401

pytestmark = pytest.mark.gpu


def _layer(ops, x, up, down, dtype, weights, router=None, topk=1):   # noqa: F811
    """(the layer's result, what it is by definition, and what its rounding errors scale with)."""
    from paper_2606_07019_amd.operators import MX
    x = _to(x, dtype)
    router = _to(np.zeros((up.shape[0], x.shape[1])) if router is None else router, dtype)
    if weights == "mx":
        args = []
        for w in (up, down):
            q = ops.quantize(_to(w.reshape(-1, w.shape[2])))
            args.append(MX(q.codes.view(*w.shape[:2], -1), q.scales.view(*w.shape[:2], -1), w.shape[2]))
        values = [O.mx_values(*(t.cpu().numpy().reshape(-1, t.shape[2]) for t in q[:2]), q.cols).reshape(w.shape)
                  for q, w in zip(args, (up, down))]
    else:
        args = [_to(up, dtype), _to(down, dtype)]
        values = [_np(a) for a in args]
    with np.errstate(over="ignore"):
        want, size = O.moe_layer(_np(x), _np(router), *values, topk, True)
    return _np(ops.moe_layer(x, router, *args, topk)), want, size


@pytest.mark.parametrize("tokens", [1, 40])
@pytest.mark.parametrize("weights", ["same", "mx"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_differences_of_inner_values(ops, dtype, weights, tokens):   # noqa: F811
    # gate 32 (silu gives 32 in 32 bits), lifts 1 + 2^-12 + 2^-23 and 1 + 2^-12: the first has 24 digits.  Down weights 1
    # and -1.  All partial sums are multiples of 2^-18 below 2^6, exact in 32 bits in any order; so is the difference, 2^-18.
    print(f"[operators] differences of inner values {dtype} {weights} {tokens}", flush=True)
    hidden, inter = 256, 136
    x = np.zeros((tokens, hidden))
    x[:, [0, 32, 64, 96]] = 1.0, 2.0 ** -6, 2.0 ** -11, 32.0
    up = np.zeros((1, 2 * inter, hidden))
    up[0, [3, 131], 96] = 1.0                                    # gates
    up[0, [inter + 3, inter + 131], 0] = 1.0                     # lifts
    up[0, [inter + 3, inter + 131], 32] = 2.0 ** -6
    up[0, inter + 3, 64] = 2.0 ** -12
    down = np.zeros((1, hidden, inter))
    down[0, ::2, 3], down[0, ::2, 131] = 1.0, -1.0
    down[0, 1::2, 3], down[0, 1::2, 131] = -1.0, 1.0
    got, want, _ = _layer(ops, x, up, down, dtype, weights)
    np.testing.assert_allclose(want, np.where(np.arange(hidden) % 2 == 0, 1, -1) * 2.0 ** -18 * np.ones((tokens, 1)), rtol=1e-6)
    np.testing.assert_array_equal(got, np.where(want > 0, 2.0 ** -18, -2.0 ** -18))


@pytest.mark.parametrize("weights", ["same", "mx"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("tokens,experts,topk,hidden,inter", [(3, 4, 2, 64, 256), (70, 3, 2, 200, 264), (1, 2, 1, 77, 33)])
def test_small_inner_values(ops, tokens, experts, topk, hidden, inter, dtype, weights):   # noqa: F811
    # inner values near 2^-25, weights that bring the results back among the normal numbers of every type
    print(f"[operators] small inner values {tokens} {experts} {hidden}x{inter} {dtype} {weights}", flush=True)
    rng = np.random.default_rng(tokens + hidden)
    x = rng.normal(size=(tokens, hidden)) * 2.0 ** -8
    up = rng.normal(size=(experts, 2 * inter, hidden)) / np.sqrt(hidden) * 2.0 ** -4
    down = rng.normal(size=(experts, hidden, inter)) / np.sqrt(inter) * 2.0 ** 14
    got, want, size = _layer(ops, x, up, down, dtype, weights, rng.normal(size=(experts, hidden)), topk)
    # sums of 32-bit products over hidden and inner values; the softmax, silu and products of both, 2^-20
    room = ((hidden + inter + topk) * 2.0 ** -24 + 2.0 ** -20) * size
    assert (np.abs(got - want) <= room + ULP[dtype] * np.abs(want) * 1.01 + TINY[dtype]).all()


@pytest.mark.parametrize("weights", ["same", "mx"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_large_inner_values_against_weights_of_both_signs(ops, dtype, weights):   # noqa: F811
    # gate = lift = 2^13, inner values 2^26; down weights 2^-12, -2^-12 and nothing: whole sums of 2^14
    print(f"[operators] large inner values, both signs, {dtype} {weights}", flush=True)
    hidden, inter = 64, 48
    x = np.full((18, hidden), 2.0 ** 7)
    up = np.ones((1, 2 * inter, hidden))
    down = np.zeros((1, hidden, inter))
    down[0, :, 0:10] = 2.0 ** -12
    down[0, ::2, 10:18], down[0, 1::2, 10:22] = -2.0 ** -12, -2.0 ** -12
    got, want, _ = _layer(ops, x, up, down, dtype, weights)
    np.testing.assert_array_equal(want, np.where(np.arange(hidden) % 2 == 0, 2, -2) * 2.0 ** 14 * np.ones((18, 1)))
    np.testing.assert_array_equal(got, want)


@pytest.mark.parametrize("weights", ["same", "mx"])
def test_the_largest_inner_values(ops, weights):   # noqa: F811
    # (2^64 - 2^54) 2^64 is finite in 32 bits and rounds to infinity in bf16; times 2^-120: 255.75, in bf16 256
    print(f"[operators] the largest inner values {weights}", flush=True)
    x = np.zeros((2, 64))
    x[:, 0], x[:, 32] = 2.0 ** 64, 2.0 ** 54
    up = np.zeros((1, 16, 64))
    up[0, 0, 0], up[0, 0, 32], up[0, 8, 0] = 1.0, -1.0, 1.0
    down = np.zeros((1, 64, 8))
    down[0, :, 0] = 2.0 ** -120
    got, want, _ = _layer(ops, x, up, down, "bf16", weights)
    np.testing.assert_array_equal(want, 255.75)
    np.testing.assert_array_equal(got, 256.0)
