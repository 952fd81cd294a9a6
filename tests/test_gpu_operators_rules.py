"""GPU: sizes on either side of the rules that choose a kernel's form, against
the 64-bit oracle with the bounds that tests/test_gpu_operators.py derives."""

import numpy as np
import pytest

from test_gpu_operators import TINY, ULP, _np, _packed, _torch, ops  # noqa: F401
from test_gpu_operators_inner import _layer

pytestmark = pytest.mark.gpu

# 256 x 256 results a workgroup or 128 x 128: 128 tiles of 256 with 256 and 258 of 128, few of either, 127 of 256
TILES = [(128, 32768, 40), (100, 33000, 300), (129, 32700, 130), (129, 32300, 257), (2000, 2100, 200), (4097, 1800, 96)]


@pytest.mark.parametrize("m,n,k", TILES)
def test_product_at_the_tiles_rule(ops, m, n, k):   # noqa: F811
    # scale 2: all values are whole numbers up to 12, sums below 2^24
    print(f"[operators] product {m}x{n}x{k} at the rule of tiles", flush=True)
    rng = np.random.default_rng(m + n + k)
    a, av = _packed(rng, m, k, 128, 128)
    b, bv = _packed(rng, n, k, 128, 128)
    np.testing.assert_array_equal(_np(ops.matmul(a, b, _torch().float32)), av @ bv.T)


# one to eight steps of k a wave, with fewer and with more tiles of 16 rows of B than 256 and 512 workgroups take at once
@pytest.mark.parametrize("k", [700, 1900, 2900, 4000, 5000, 6000, 7100])
@pytest.mark.parametrize("m,n", [(1, 4100), (16, 8300), (33, 4100), (64, 9000)])
def test_product_of_few_rows_over_many_tiles(ops, m, n, k):   # noqa: F811
    print(f"[operators] product {m}x{n}x{k}, few rows", flush=True)
    rng = np.random.default_rng(m + n + k)
    a, av = _packed(rng, m, k, 127, 127)
    b, bv = _packed(rng, n, k, 127, 127)
    want = av @ bv.T                                             # quarters below 2^22
    assert (np.abs(av) @ np.abs(bv[:50]).T).max() < 2.0 ** 22
    np.testing.assert_array_equal(_np(ops.matmul(a, b, _torch().float32)), want)


# tokens of an expert on either side of 12 and 24; seven blocks of k and eight for either kind of weights, 2,048 tiles and fewer
LAYERS = [(48, 32, 8, 136, 72), (49, 32, 8, 136, 72), (96, 32, 8, 136, 72), (97, 32, 8, 136, 72),
          (64, 8, 2, 448, 448)]
LAYERS = [(*l, d, w) for l in LAYERS for d in ("bf16", "f16") for w in ("same", "mx")]
LAYERS += [(16, 128, 8, 448, 448, "bf16", "same"), (16, 128, 8, 512, 512, "f16", "same"), (16, 32, 8, 1792, 1000, "f16", "mx"), (16, 32, 8, 2048, 1100, "bf16", "mx")]


@pytest.mark.parametrize("tokens,experts,topk,hidden,inter,dtype,weights", LAYERS)
def test_layer_at_its_rules(ops, tokens, experts, topk, hidden, inter, dtype, weights):   # noqa: F811
    print(f"[operators] layer {tokens} of {experts}/{topk}, {hidden}x{inter} {dtype} {weights}", flush=True)
    rng = np.random.default_rng(tokens + hidden)
    x = rng.normal(size=(tokens, hidden))
    up = rng.standard_normal(size=(experts, 2 * inter, hidden), dtype=np.float32) / np.float32(np.sqrt(hidden))
    down = rng.standard_normal(size=(experts, hidden, inter), dtype=np.float32) / np.float32(np.sqrt(inter))
    got, want, size = _layer(ops, x, up, down, dtype, weights, rng.normal(size=(experts, hidden)) * 2 / np.sqrt(hidden), topk)
    # sums of 32-bit products over hidden and inner values; the softmax, silu and products of both, 2^-20
    room = ((hidden + inter + topk) * 2.0 ** -24 + 2.0 ** -20) * size
    assert (np.abs(got - want) <= room + ULP[dtype] * np.abs(want) * 1.01 + TINY[dtype]).all()
