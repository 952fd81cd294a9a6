"""GPU: sizes on either side of the rules that choose a kernel's form, against
the 64-bit oracle with the bounds that tests/test_gpu_operators.py derives."""

import numpy as np
import pytest

from test_gpu_operators import _np, _packed, _torch, ops  # noqa: F401

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
