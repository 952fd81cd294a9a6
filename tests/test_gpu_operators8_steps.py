"""GPU: the few-row form of the 8-bit product in each of its kernels, which are
made for a number of sixteens of rows and a number of steps a wave holds: waits
and the order of a wave's ring depend on both.  Whole results must be equal."""

import pytest

from test_gpu_operators8 import _torch, ops  # noqa: F401
from test_gpu_operators8_far import _whole

pytestmark = pytest.mark.gpu

MADE = (1, 2, 3, 4, 5, 6, 8)                                     # steps that kernels are made for
MOST = {1: 8, 2: 8, 3: 5, 4: 4}                                  # and how many so many sixteens of rows can hold


def kernel(m, k):
    """(sixteens of rows, steps) of the kernel that takes m <= 64 rows of k values: eight waves share out a part of k."""
    rows, blocks = -(-m // 16), -(-k // 128)
    parts = -(-blocks // (8 * MOST[rows]))
    each = -(-blocks // (8 * parts))
    return rows, min(s for s in MADE if s >= each)


# for each kernel a k that ends within a block and within the last waves' steps, and where there is one a k in several parts
SHAPES = [(m, n, k)
          for rows, m, n in ((1, 16, 40), (1, 3, 4200), (2, 17, 70), (2, 32, 33), (3, 48, 40), (3, 35, 100), (4, 64, 40), (4, 49, 130))
          for s in range(1, MOST[rows] + 1)
          for k in (1024 * s - 500, 1024 * (s + MOST[rows]) - 130)]


@pytest.mark.parametrize("m,n,k", SHAPES)
def test_product(ops, m, n, k):   # noqa: F811
    print(f"[operators8] product {m}x{n}x{k}, kernel of {kernel(m, k)}", flush=True)
    _whole(ops, m, n, k)
