"""Launches of the operators at their largest extents (CPU: a HIP runtime that
notes launches instead of running them): what is within the stated limits is
launched, in grids that a launch can have, and what is not is refused."""

import pytest

from test_operators_device import run_with_recorder

TOP = """
h = P.pccl_create(0, 0)


def attempt(fn, *args):
    count.value = 0
    try:
        fn(h, *args)
    except P.PcclError as e:
        assert count.value == 0, "a call that is refused launches nothing"
        return e.name[5:]
    for i in range(count.value):
        g, b = noted[i].grid, noted[i].block
        for d in range(3):
            assert g[d] * b[d] < 1 << 32, ("threads of a launch", list(g), list(b))
    return count.value


def slices(first, rows):
    # what the launches' first arguments say of where their rows start, and how many they have
    return [(noted[i].arg[first], noted[i].arg[rows]) for i in range(count.value)]


TOP = (1 << 31) - 1
"""

ROWS = TOP + """
for rows, cols in ((1 << 24, 8), ((1 << 29) - 32, 8), ((1 << 29) - 31, 8), ((1 << 29) + 64, 8), (TOP, 1), (1 << 28, 600), (TOP, 512), (1 << 24, 70000)):
    assert attempt(P.pccl_mx_quantize, M, P.PCCL_BF16, rows, cols, cols + 3, M, M) == count.value > 0, (rows, cols)
    at = M
    for start, n in slices(0, 1):
        assert start == at and n > 0
        at += n * (cols + 3) * 2
    assert at == M + rows * (cols + 3) * 2, (rows, cols)
print("rows fit")
"""

UNPACKED = TOP + """
for rows, cols in ((1000, 70000), ((1 << 26) - 4, 8), (1 << 26, 8), (1 << 27, 8), (TOP, 1), (1 << 24, 70000)):
    assert attempt(P.pccl_mx_dequantize, M, M, rows, cols, M, P.PCCL_BF16, cols + 3) == count.value > 0, (rows, cols)
    at = M
    for start, n in slices(0, 2):
        assert start == at and n > 0
        at += n * ((cols + 127) // 128 * 64)
    assert at == M + rows * ((cols + 127) // 128 * 64), (rows, cols)
print("unpacked fits")
"""

COLUMNS = TOP + """
for rows, cols, want in ((70000, 70000, 1), (128, TOP, "EUNSUPPORTED"), (128, TOP - 128, 1), (TOP, 128, "EUNSUPPORTED"), (TOP - 128, 1, 1), (1 << 20, 1 << 20, "EUNSUPPORTED")):
    for codes in (None, M):
        assert attempt(P.pccl_mx_quantize, M, P.PCCL_BF16, rows, cols, cols, codes, codes, M, M) == want, (rows, cols, codes)
print("columns fit")
"""

PRODUCTS = TOP + """
for m, n, want in ((131072, 131072, 1), (65536, 262144, 1), (200000, 200000, 1), (1, 1 << 27, 1), (64, TOP, 1), (1, TOP, 1), (70000, 70000, 1),
                   (1 << 20, 1 << 20, "EUNSUPPORTED"), (TOP, 1, "EUNSUPPORTED"), (TOP - 255, 1, 1), (65, TOP, "EUNSUPPORTED")):
    assert attempt(P.pccl_mx_matmul, M, M, M, M, m, n, 256, M, P.PCCL_BF16, n) == want, (m, n)
# k shared out between workgroups where 128 x 128 tiles leave two or more parts for each: the product and the joining
for n, want in ((20000, 1), (10000, 2)):
    assert attempt(P.pccl_mx_matmul, M, M, M, M, 70, n, 1 << 24, M, P.PCCL_BF16, n, M, 1 << 40) == want
print("products fit")
"""

ROUTES = TOP + """
most = 64 * ((1 << 22) - 1)
for tokens, experts, topk, want in ((most, 8, 2, 3), (most + 1, 8, 2, "EUNSUPPORTED"), (most, 300, 7, 3), (TOP // 8, 300, 8, "EUNSUPPORTED"), (most // 2, 300, 8, 3)):
    assert attempt(P.pccl_moe_route, M, P.PCCL_BF16, tokens, experts, experts, topk, 1, None, M, M, M, M, M, 1 << 40) == want, (tokens, experts, topk)
# the gradient of whatever the router takes, at either width of a row
for tokens, experts in ((most, 8), (most, 300), (1 << 26, 8), (1 << 26, 1000), (70000000, 512)):
    for normalize in (0, 1):
        assert attempt(P.pccl_moe_route_backward, M, P.PCCL_BF16, tokens, experts, experts + 1, 2, normalize, None, M, M, M, M, experts) == count.value > 0
        at, total = M, 0
        for start, n in slices(0, 1):
            assert start == M + total * (experts + 1) * 2 and n > 0
            total += n
        assert total == tokens, (tokens, experts)
print("routes fit")
"""


@pytest.mark.parametrize("body,word", [(ROWS, "rows fit"), (UNPACKED, "unpacked fits"), (COLUMNS, "columns fit"), (PRODUCTS, "products fit"),
                                       (ROUTES, "routes fit")], ids=["rows", "unpacked", "columns", "products", "routes"])
def test_launches_fit(tmp_path, body, word):
    assert word in run_with_recorder(tmp_path, body)
