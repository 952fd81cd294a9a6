"""Which tiles an experts' product takes (CPU: a HIP runtime that notes launches instead of running them)."""

from test_operators_device import run_with_recorder
from test_operators_limits import TOP

EXPERTS = TOP + """
def side(rows, experts, n, dtype):
    assert attempt(P.pccl_f8_expert_matmul, M, M, M, M, rows, experts, n, 2048, M, M, dtype, n) == 1
    up = lambda a, b: (a + b - 1) // b
    grids = {s: (rows // s + min(experts, rows)) * up(n, s) for s in (128, 256)}
    assert noted[0].grid[0] in grids.values(), (rows, experts, n)
    return 256 if noted[0].grid[0] == grids[256] else 128


for experts in (1, 2, 16, 61, 62, 64, 128, 256):
    for n in (520, 1000, 2048, 4096, 5120, 8192, 14336):
        for rows in {1, 16, 127, 128, 192, 255, 256, 257, 64 * experts - 1, 64 * experts + 3, 100 * experts, 128 * experts}:
            for dtype in (P.PCCL_F32, P.PCCL_BF16, P.PCCL_F16):
                if rows <= 128 * experts:
                    assert side(rows, experts, n, dtype) == 128, (rows, experts, n, dtype)
for rows in (130, 192, 255):   # one expert, fewer rows than a large tile has
    assert side(rows, 1, 4096, P.PCCL_BF16) == side(rows, 1, 4096, P.PCCL_F32) == 128
assert side(32768, 64, 4096, P.PCCL_BF16) == 256
print("as measured")
"""


def test_experts_of_few_rows_take_small_tiles(tmp_path):
    assert "as measured" in run_with_recorder(tmp_path, EXPERTS)


def test_every_kernel_of_few_rows_is_run():
    from test_gpu_operators8_steps import MADE, MOST, SHAPES, kernel
    reached = {kernel(m, 128 * blocks) for m in (1, 20, 40, 60) for blocks in range(1, 4097)}
    assert {kernel(m, k) for m, _, k in SHAPES} == reached
    assert reached == {(rows, s) for rows, most in MOST.items() for s in MADE if s <= most}
