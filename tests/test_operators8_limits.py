"""The 8-bit operators, the experts' products and the balance loss without a GPU
(a HIP runtime that notes launches instead of running them): what is refused
launches nothing, what is within the stated limits is launched in grids that a
launch can have, and the caller's current device stays as it was."""

import os
import re

import pytest

from paper_2606_07019_amd import pccl as P
from test_operators_device import run_with_recorder
from test_operators_limits import TOP

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

REFUSALS = TOP + """
EI, EU, EM = "EINVAL", "EUNSUPPORTED", "ENOMEM"
Q = P.pccl_f8_quantize
assert attempt(Q, M, 7, 1, 4, 4, 4, 0, M, M) == EI                       # type
assert attempt(Q, None, 0, 1, 4, 4, 4, 0, M, M) == EI
assert attempt(Q, M + 1, 0, 1, 4, 4, 4, 0, M, M) == EI
assert attempt(Q, M, 0, 1, 4, 4, 3, 0, M, M) == EI                       # stride below the row
assert attempt(Q, M, 0, 1, 4, 4, 4, 0) == EI                             # no output
assert attempt(Q, M, 0, 1, 4, 4, 4, 0, M, None) == EI
assert attempt(Q, M, 0, 1, 4, 4, 4, 0, M + 8, M) == EI
assert attempt(Q, M, 0, 1, 4, 4, 4, 0, None, None, M, M + 2) == EI
assert attempt(Q, M, 0, 1, 4, 4, 4, 1, M, M) == EI                       # tiles go both ways
assert attempt(Q, M, 0, 1, 1 << 31, 4, 4, 0, M, M) == EU
assert attempt(Q, M, 0, 1 << 16, 1 << 16, 4, 4, 0, M, M) == EU           # rows of all matrices
assert attempt(Q, M, 0, 1 << 20, 1, 1 << 12, 1 << 12, 1, M, M, M, M) == EU   # columns of all matrices
assert attempt(Q, None, 0, 1, 0, 4, 4, 0, M, M) == 0 and attempt(Q, None, 0, 0, 4, 4, 4, 1) == 0
X = P.pccl_f8_quantize_experts
assert attempt(X, M, 0, 4, 4, 4, None, 2, M, M, M, M) == EI              # no groups
assert attempt(X, M, 0, 4, 4, 4, M, 0, M, M, M, M) == EI                 # no experts
assert attempt(X, M, 0, 4, 4, 4, M, 1025, M, M, M, M) == EU
assert attempt(X, M, 0, 4, 4, 4, M, 2, M, M) == EI                       # the columns are what it is for
assert attempt(X, M, 0, 0, 4, 4, None, 2) == 0
D = P.pccl_f8_dequantize
assert attempt(D, None, M, 4, 4, M, 0, 4) == EI and attempt(D, M, M, 4, 4, M, 0, 2) == EI and attempt(D, None, None, 0, 4, None, 0, 4) == 0
G = P.pccl_moe_groups
assert attempt(G, M, 0, 4, M) == EI and attempt(G, M, 1025, 4, M) == EU and attempt(G, M, 4, 1 << 31, M) == EU
assert attempt(G, None, 4, 4, M) == EI and attempt(G, M, 4, 4, None) == EI and attempt(G, M + 2, 4, 4, M) == EI
T = P.pccl_f8_matmul
assert attempt(T, None, M, M, M, 4, 4, 4, M, 0, 4) == EI
assert attempt(T, M, M, M, M + 1, 4, 4, 4, M, 0, 4) == EI
assert attempt(T, M, M, M, M, 4, 4, 4, M, 0, 3) == EI
assert attempt(T, M, M, M, M, 4, 4, (1 << 23) + 1, M, 0, 4) == EU
assert attempt(T, M, M, M, M, 70, 128, 1 << 13, M, 0, 128) == EI         # workspace missing
assert attempt(T, M, M, M, M, 70, 128, 1 << 13, M, 0, 128, M, 16) == EM
assert attempt(T, M, M, M, M, 70, 128, 1 << 13, M, 0, 128, M + 64, 1 << 30) == EI
assert attempt(T, None, None, None, None, 0, 4, 4, None, 0, 4) == 0 and attempt(T, None, None, None, None, 4, 4, 0, M, 0, 4) == 1
E = P.pccl_f8_expert_matmul
assert attempt(E, M, M, M, M, 4, 2, 4, 4, None, M, 0, 4) == EI           # no groups
assert attempt(E, None, M, M, M, 4, 2, 4, 4, M, M, 0, 4) == EI
assert attempt(E, M, M, M, M, 4, 0, 4, 4, M, M, 0, 4) == EI
assert attempt(E, M, M, M, M, 4, 2, 4, 4, M, M, 0, 3) == EI
assert attempt(E, M, M, M, M, 4, 2, 4, 1 << 24, M, M, 0, 4) == EU
assert attempt(E, None, None, None, None, 0, 2, 4, 4, None, None, 0, 4) == 0
W = P.pccl_f8_expert_gradient
assert attempt(W, M, M, M, M, 4, 2, 4, 4, None, M, 0) == EI
assert attempt(W, M, None, M, M, 4, 2, 4, 4, M, M, 0) == EI
assert attempt(W, M, M, M, M, 4, 2, 4, 4, M, M + 1, 0) == EI
assert attempt(W, M, M, M, M, 1 << 23, 2, 4, 4, M, M, 0) == EU           # blocks
assert attempt(W, None, None, None, None, 0, 2, 4, 4, M, M, 0) == 1      # no rows: zeros
B = P.pccl_moe_balance
space = P.pccl_moe_balance_workspace(h, 1000, 8)
assert P.pccl_moe_balance_workspace(h, 100, 8) == 0 and attempt(B, M, 0, 100, 8, 8, M, 2, None, M, M, M, M) == 1   # one launch
ok = (M, 0, 1000, 8, 8, M, 2, None, M, M, M, M)
assert attempt(B, *ok, M, space) == 2
assert attempt(B, *ok, M, space - 1) == EM and attempt(B, *ok) == EI and attempt(B, *ok, M + 4, space) == EI
for i, bad, want in ((1, 9, EI), (3, 0, EI), (3, 1025, EU), (4, 7, EI), (5, None, EI), (6, 0, EI), (6, 9, EI), (8, None, EI), (9, None, EI), (10, None, EI), (11, M + 2, EI)):
    args = list(ok)
    args[i] = bad
    assert attempt(B, *args, M, space) == want, (i, bad)
assert attempt(B, M, 0, 100, 1025, 1025, M, 2, None, M, M, M, M, M, 1 << 30) == EU
assert attempt(B, None, 0, 0, 8, 8, None, 2, None, M, M, M, M) == 1   # no tokens: zeros
K = P.pccl_moe_balance_backward
assert attempt(K, M, 0, 4, 8, 8, None, M, M, M, None, M, 8) == 1 and attempt(K, M, 0, 4, 8, 8, None, M, M, None, None, M, 8) == 1
assert attempt(K, M, 0, 4, 8, 8, None, None, M, M, None, M, 8) == EI and attempt(K, M, 0, 4, 8, 8, None, M, None, M, None, M, 8) == EI
assert attempt(K, M, 0, 4, 8, 8, None, M, M, M + 1, None, M, 8) == EI and attempt(K, M, 0, 4, 8, 8, None, M, M, M, None, M, 7) == EI
assert attempt(K, None, 0, 0, 8, 8, None, M, M, M, None, None, 8) == 0
print("refused")
"""

LARGEST = TOP + """
EU = "EUNSUPPORTED"
for rows, cols in ((1 << 24, 8), (TOP, 1), (1 << 28, 600), (TOP, 512), (1 << 24, 70000)):
    assert attempt(P.pccl_f8_quantize, M, P.PCCL_BF16, 1, rows, cols, cols + 3, 0, M, M) == count.value > 0, (rows, cols)
    at = M
    for i in range(count.value):
        assert noted[i].arg[0] == at and noted[i].arg[1] == 1 and noted[i].arg[2] > 0      # x, batch, rows
        at += noted[i].arg[2] * (cols + 3) * 2
    assert at == M + rows * (cols + 3) * 2, (rows, cols)
for rows, cols in ((1000, 70000), (1 << 26, 8), (TOP, 1), (1 << 24, 70000)):
    assert attempt(P.pccl_f8_dequantize, M, M, rows, cols, M, P.PCCL_BF16, cols + 3) == count.value > 0, (rows, cols)
    at = M
    for start, n in slices(0, 2):
        assert start == at and n > 0
        at += n * ((cols + 127) // 128 * 128)
    assert at == M + rows * ((cols + 127) // 128 * 128), (rows, cols)
for batch, rows, cols, want in ((1, 70000, 70000, 1), (1, 256, TOP, EU), (1, 128, (1 << 30) - 128, 1), (1, TOP, 128, EU), (61, 1000, 2040, 1), (1 << 12, 1 << 12, 1 << 12, 1), (1 << 13, 1 << 13, 1 << 13, EU)):
    for tiles in (0, 1):
        assert attempt(P.pccl_f8_quantize, M, P.PCCL_BF16, batch, rows, cols, cols, tiles, M, M, M, M) == want, (batch, rows, cols)
for rows, cols, want in ((1 << 20, 8192, 1), (1 << 30, 128, EU), ((1 << 30) - 2000 * 128, 1, 1)):
    assert attempt(P.pccl_f8_quantize_experts, M, P.PCCL_BF16, rows, cols, cols, M, 1000, M, M, M, M) == want, (rows, cols)
for m, n, k, want in ((131072, 131072, 256, 1), (200000, 200000, 256, 1), (1, 1 << 27, 256, 1), (64, TOP, 256, 1), (1 << 20, 1 << 20, 256, EU),
                      (TOP, 1, 256, EU), (65, TOP, 256, EU), (70, 10000, 1 << 23, 2), (70, 20000, 1 << 23, 1), (1, 100, 1 << 23, 2), (64, TOP, 1 << 14, EU)):
    assert attempt(P.pccl_f8_matmul, M, M, M, M, m, n, k, M, P.PCCL_BF16, n, M, 1 << 60) == want, (m, n, k)
for rows, experts, n, want in ((1 << 20, 64, 8192, 1), (TOP - 131072, 1024, 128, 1), (TOP, 1024, 129, EU), (1, 1024, TOP, EU), (1, 1, TOP - 128, 1)):
    assert attempt(P.pccl_f8_expert_matmul, M, M, M, M, rows, experts, n, 256, M, M, P.PCCL_BF16, n) == want, (rows, experts, n)
for rows, experts, m, n, want in ((1 << 20, 1024, 8192, 8192, 1), (1 << 20, 1024, 1 << 15, 1 << 14, EU), ((1 << 23) - 128000, 1000, 128, 128, 1), (1 << 23, 1, 8, 8, EU), (0, 1, 1 << 18, 1 << 18, 1)):
    assert attempt(P.pccl_f8_expert_gradient, M, M, M, M, rows, experts, m, n, M, M, P.PCCL_F32) == want, (rows, experts, m, n)
for experts, rows in ((1024, TOP), (1, 0), (1024, 5)):
    assert attempt(P.pccl_moe_groups, M, experts, rows, M) == 1
for tokens, experts, topk, want in ((TOP // 8, 8, 8, 2), (TOP // 32, 1024, 32, 2), (TOP // 8 + 1, 8, 8, EU), (0, 300, 3, 1)):
    assert attempt(P.pccl_moe_balance, M, P.PCCL_F32, tokens, experts, experts, M, topk, None, M, M, M, M, M, 1 << 40) == want, (tokens, experts)
for tokens, experts in ((TOP, 1), (TOP, 1024), (1, 300)):
    assert attempt(P.pccl_moe_balance_backward, M, P.PCCL_F32, tokens, experts, experts, None, M, M, M, M, M, experts) == 1
print("fit")
"""

DEVICE = """
h = P.pccl_create(1, 0)
calls = [
    lambda m: P.pccl_moe_groups(h, m, 4, 900, M),
    lambda m: P.pccl_f8_quantize(h, m, P.PCCL_BF16, 1, 200, 300, 300, 0, M, M, M, M),
    lambda m: P.pccl_f8_quantize(h, m, P.PCCL_F32, 1, 200, 300, 300, 0, M, M),
    lambda m: P.pccl_f8_quantize(h, m, P.PCCL_F16, 3, 200, 300, 300, 1, M, M, M, M),
    lambda m: P.pccl_f8_quantize_experts(h, m, P.PCCL_BF16, 200, 300, 300, M, 4, M, M, M, M),
    lambda m: P.pccl_f8_dequantize(h, m, M, 200, 300, M, P.PCCL_F32, 300),
    lambda m: P.pccl_f8_matmul(h, m, M, M, M, 7, 300, 300, M, P.PCCL_F32, 300),
    lambda m: P.pccl_f8_matmul(h, m, M, M, M, 7, 300, 30000, M, P.PCCL_F16, 300, M, 1 << 30),
    lambda m: P.pccl_f8_matmul(h, m, M, M, M, 700, 300, 300, M, P.PCCL_BF16, 300),
    lambda m: P.pccl_f8_matmul(h, m, M, M, M, 9000, 9000, 300, M, P.PCCL_F32, 9000),
    lambda m: P.pccl_f8_expert_matmul(h, m, M, M, M, 700, 4, 300, 300, M, M, P.PCCL_BF16, 300),
    lambda m: P.pccl_f8_expert_gradient(h, m, M, M, M, 700, 4, 300, 300, M, M, P.PCCL_F32),
    lambda m: P.pccl_moe_balance(h, m, P.PCCL_BF16, 20, 8, 8, M, 2, None, M, M, M, M, M, 1 << 20),
    lambda m: P.pccl_moe_balance(h, m, P.PCCL_F32, 20000, 500, 500, M, 2, None, M, M, M, M, M, 1 << 30),
    lambda m: P.pccl_moe_balance_backward(h, m, P.PCCL_F32, 20, 8, 8, None, M, M, M, None, M, 8),
]
for i, call in enumerate(calls):
    for at in (0, 1):
        now.value, count.value = at, 0
        call(M)
        assert now.value == at, (i, at, "a call that succeeds")
        assert count.value and all(noted[j].device == 1 for j in range(count.value)), (i, at)
        for address, error in ((None, 0), (M, 98)):
            broken.value = error
            try:
                call(address)
            except P.PcclError as e:
                assert e.name == ("PCCL_EDEVICE" if error else "PCCL_EINVAL"), (i, e)
            else:
                raise AssertionError(i)
            assert now.value == at, (i, at, "a call that fails")
print("left alone")
"""


@pytest.mark.parametrize("body,word", [(REFUSALS, "refused"), (LARGEST, "fit"), (DEVICE, "left alone")], ids=["refusals", "largest", "device"])
def test_calls(tmp_path, body, word):
    assert word in run_with_recorder(tmp_path, body)


def test_the_binding_has_every_name_of_the_header():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "pccl.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(pccl_\w+)\s*\(", text))
    assert {"pccl_f8_quantize", "pccl_f8_expert_gradient", "pccl_moe_balance"} <= names
    lib = P.load_library()
    for n in names:
        assert hasattr(lib, n) and callable(getattr(P, n)), n


def test_refusals_of_tensors(monkeypatch):
    torch = pytest.importorskip("torch")
    from paper_2606_07019_amd import operators as W
    ops = W.Operators.__new__(W.Operators)
    ops.device, ops.h = torch.device("cpu"), None
    called = []
    monkeypatch.setattr(W.Operators, "_call", lambda self, function, *args: called.append(function))
    monkeypatch.setattr(W.Operators, "_space", lambda self, ask, *sizes: (None, None, 0))
    monkeypatch.setattr(W.Operators, "_stream", lambda self: None)
    ops._lib = P.load_library()
    f32, bf16, i32 = torch.float32, torch.bfloat16, torch.int32
    x = torch.zeros(6, 8)

    def packed(*shape):
        cb, sb = W.f8_bytes(shape[-1])
        return W.F8(torch.zeros(*shape[:-1], cb, dtype=torch.uint8), torch.zeros(*shape[:-1], sb, dtype=torch.uint8), shape[-1])

    g = ops.expert_groups(torch.zeros(3, dtype=i32), 6)
    cols = 128 * W.group_blocks(3, 6)
    q, w, c = packed(6, 8), packed(3, 4, 8), packed(5, cols)
    mine = torch.zeros(6, 4)
    loss, counts, probs, rows = ops.balance_loss(x, torch.zeros(6, 2, dtype=i32))
    good = [lambda: ops.quantize8(x), lambda: ops.quantize8_both(x, g), lambda: ops.quantize8_tiles(torch.zeros(2, 3, 4)), lambda: ops.quantize8_tiles(torch.zeros(0, 3, 4)),
            lambda: ops.quantize8_tiles(torch.zeros(2, 3, 0)), lambda: ops.quantize8_tiles(torch.zeros(2, 6, 4)[:, ::2]), lambda: ops.dequantize8(w, bf16),
            lambda: ops.matmul8(q, packed(4, 8), f32, out=mine), lambda: ops.expert_matmul8(q, w, g, f32, out=mine), lambda: ops.expert_gradient8(c, c, g, f32),
            lambda: ops.balance_loss(x, torch.zeros(6, 2, dtype=i32), mask=torch.ones(6, dtype=torch.bool)),
            lambda: ops.balance_loss_backward(x, counts, rows, loss, probs)]
    bad = [lambda: ops.quantize8(x.double()), lambda: ops.quantize8(x.t()), lambda: ops.quantize8(x[0]), lambda: ops.quantize8(torch.zeros(2, 3, 4)),
           lambda: ops.quantize8_both(torch.zeros(7, 8), g), lambda: ops.quantize8_columns(x, g._replace(table=g.table[1:])),
           lambda: ops.quantize8_tiles(torch.zeros(2, 6, 4)[:, :3]), lambda: ops.quantize8_tiles(torch.zeros(2, 3, 4).transpose(1, 2)),
           lambda: ops.dequantize8(q, torch.int8), lambda: ops.dequantize8(q._replace(cols=200), f32), lambda: ops.dequantize8(q._replace(codes=q.codes.float()), f32),
           lambda: ops.matmul8(q, packed(4, 9), f32), lambda: ops.matmul8(q, w, f32), lambda: ops.matmul8(q, packed(4, 8), torch.float64),
           lambda: ops.matmul8(q, packed(4, 8), bf16, out=mine), lambda: ops.matmul8(q, packed(4, 8), f32, out=mine.t()),
           lambda: ops.matmul8(q, packed(4, 8), f32, out=torch.zeros(6, 4, requires_grad=True)),
           lambda: ops.expert_groups(torch.zeros(3), 6), lambda: ops.expert_groups(torch.zeros(3, 1, dtype=i32), 6), lambda: ops.expert_groups(torch.zeros(3, dtype=i32), -1),
           lambda: ops.expert_matmul8(packed(7, 8), w, g, f32), lambda: ops.expert_matmul8(q, packed(4, 4, 8), g, f32), lambda: ops.expert_matmul8(q, packed(4, 8), g, f32),
           lambda: ops.expert_matmul8(q, packed(3, 4, 7), g, f32), lambda: ops.expert_matmul8(q, w, g._replace(rows=700), f32),
           lambda: ops.expert_gradient8(c, packed(5, cols + 128), g, f32), lambda: ops.expert_gradient8(q, q, g, f32), lambda: ops.expert_gradient8(c, c, g, i32),
           lambda: ops.balance_loss(x, torch.zeros(6, 2)), lambda: ops.balance_loss(x, torch.zeros(5, 2, dtype=i32)), lambda: ops.balance_loss(x, torch.zeros(6, dtype=i32)),
           lambda: ops.balance_loss(x, torch.zeros(6, 2, dtype=i32), mask=torch.ones(5, dtype=torch.bool)),
           lambda: ops.balance_loss_backward(x, counts[:7], rows, loss), lambda: ops.balance_loss_backward(x, counts, rows, loss.double()),
           lambda: ops.balance_loss_backward(x, counts, rows.view(1), loss), lambda: ops.balance_loss_backward(x, counts, rows, loss, probs[:3])]
    for i, call in enumerate(good):
        called.clear()
        call()
        assert called, i
    for i, call in enumerate(bad):
        called.clear()
        with pytest.raises(ValueError):
            call()
        assert not called, i
    with pytest.raises(RuntimeError):
        with torch.autograd.forward_ad.dual_level():
            ops.balance_loss(torch.autograd.forward_ad.make_dual(x, x), torch.zeros(6, 2, dtype=i32))
