"""GPU: 8-bit packing, its products and the experts' products against the 64-bit oracle.

Codes, scales and blocks are whole numbers and must be equal.  A result of 32
bits is within (k + 2) 2^-24 of the sum of its products' magnitudes.  One of 16
bits may lack, of every eight neighbouring products, what lies below 2^-13 of
the largest one's power of two, and is then rounded: half its last place.
"""

import numpy as np
import pytest

from oracle import operators as O

pytestmark = pytest.mark.gpu

ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}   # half a last place, relative
TINY = {"f32": 0.0, "bf16": 0.0, "f16": 2.0 ** -25}               # and below the normal numbers
TYPES = ["f32", "bf16", "f16"]


def _torch():
    import torch
    return torch


def _type(name):
    t = _torch()
    return {"f32": t.float32, "bf16": t.bfloat16, "f16": t.float16}[name]


@pytest.fixture(scope="module")
def ops():
    from paper_2606_07019_amd.operators import Operators
    o = Operators(0)
    yield o
    o.close()


def _to(a, dtype="f32"):
    return _torch().from_numpy(np.ascontiguousarray(a)).to("cuda").to(_type(dtype))


def _np(t):
    return t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def _values(rng, rows, cols, dtype):
    """Values over the whole range of the type, on the codes and halfway between them, zeros, and blocks that are not finite."""
    span = {"f32": 120, "bf16": 120, "f16": 12}[dtype]
    x = rng.normal(size=(rows, cols)) * np.exp2(rng.integers(-span, span, size=(rows, 1)))
    ties = (rng.integers(-64, 65, size=(rows, cols)) / 4.0) * np.exp2(rng.integers(-4, 5, size=(rows, cols)))
    x = np.where(rng.random((rows, 1)) < 0.4, ties, x)
    x[rng.random((rows, cols)) < 0.01] = 448.0                   # the largest code, and just past it
    x[rng.random((rows, cols)) < 0.01] = 450.0
    x[rng.random((rows, cols)) < 0.02] = 0.0
    x[rng.random((rows, cols)) < 0.0005] = np.inf
    x[rng.random((rows, cols)) < 0.0005] = np.nan
    x[rng.random(rows) < 0.1] = 0.0
    if dtype != "f16":
        x[rng.random(rows) < 0.1] = -0.0
        small = rng.random(rows) < 0.1                           # below the normal numbers
        x[small] = (rng.integers(-127, 128, size=(int(small.sum()), cols))) * 2.0 ** -133
    return _to(x, dtype)


def _same(q, want, tiles=False):
    codes, scales = O.f8_quantize(want, tiles)
    np.testing.assert_array_equal(q.scales.cpu().numpy(), scales)
    np.testing.assert_array_equal(q.codes.cpu().numpy(), codes)
    return codes, scales


SHAPES = [(1, 1), (1, 128), (3, 127), (5, 129), (128, 128), (129, 33), (130, 257), (7, 1000), (300, 640), (16, 513)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_packing(ops, rows, cols, dtype):
    print(f"[operators8] packing {rows}x{cols} {dtype}", flush=True)
    t = _torch()
    x = _values(np.random.default_rng(rows * 1000 + cols), rows, cols, dtype)
    both = ops.quantize8_both(x)
    for q, want in zip(both, (_np(x), _np(x).T)):
        codes, scales = _same(q, want)
        np.testing.assert_array_equal(_np(ops.dequantize8(q, t.float32)), O.f8_values(codes, scales, want.shape[1]))
    for one, q in ((ops.quantize8(x), both[0]), (ops.quantize8_columns(x), both[1])):
        assert t.equal(one.codes, q.codes) and t.equal(one.scales, q.scales)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_packing_in_tiles(ops, rows, cols, dtype):
    print(f"[operators8] tiles {rows}x{cols} {dtype}", flush=True)
    x = _values(np.random.default_rng(rows * 1000 + cols), rows, cols, dtype)
    r, c = ops.quantize8_tiles(x)
    _same(r, _np(x), True)
    _same(c, _np(x).T, True)
    np.testing.assert_array_equal(_np(ops.dequantize8(r, x.dtype)), _np(ops.dequantize8(c, x.dtype)).T)


def test_packing_of_several_matrices(ops):
    print("[operators8] several matrices", flush=True)
    t = _torch()
    x = _values(np.random.default_rng(2), 3 * 200, 140, "bf16").view(3, 200, 140)
    r, c = ops.quantize8_tiles(x)
    assert r.codes.shape == (3, 200, 256) and c.codes.shape == (3, 140, 256) and c.scales.shape == (3, 140, 4)
    for i in range(3):
        for q, one in zip((r, c), ops.quantize8_tiles(x[i])):
            assert t.equal(q.codes[i], one.codes) and t.equal(q.scales[i], one.scales)
    for shape in ((0, 200, 140), (3, 0, 140), (3, 200, 0)):   # of none, and of matrices of nothing
        for q, (rows, cols) in zip(ops.quantize8_tiles(x.new_empty(shape)), (shape[1:], shape[:0:-1])):
            cb, sb = -(-cols // 128) * 128, -(-cols // 512) * 4
            assert q.codes.shape == (shape[0], rows, cb) and q.scales.shape == (shape[0], rows, sb) and q.cols == cols
            assert ops.dequantize8(q, t.float16).shape == (shape[0], rows, cols)


@pytest.mark.parametrize("dtype", TYPES)
def test_packing_of_strided_and_unaligned_rows(ops, dtype):
    print(f"[operators8] strided packing {dtype}", flush=True)
    whole = _values(np.random.default_rng(3), 270, 211, dtype)
    for x in (whole[:, 1:], whole[::2, 3:100], whole[5:6, 7:8], whole[:, 8:200]):
        for q, want in zip(ops.quantize8_both(x), (_np(x), _np(x).T)):
            _same(q, want)
        _same(ops.quantize8(x), _np(x))
        _same(ops.quantize8_tiles(x)[1], _np(x).T, True)


def test_unpacking_of_every_code_and_scale(ops):
    from paper_2606_07019_amd.operators import F8
    t = _torch()
    codes = np.tile(np.arange(256, dtype=np.uint8), (64, 2))     # 512 a row
    scales = np.arange(256, dtype=np.uint8).reshape(64, 4)
    q = F8(t.from_numpy(codes).cuda(), t.from_numpy(scales).cuda(), 512)
    want = O.f8_values(codes, scales, 512)
    with np.errstate(over="ignore"):                             # 2^127 times 448 passes the largest number
        np.testing.assert_array_equal(_np(ops.dequantize8(q, t.float32)), want.astype(np.float32).astype(np.float64))
        np.testing.assert_array_equal(_np(ops.dequantize8(q, t.float16)), want.astype(np.float16).astype(np.float64))
    with np.errstate(over="ignore"):
        bf16 = t.from_numpy(want.astype(np.float32)).to(t.bfloat16)
    np.testing.assert_array_equal(_np(ops.dequantize8(q, t.bfloat16)), _np(bf16))


COUNTS = [[5], [0, 0, 0], [128, 128], [129, 0, 1, 300], [0, 700, 0], [1] * 40, [100, -3, 60], [256, 257, 255], [50, 10 ** 9, 7]]


@pytest.mark.parametrize("counts", COUNTS, ids=lambda c: "-".join(map(str, c[:4])))
@pytest.mark.parametrize("rows", [0, 1, 900, 512])
def test_groups(ops, counts, rows):
    print(f"[operators8] groups {counts} of {rows}", flush=True)
    from paper_2606_07019_amd.operators import group_blocks
    t = _torch()
    g = ops.expert_groups(t.tensor(counts, dtype=t.int32, device="cuda"), rows)
    table, e = g.table.cpu().numpy(), len(counts)
    at = e + 2
    assert table[e + 1] == len(O.expert_blocks(counts, rows, 256)[1])
    for block in (128, 256):
        starts, want = O.expert_blocks(counts, rows, block)
        if block == 128:
            np.testing.assert_array_equal(table[:e + 1], starts)
        room = group_blocks(e, rows, block)
        assert len(want) <= room
        got = table[at:at + 2 * room].reshape(room, 2)
        np.testing.assert_array_equal(got[:len(want)], [[r, x | n << 16] for r, n, x in want] if want else np.zeros((0, 2)))
        assert (got[len(want):] == 0).all()
        at += 2 * room
    assert at == len(table)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("counts", [[129, 0, 1, 300], [0, 64, 0], [7]], ids=["uneven", "one", "rest"])
def test_packing_by_experts(ops, counts, dtype):
    print(f"[operators8] packing by experts {counts} {dtype}", flush=True)
    from paper_2606_07019_amd.operators import F8, group_blocks
    from paper_2606_07019_amd import pccl as P
    t = _torch()
    rows, cols = sum(counts) + (5 if len(counts) < 4 else 0), 300
    x = _values(np.random.default_rng(4), rows, cols, dtype)
    g = ops.expert_groups(t.tensor(counts, dtype=t.int32, device="cuda"), rows)
    r, c = ops.quantize8_both(x, g)
    used = sum(counts)
    codes, scales = O.f8_quantize(_np(x))
    np.testing.assert_array_equal(r.codes[:used].cpu().numpy(), codes[:used])
    np.testing.assert_array_equal(r.scales[:used].cpu().numpy(), scales[:used])
    assert c.cols == 128 * group_blocks(len(counts), rows)
    one = ops.quantize8_columns(x, g)
    for j, (first, n, _) in enumerate(O.expert_blocks(counts, rows)[1]):
        codes, scales = O.f8_quantize(_np(x)[first:first + n].T)
        for q in (c, one):
            np.testing.assert_array_equal(q.codes[:, 128 * j:128 * j + 128].cpu().numpy(), codes)
            np.testing.assert_array_equal(q.scales[:, j].cpu().numpy(), scales[:, 0])
    # what is no one's is left as it was
    full = [t.full_like(v, 77) for v in (r.codes, r.scales, c.codes, c.scales)]
    P.pccl_f8_quantize_experts(ops.h, x.data_ptr(), P.PCCL_BF16 if dtype == "bf16" else P.PCCL_F32, rows, cols, cols, g.table.data_ptr(),
                               len(counts), *[v.data_ptr() for v in full], t.cuda.current_stream().cuda_stream)
    blocks = O.expert_blocks(counts, rows)[0][-1]
    assert (full[0][used:] == 77).all() and (full[1][used:] == 77).all() and (full[2][:, 128 * blocks:] == 77).all()
    assert t.equal(full[0][:used], r.codes[:used]) and t.equal(full[2][:, :128 * blocks], c.codes[:, :128 * blocks])


# ---- products ---------------------------------------------------------------------

def _packed(rng, rows, cols, lo=120, hi=130, codes=None):
    """Random packed rows; what is stored behind a row is zero."""
    from paper_2606_07019_amd.operators import F8
    t = _torch()
    nb = -(-cols // 128)
    c = np.zeros((rows, nb * 128), np.uint8)
    c[:, :cols] = rng.integers(0, 127, size=(rows, cols)) + 128 * rng.integers(0, 2, size=(rows, cols)) if codes is None else rng.choice(codes, size=(rows, cols))
    s = np.zeros((rows, -(-nb // 4) * 4), np.uint8)
    s[:, :nb] = rng.integers(lo, hi + 1, size=(rows, nb))
    return F8(t.from_numpy(c).cuda(), t.from_numpy(s).cuda(), cols), O.f8_values(c, s, cols)


WHOLE = np.array([0, 0x38, 0x40, 0x44, 0x48, 0x4A, 0x4C, 0x4E, 0xB8, 0xC0, 0xC4, 0xC8, 0xCA, 0xCC, 0xCE], np.uint8)   # 0 ... 7, and their negatives


def _nominal(q):
    """The power of two that a code's exponent stands for, 2^-6 below the normal numbers too, scaled."""
    c = q.codes.cpu().numpy() & 127
    s = np.exp2(q.scales.cpu().numpy().astype(np.float64) - 127)
    return np.exp2(np.maximum(c >> 3, 1) - 7.0) * np.repeat(s, 128, axis=1)[:, :c.shape[1]]


def _bound(a, av, b, bv, dtype):
    """How far a product may be from av bv^T, rounding to its type left out."""
    k = av.shape[1]
    bound = (k + 2) * 2.0 ** -24 * (np.abs(av) @ np.abs(bv).T)
    if dtype != "f32":
        na, nb = _nominal(a), _nominal(b)
        for g in range(0, na.shape[1], 8):
            most = np.zeros((na.shape[0], nb.shape[0]))
            for i in range(g, g + 8):
                most = np.maximum(most, na[:, i:i + 1] * nb[:, i])
            bound += 8 * 2.0 ** -13 * most
    return bound


def _close(got, want, bound, dtype):
    assert (np.abs(got - want) <= bound * (1 + ULP[dtype]) + ULP[dtype] * np.abs(want) * 1.01 + TINY[dtype]).all()


PRODUCTS = [(1, 1, 1), (1, 16, 128), (1, 17, 33), (3, 100, 129), (16, 64, 4096), (17, 40, 300), (33, 1000, 256), (48, 31, 1111),
            (64, 129, 640), (65, 1, 5), (65, 128, 128), (100, 130, 384), (129, 257, 700), (300, 520, 1025), (257, 64, 2048)]


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("m,n,k", PRODUCTS + [(2200, 4100, 160)])
def test_product_is_exact_on_whole_numbers(ops, m, n, k, dtype):
    # values up to 7, so that nothing lies below 2^-13 of a product and sums pass through 16 bits' whole numbers
    print(f"[operators8] product {m}x{n}x{k} {dtype}, whole numbers", flush=True)
    rng = np.random.default_rng(m + 7 * n + 13 * k)
    a, av = _packed(rng, m, k, 127, 127, WHOLE)
    b, bv = _packed(rng, n, k, 127, 127, WHOLE)
    want = av @ bv.T
    if dtype == "f16":
        want = want.astype(np.float16).astype(np.float64)
    np.testing.assert_array_equal(_np(ops.matmul8(a, b, _type(dtype))), want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product(ops, m, n, k, dtype):
    print(f"[operators8] product {m}x{n}x{k} {dtype}", flush=True)
    rng = np.random.default_rng(m + 7 * n + 13 * k)
    a, av = _packed(rng, m, k, 116, 122)
    b, bv = _packed(rng, n, k, 112, 118)
    _close(_np(ops.matmul8(a, b, _type(dtype))), av @ bv.T, _bound(a, av, b, bv, dtype), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n", [(5, 40), (200, 300)])
def test_product_of_blocks_that_are_not_numbers(ops, m, n, dtype):
    print(f"[operators8] NaN blocks {m}x{n} {dtype}", flush=True)
    rng = np.random.default_rng(5)
    a, av = _packed(rng, m, 640)
    b, bv = _packed(rng, n, 640)
    a.scales[m - 1, 3] = 255
    b.scales[2, 4] = 255
    a.codes[1, 600] = 127                                        # a value that is not a number
    got = _np(ops.matmul8(a, b, _type(dtype)))
    nan = np.zeros((m, n), bool)
    nan[m - 1], nan[:, 2], nan[1] = True, True, True
    np.testing.assert_array_equal(np.isnan(got), nan)


def test_product_into_a_view_and_of_nothing(ops):
    print("[operators8] product into a view", flush=True)
    t = _torch()
    rng = np.random.default_rng(6)
    for m, n in ((20, 33), (140, 33)):
        for dtype in ("f32", "bf16"):
            a, av = _packed(rng, m, 64, 127, 127, WHOLE)
            b, bv = _packed(rng, n, 64, 127, 127, WHOLE)
            room = t.full((m, n + 8), 7.0, device="cuda", dtype=_type(dtype))
            ops.matmul8(a, b, room.dtype, out=room[:, 3:3 + n])
            want = np.full((m, n + 8), 7.0)
            want[:, 3:3 + n] = _np(_to(av @ bv.T, dtype))
            np.testing.assert_array_equal(_np(room), want)
    a, _ = _packed(rng, 0, 64)
    assert ops.matmul8(a, b, t.float32).shape == (0, 33)
    a, _ = _packed(rng, 4, 0)
    b, _ = _packed(rng, 6, 0)
    assert (ops.matmul8(a, b, t.bfloat16) == 0).all() and (ops.matmul8(a, b, t.float32) == 0).all()


EXPERTS = [([5], 5, 16, 128), ([0, 3, 0], 10, 33, 130), ([129, 0, 1, 300], 430, 140, 300), ([1] * 17, 17, 65, 520), ([256, 257, 31], 600, 200, 640),
           ([0, 0], 4, 20, 20), ([2, 700, 40], 742, 264, 1100)]


def _experts(rng, experts, n, k, *args):
    from paper_2606_07019_amd.operators import F8
    q, v = _packed(rng, experts * n, k, *args)
    return F8(q.codes.view(experts, n, -1), q.scales.view(experts, n, -1), k), v.reshape(experts, n, k)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("counts,rows,n,k", EXPERTS, ids=lambda v: "-".join(map(str, v[:3])) if isinstance(v, list) else str(v))
def test_experts_product(ops, counts, rows, n, k, dtype):
    print(f"[operators8] experts {counts} of {rows}, {n}x{k} {dtype}", flush=True)
    from paper_2606_07019_amd.operators import F8
    t = _torch()
    rng = np.random.default_rng(n + k)
    a, av = _packed(rng, rows, k, 116, 122)
    w, wv = _experts(rng, len(counts), n, k, 112, 118)
    g = ops.expert_groups(t.tensor(counts, dtype=t.int32, device="cuda"), rows)
    room = t.full((rows, n + 5), 7.0, device="cuda", dtype=_type(dtype))
    got = _np(ops.expert_matmul8(a, w, g, room.dtype, out=room[:, 2:2 + n]))
    at = 0
    for e, c in enumerate(counts):
        one = F8(a.codes[at:at + c], a.scales[at:at + c], k)
        _close(got[at:at + c], av[at:at + c] @ wv[e].T, _bound(one, av[at:at + c], F8(w.codes[e], w.scales[e], k), wv[e], dtype), dtype)
        at += c
    assert (got[at:] == 7).all() and (room[:, :2] == 7).all() and (room[:, 2 + n:] == 7).all()
    made = _np(ops.expert_matmul8(a, w, g, room.dtype))
    np.testing.assert_array_equal(made[:at], got[:at])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("counts,rows,m,n", EXPERTS, ids=lambda v: "-".join(map(str, v[:3])) if isinstance(v, list) else str(v))
def test_experts_gradient(ops, counts, rows, m, n, dtype):
    print(f"[operators8] gradient {counts} of {rows}, {m}x{n} {dtype}", flush=True)
    from paper_2606_07019_amd.operators import F8
    t = _torch()
    rng = np.random.default_rng(n + m)
    x, dy = rng.normal(size=(rows, n)) * 10, rng.normal(size=(rows, m))
    x[:, n // 2] *= 30
    x, dy = _to(x, "bf16"), _to(dy, "bf16")
    g = ops.expert_groups(t.tensor(counts, dtype=t.int32, device="cuda"), rows)
    a, b = ops.quantize8_columns(dy, g), ops.quantize8_both(x, g)[1]
    got = _np(ops.expert_gradient8(a, b, g, _type(dtype)))
    assert got.shape == (len(counts), m, n)
    starts, _ = O.expert_blocks(counts, rows)
    for e in range(len(counts)):
        if starts[e] == starts[e + 1]:
            assert (got[e] == 0).all()
            continue
        cut = slice(128 * starts[e], 128 * starts[e + 1])
        part = [F8(q.codes[:, cut].contiguous(), q.scales[:, starts[e]:starts[e + 1]].contiguous(), cut.stop - cut.start) for q in (a, b)]
        v = [O.f8_values(q.codes.cpu().numpy(), q.scales.cpu().numpy(), q.cols) for q in part]
        _close(got[e], v[0] @ v[1].T, _bound(part[0], v[0], part[1], v[1], dtype), dtype)


# ---- balance loss ---------------------------------------------------------------------

BALANCES = [(1, 1, 1), (1, 64, 4), (2, 8, 8), (63, 61, 3), (65, 65, 2), (200, 128, 8), (257, 200, 1), (130, 256, 32), (70, 300, 8),
            (129, 512, 6), (33, 1000, 5), (66, 1024, 32), (5000, 17, 17)]


def _balance_inputs(rng, tokens, experts, topk, dtype, barred):
    l = rng.normal(size=(tokens, experts)) * 3
    mask = None
    if barred:
        l[rng.random((tokens, experts)) < 0.3] = -np.inf
        l[rng.random(tokens) < 0.1] = -np.inf
        mask = (rng.random(tokens) >= 0.1).astype(np.uint8)
    logits = _to(l, dtype)
    ids = O.route(_np(logits), topk, True, mask)[1]
    if barred:                                                    # picks of rows that do not count, and of no expert
        ids[rng.random(ids.shape) < 0.1] = 7 * experts
    t = _torch()
    return logits, t.from_numpy(ids).cuda(), None if mask is None else t.from_numpy(mask).cuda()


@pytest.mark.parametrize("barred", [False, True], ids=["all", "barred"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,experts,topk", BALANCES)
def test_balance(ops, tokens, experts, topk, dtype, barred):
    print(f"[operators8] balance {tokens}x{experts}, {topk} {dtype} {barred}", flush=True)
    t = _torch()
    rng = np.random.default_rng(tokens + experts)
    logits, ids, mask = _balance_inputs(rng, tokens, experts, topk, dtype, barred)
    _balance_checked(ops, rng, logits, ids, mask, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,experts,topk", [(70, 61, 3), (300, 256, 8), (140, 520, 4)])
def test_balance_of_lowest_values_of_padding_and_of_strided_rows(ops, tokens, experts, topk, dtype):
    print(f"[operators8] balance {tokens}x{experts} lowest, padding, strides {dtype}", flush=True)
    t = _torch()
    rng = np.random.default_rng(tokens)
    logits, ids, mask = _balance_inputs(rng, tokens, experts, topk, dtype, True)
    lowest = t.finfo(logits.dtype).min
    low = t.where(logits == -float("inf"), lowest, logits)        # barred by the type's lowest value: whole rows are even then
    _balance_checked(ops, rng, low, ids, mask, dtype)
    garbage = logits.clone()                                      # what padding holds does not count
    off = (mask == 0).nonzero().flatten()
    assert len(off) >= 3
    garbage[off[0]], garbage[off[1]], garbage[off[2], 0] = float("nan"), float("inf"), float("nan")
    for got, want in zip(ops.balance_loss(garbage, ids, mask=mask), ops.balance_loss(logits, ids, mask=mask)):
        assert t.equal(got, want)
    _, counts, _, rows = ops.balance_loss(logits, ids, mask=mask)
    one = t.ones((), device="cuda")
    assert t.equal(ops.balance_loss_backward(garbage, counts, rows, one, mask=mask), ops.balance_loss_backward(logits, counts, rows, one, mask=mask))
    whole = t.full((tokens * 2, experts + 5), float("nan"), dtype=logits.dtype, device="cuda")
    for view in (whole[::2, 1:experts + 1], whole[:tokens, 4:experts + 4], whole[tokens:, :experts]):
        view.copy_(logits)
        for got, want in zip(ops.balance_loss(view, ids, mask=mask), ops.balance_loss(logits, ids, mask=mask)):
            assert t.equal(got, want)
        assert t.equal(ops.balance_loss_backward(view, counts, rows, one, mask=mask), ops.balance_loss_backward(logits, counts, rows, one, mask=mask))


def _balance_checked(ops, rng, logits, ids, mask, dtype):
    t = _torch()
    tokens, experts = logits.shape
    loss, counts, probs, rows = ops.balance_loss(logits, ids, mask=mask)
    m = None if mask is None else mask.cpu().numpy()
    wl, wc, wp, wr = O.balance(_np(logits), ids.cpu().numpy(), m)
    np.testing.assert_array_equal(counts.cpu().numpy(), wc)
    assert int(rows) == wr
    # a probability: an exponential of 2 ulp whose argument, up to 2^5, is off by 2^-24 of it, over a sum of `experts`
    # such; then `tokens` of them are added up
    share = (2.0 ** 5 + 8 + experts + tokens + 4) * 2.0 ** -24
    assert (np.abs(_np(probs) - wp) <= share * wp).all()
    assert abs(float(loss) - wl) <= (share + (experts + 4) * 2.0 ** -24) * wl
    dloss = t.full((), 3.0, device="cuda")
    dprobs = _to(rng.normal(size=experts), "f32")
    scale = max(1.0, float(wr)) if dtype == "f16" else 1.0       # as a loss scale does
    dloss, dprobs = dloss * scale, dprobs * scale
    for given in (None, dprobs):
        got = _np(ops.balance_loss_backward(logits, counts, rows, dloss, given, mask))
        v = None if given is None else _np(given)
        want = O.balance_backward(_np(logits), wc, wr, float(dloss), v, m)
        # the difference v - sum v p: errors as large as its parts
        size = np.abs(float(dloss) * experts * wc / max(wc.sum(), 1)) + (0 if v is None else np.abs(v))
        p = np.abs(want) * 0
        l = _np(logits).copy()
        if m is not None:
            l[m == 0] = -np.inf
        for i in range(tokens):
            if (l[i] > -np.inf).any():
                e = np.exp(l[i] - l[i].max())
                p[i] = e / e.sum()
        bound = p * (size + (p * size).sum(axis=1, keepdims=True)) / max(wr, 1) * (2.0 ** 5 + 2 * experts + 16) * 2.0 ** -24
        _close(got, want, bound + 1e-44, dtype)


@pytest.mark.parametrize("barred", [False, True], ids=["all", "barred"])
def test_balance_gradient_is_the_difference(barred):
    rng = np.random.default_rng(8)
    l = rng.normal(size=(7, 5))
    mask = None
    if barred:
        l[2], l[3, 1] = -np.inf, -np.inf
        mask = np.array([1, 0, 1, 1, 1, 1, 1])
    ids = O.route(l, 2, True, mask)[1]
    dloss, dprobs = 1.5, rng.normal(size=5)

    def value(x):
        loss, _, probs, _ = O.balance(x, ids, mask)
        return dloss * loss + (dprobs * probs).sum()

    _, counts, _, rows = O.balance(l, ids, mask)
    d = O.balance_backward(l, counts, rows, dloss, dprobs, mask)
    for t in range(7):
        for e in range(5):
            if l[t, e] > -np.inf:
                up, down = l.copy(), l.copy()
                up[t, e] += 1e-5
                down[t, e] -= 1e-5
                assert abs((value(up) - value(down)) / 2e-5 - d[t, e]) < 1e-8


def test_balance_of_nothing_and_of_no_numbers(ops):
    print("[operators8] balance of nothing", flush=True)
    t = _torch()
    ids = t.zeros((0, 2), dtype=t.int32, device="cuda")
    loss, counts, probs, rows = ops.balance_loss(t.zeros((0, 6), device="cuda"), ids)
    assert float(loss) == 0 and int(rows) == 0 and (counts == 0).all() and (probs == 0).all()
    assert ops.balance_loss_backward(t.zeros((0, 6), device="cuda"), counts, rows, loss).shape == (0, 6)
    l = t.full((3, 6), -float("inf"), device="cuda")
    none = t.full((3, 2), -1, dtype=t.int32, device="cuda")
    loss, counts, probs, rows = ops.balance_loss(l, none)
    assert float(loss) == 0 and int(rows) == 0 and (probs == 0).all()
    assert (ops.balance_loss_backward(l, counts, rows, t.ones((), device="cuda")) == 0).all()
    l = t.zeros((3, 6), device="cuda")
    loss, counts, probs, rows = ops.balance_loss(l, none)        # rows without picks
    assert float(loss) == 0 and int(rows) == 3 and (counts == 0).all()
    assert (ops.balance_loss_backward(l, counts, rows, t.ones((), device="cuda")) == 0).all()
    picks = t.tensor([[0, 1], [2, 3], [4, 5]], dtype=t.int32, device="cuda")
    assert abs(float(ops.balance_loss(l, picks)[0]) - 1) < 8 * 2.0 ** -24
    for bad in (float("nan"), float("inf")):
        l[1, 2] = bad
        loss, counts, probs, rows = ops.balance_loss(l, picks)
        assert int(rows) == 3 and (counts == 1).all() and bool(loss.isnan())
        d = ops.balance_loss_backward(l, counts, rows, t.ones((), device="cuda"))
        assert d[1].isnan().any() and not d[0].isnan().any() and not d[2].isnan().any()


def test_balance_under_automatic_differentiation(ops):
    print("[operators8] balance, autograd", flush=True)
    t = _torch()
    rng = np.random.default_rng(9)
    logits, ids, mask = _balance_inputs(rng, 50, 12, 3, "f32", True)
    l = logits.clone().requires_grad_()
    loss, counts, probs, rows = ops.balance_loss(l, ids, mask=mask)
    assert loss.requires_grad and probs.requires_grad and not counts.requires_grad and not rows.requires_grad
    g = _to(rng.normal(size=12), "f32")
    for out, dloss, dprobs in ((2 * loss, 2.0, None), ((probs * g).sum(), None, g), (loss + (probs * g).sum(), 1.0, g)):
        grad, = t.autograd.grad(out, l, retain_graph=True)
        want = ops.balance_loss_backward(logits, counts, rows, None if dloss is None else t.full((), dloss, device="cuda"), dprobs, mask)
        assert t.equal(grad, want)
    # the loss of a joint batch from the counts of all ranks, through the probabilities
    both, n = counts * 2 + 1, rows * 2
    joint = (both.float() / both.sum() * 12 * probs).sum() * (rows / n)
    grad, = t.autograd.grad(joint, l)
    want = ops.balance_loss_backward(logits, both, n, t.ones((), device="cuda"), None, mask)
    assert (grad - want).abs().max() <= 64 * 2.0 ** -24 * want.abs().max()
