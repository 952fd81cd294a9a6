"""GPU: the 8-bit operators at sizes and values further out: a long k that is
shared out, either side of the rules that choose a form, rows that start
anywhere, offsets past 32 bits, values that are not finite.  Whole results must
be equal; floating ones carry the bounds that tests/test_gpu_operators8.py derives."""

import numpy as np
import pytest

from oracle import operators as O
from test_gpu_operators8 import WHOLE, _experts, _np, _packed, _to, _torch, _type, ops  # noqa: F401

pytestmark = pytest.mark.gpu


def _whole(ops, m, n, k, dtypes=("f32", "bf16")):   # noqa: F811
    """Values up to 7: sums of products, and their bf16 roundings, are exact."""
    rng = np.random.default_rng(m + 7 * n + 13 * k)
    a, av = _packed(rng, m, k, 127, 127, WHOLE)
    b, bv = _packed(rng, n, k, 127, 127, WHOLE)
    want = _torch().from_numpy(av).cuda() @ _torch().from_numpy(bv).cuda().t().contiguous()
    for dtype in dtypes:
        got = ops.matmul8(a, b, _type(dtype))
        assert _torch().equal(got.double(), want.to(_type(dtype)).double()), dtype


# every number of steps that a wave of the few-row form holds, with whole and broken last ones; k shared out
# between workgroups, evenly and not; more tiles of 16 rows of B than there are workgroups
FEW = [(1, 16, 1024), (5, 33, 1025), (16, 40, 2049), (17, 31, 2900), (33, 64, 3333), (20, 70, 5120), (48, 20, 5100), (49, 20, 5500), (64, 17, 7000),
       (8, 500, 8192), (64, 100, 8193), (7, 33, 20000), (1, 1, 65536), (16, 4100, 700), (33, 8300, 300), (64, 9000, 4096), (1, 9000, 6144)]


@pytest.mark.parametrize("m,n,k", FEW)
def test_product_of_few_rows(ops, m, n, k):   # noqa: F811
    print(f"[operators8] product {m}x{n}x{k}, few rows", flush=True)
    _whole(ops, m, n, k)


# tiles of 128 shared out over k, one and two a compute unit (256 and 257 of them, 512), tiles of 256 (three and
# three and a half rounds to one), broken ends either way
MANY = [(65, 130, 4097), (200, 300, 5000), (129, 257, 9000), (2048, 2048, 256), (2049, 2048, 130), (2048, 4096, 128), (2100, 4100, 300),
        (4000, 4096, 200), (4097, 4160, 129), (100, 33000, 257), (300, 16500, 500), (6000, 6200, 100)]


@pytest.mark.parametrize("m,n,k", MANY)
def test_product_of_many_rows(ops, m, n, k):   # noqa: F811
    print(f"[operators8] product {m}x{n}x{k}, many rows", flush=True)
    _whole(ops, m, n, k)


@pytest.mark.parametrize("m,n,k", [(40, 70, 9000), (129, 257, 9000)])
def test_shared_out_product_into_a_view_with_not_numbers(ops, m, n, k):   # noqa: F811
    print(f"[operators8] shared-out product {m}x{n}x{k}", flush=True)
    t = _torch()
    rng = np.random.default_rng(1)
    a, av = _packed(rng, m, k, 127, 127, WHOLE)
    b, bv = _packed(rng, n, k, 127, 127, WHOLE)
    a.scales[3, 60] = 255
    want = t.from_numpy(av @ bv.T)
    want[3] = float("nan")
    for dtype in ("f32", "f16"):
        room = t.full((m, n + 9), 5.0, device="cuda", dtype=_type(dtype))
        ops.matmul8(a, b, room.dtype, out=room[:, 5:5 + n])
        assert (room[:, :5] == 5).all() and (room[:, 5 + n:] == 5).all()
        np.testing.assert_array_equal(_np(room[:, 5:5 + n]), want.to(_type(dtype)).double().numpy())


# experts in tiles of 128 and of 256, empty ones first, between and last, rows that no one has
MIXES = [([0, 700, 0, 300, 1, 0, 900, 0], 2000, 1100, 300), ([257] * 40, 10280, 1000, 260), ([512] * 16, 8192, 4096, 130), ([3] * 300, 900, 300, 140)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("counts,rows,n,k", MIXES, ids=["mixed", "257", "512", "3"])
def test_experts(ops, counts, rows, n, k, dtype):   # noqa: F811
    print(f"[operators8] {len(counts)} experts, {rows} rows, {n}x{k} {dtype}", flush=True)
    t = _torch()
    rng = np.random.default_rng(n + k)
    a, av = _packed(rng, rows, k, 127, 127, WHOLE)
    w, wv = _experts(rng, len(counts), n, k, 127, 127, WHOLE)
    g = ops.expert_groups(t.tensor(counts, dtype=t.int32, device="cuda"), rows)
    out = t.full((rows, n), 7.0, device="cuda", dtype=_type(dtype))
    got = ops.expert_matmul8(a, w, g, out.dtype, out=out)
    assert got is out
    at, av, wv = 0, t.from_numpy(av).cuda(), t.from_numpy(wv).cuda()
    for e, c in enumerate(counts):
        assert t.equal(out[at:at + c].double(), (av[at:at + c] @ wv[e].t().contiguous()).to(out.dtype).double()), e
        at += c
    assert (out[at:] == 7).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("counts,rows,m,n", [([0, 700, 0, 300, 1, 0, 900, 0], 2000, 270, 130), ([40] * 50, 2000, 700, 1100), ([600] * 16, 9600, 1024, 2048)],
                         ids=["mixed", "50", "16"])
def test_experts_gradient_on_whole_numbers(ops, counts, rows, m, n, dtype):   # noqa: F811
    print(f"[operators8] gradient of {len(counts)} experts, {rows} rows, {m}x{n} {dtype}", flush=True)
    t = _torch()
    gen = t.Generator(device="cuda").manual_seed(m)
    dy, x = (t.randint(-7, 8, (rows, c), generator=gen, device="cuda").to(t.bfloat16) for c in (m, n))
    g = ops.expert_groups(t.tensor(counts, dtype=t.int32, device="cuda"), rows)
    got = ops.expert_gradient8(ops.quantize8_columns(dy, g), ops.quantize8_both(x, g)[1], g, _type(dtype))
    at = 0
    for e, c in enumerate(counts):
        want = dy[at:at + c].double().t().contiguous() @ x[at:at + c].double()
        assert t.equal(got[e].double(), want.to(got.dtype).double()), e
        at += c


def test_offsets_past_32_bits(ops):   # noqa: F811
    print("[operators8] far offsets", flush=True)
    from paper_2606_07019_amd.operators import F8, f8_bytes
    t = _torch()
    rng = np.random.default_rng(2)
    k = 4096
    cb, sb = f8_bytes(k)

    def far(*lead):   # zeros, but for the last rows
        return F8(t.zeros(*lead, cb, dtype=t.uint8, device="cuda"), t.full((*lead, sb), 127, dtype=t.uint8, device="cuda"), k)

    a, av = _packed(rng, 200, k, 127, 127, WHOLE)
    b, bv = _packed(rng, 50, k, 127, 127, WHOLE)
    want = t.from_numpy(av @ bv.T).cuda()
    n = (1 << 20) + 321                                          # rows of B: 4.3 GB of codes
    w = far(n)
    w.codes[-50:], w.scales[-50:] = b.codes, b.scales
    for m in (3, 200):                                           # few rows; many, 200 x n results of 2 bytes
        got = ops.matmul8(F8(a.codes[:m].contiguous(), a.scales[:m].contiguous(), k), w, t.bfloat16)
        assert t.equal(got[:, -50:].double(), want[:m].bfloat16().double()) and (got[:, :-50] == 0).all()
    got = ops.matmul8(w, F8(b.codes[:9].contiguous(), b.scales[:9].contiguous(), k), t.float32)   # rows of A
    assert t.equal(got[-50:].double(), t.from_numpy(bv @ bv[:9].T).cuda()) and (got[:-50] == 0).all()
    del w, got
    e, each = 257, 4096                                          # experts' weights
    w = far(e, each)
    w.codes[-1, -50:], w.scales[-1, -50:] = b.codes, b.scales
    counts = t.zeros(e, dtype=t.int32, device="cuda")
    counts[-1] = 200
    got = ops.expert_matmul8(a, w, ops.expert_groups(counts, 200), t.bfloat16)
    assert t.equal(got[:, -50:].double(), want.bfloat16().double()) and (got[:, :-50] == 0).all()
    del w, got
    x = t.zeros(66000, 66000, dtype=t.bfloat16, device="cuda")   # 2^32 values and more
    x[-130:, -130:] = _to(rng.normal(size=(130, 130)), "bf16")
    r, c = ops.quantize8_both(x)
    for q, want in ((r, x[-130:]), (c, x.t()[-130:])):
        got = _np(ops.dequantize8(F8(q.codes[-130:].contiguous(), q.scales[-130:].contiguous(), 66000), t.float32))
        assert (got[:, :65536] == 0).all()                       # whole blocks; 464 values are left
        np.testing.assert_array_equal(got[:, 65536:], O.f8_values(*O.f8_quantize(_np(want[:, 65536:])), 464))
    one = ops.quantize8(x)
    assert t.equal(one.codes, r.codes)
    back = ops.dequantize8(r, t.bfloat16)
    assert t.equal(back[-130:, -130:].float(), ops.dequantize8(F8(r.codes[-130:].contiguous(), r.scales[-130:].contiguous(), 66000), t.float32)[:, -130:])


def test_balance_of_many_rows(ops):   # noqa: F811
    print("[operators8] balance, many rows", flush=True)
    t = _torch()
    tokens, experts = 70000000, 64                               # logits past 2^32 bytes
    l = t.zeros(tokens, experts, dtype=t.bfloat16, device="cuda")
    l[-1, 5] = 8.0
    ids = t.zeros(tokens, 1, dtype=t.int32, device="cuda")
    ids[-1] = 5
    loss, counts, probs, rows = ops.balance_loss(l, ids)
    assert int(rows) == tokens and int(counts[0]) == tokens - 1 and int(counts[5]) == 1
    # a lane adds up tokens / 16384 rows, then lanes, waves and workgroups are joined: 2^-24 a step; a probability 2^-20
    assert (probs.double() * experts - 1).abs().max() <= (tokens / 16384 + 600) * 2.0 ** -24 + 2.0 ** -20
    d = ops.balance_loss_backward(l, counts, rows, t.full((), float(tokens), device="cuda"))
    p = t.softmax(l[-1].double(), 0)
    v = counts.double() * experts / tokens
    want = p * (v - (v * p).sum())
    assert (d[-1].double() - want).abs().max() <= 2.0 ** -8 * want.abs().max()
    assert t.equal(d[0], d[tokens // 2]) and d[0].abs().max() > 0
