"""GPU: rows beyond what one launch holds go to a further one; what is found on
either side of the seam is what a call on those rows alone gives."""

import pytest

from test_gpu_operators import _torch, ops  # noqa: F401

pytestmark = pytest.mark.gpu

PER = 0xFFFFFFFF // 256     # workgroups of a launch


def test_packing_and_unpacking_over_two_launches(ops):   # noqa: F811
    print("[operators] packing of 2^29 rows of 8", flush=True)
    from paper_2606_07019_amd.operators import MX
    t = _torch()
    rows = PER * 32 + 4000
    x = t.empty((rows, 8), dtype=t.bfloat16, device="cuda").normal_()
    q = ops.quantize(x)
    whole = ops.dequantize(q, t.bfloat16)
    for seam in (PER * 32, PER * 4, rows):                       # of the packing, of the unpacking, the end
        r = slice(seam - 3000, min(rows, seam + 3000))
        want = ops.quantize(x[r])
        assert t.equal(q.codes[r], want.codes) and t.equal(q.scales[r], want.scales)
        assert t.equal(whole[r], ops.dequantize(MX(want.codes, want.scales, 8), t.bfloat16))
    del x, q, whole
    t.cuda.empty_cache()


def test_router_gradient_over_two_launches(ops):   # noqa: F811
    print("[operators] gradient of 2^26 rows of 257", flush=True)
    t = _torch()
    tokens, experts = PER * 4 + 4000, 257
    logits = t.empty((tokens, experts), dtype=t.bfloat16, device="cuda").normal_()
    ids = t.randint(0, experts - 1, (tokens, 2), dtype=t.int32, device="cuda")
    ids[:, 1] = (ids[:, 0] + 1)
    weights, g = t.rand((tokens, 2), device="cuda"), t.randn((tokens, 2), device="cuda")
    mask = t.rand(tokens, device="cuda") < 0.9
    for normalize in (True, False):
        d = ops.route_backward(logits, weights, ids, g, normalize=normalize, mask=mask)
        for seam in (PER * 4, tokens):
            r = slice(seam - 3000, min(tokens, seam + 3000))
            want = ops.route_backward(logits[r], weights[r], ids[r], g[r], normalize=normalize, mask=mask[r])
            assert t.equal(d[r], want) and (want != 0).any()
        del d
    del logits, ids, weights, g, mask
    t.cuda.empty_cache()
