"""The All-to-Allv builder (CPU), and the example that joins the operators with the synthesizer (GPU)."""

import importlib.util
import os

import numpy as np
import pytest

from oracle import oracle as O
from paper_2606_07019_amd import workloads as W

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_all_to_all_v_of_one_chunk_each_is_all_to_all():
    ones = W.all_to_all_v(9, [0, 2, 6, 8], np.ones((4, 4), int), 1000)
    same = W.all_to_all(9, [0, 2, 6, 8], 1000)
    for field in ("pre", "post", "group_masks"):
        np.testing.assert_array_equal(getattr(ones, field), getattr(same, field))
    assert (ones.n_chunks, ones.chunk_bytes, ones.op) == (16, 1000, W.OP_COPY)


def test_all_to_all_v_carries_every_chunk():
    counts = np.array([[3, 0, 70], [1, 0, 2], [0, 5, 1]])
    coll = W.all_to_all_v(4, [3, 0, 1], counts, 64)
    assert coll.n_chunks == counts.sum()
    c = 0
    for i, v in enumerate([3, 0, 1]):
        for j, u in enumerate([3, 0, 1]):
            for _ in range(counts[i, j]):
                assert [W.get_bit(coll.pre, d, c) for d in range(4)] == [d == v for d in range(4)]
                assert [W.get_bit(coll.post, d, c) for d in range(4)] == [d == u for d in range(4)]
                c += 1
    r = O.run_workload(W.Workload("counts", W.ring(4), coll))
    assert r.status == 0
    # on a ring of four each chunk crosses one link or two
    hops = sum(counts[i, j] * min((u - v) % 4, (v - u) % 4) for i, v in enumerate([3, 0, 1]) for j, u in enumerate([3, 0, 1]))
    assert len(r.sends) == hops


@pytest.mark.gpu
def test_example():
    spec = importlib.util.spec_from_file_location("expert_parallel", os.path.join(ROOT, "examples", "expert_parallel.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    print("[operators] example", flush=True)
    r = example.run()
    assert r["counts"].sum() == 4 * 48 * 2
    ref = O.run_workload(r["workload"])
    assert ref.status == 0 and ref.collective_time == r["ns"]
    np.testing.assert_array_equal(r["sends"], ref.sends)
    assert r["row_bytes"] == 256 + 16 and r["ns"] < r["ns16"]
    # a value is off by a quarter at most (8 - 2^-k becomes 6), twice: tokens and inner values; the latter's factors
    # add theirs.  Errors of both signs leave far less than that of a sum.
    assert r["off"] < 0.5
    for g in r["gradients"]:                     # a softmax moves no sum of its logits
        assert g.abs().max() > 0 and g.sum(dim=1).abs().max() <= 2.0 ** -19 * 16 * g.abs().max()
