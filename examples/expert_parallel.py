#!/usr/bin/env python3
"""Expert-parallel dispatch from one end to the other, on one GPU.

Every NPU of a process group has tokens and a share of the experts.

  route      each NPU's router picks experts for its tokens (and its gradient
             comes back through the same picks);
  quantize   the tokens are packed to microscaled 4-bit values, the payload;
  synthesize the picks' counts say how many rows go from each NPU to each
             other one: an All-to-Allv of that many chunks, for which the
             synthesizer finds the schedule (and, for comparison, the one of
             the payload in 16 bits);
  matmul     each expert multiplies the packed rows that reached it with its
             packed weights, and the results are weighted and summed up where
             their tokens came from;
  moe_layer  for few tokens no dispatch pays: one NPU that holds all experts
             runs the layer at once.  Here it is also the result to compare with.

    python examples/expert_parallel.py
"""

import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import numpy as np
import torch

from paper_2606_07019_amd import workloads as W
from paper_2606_07019_amd.operators import MX, Operators, mx_bytes
from paper_2606_07019_amd.pccl import Synthesizer


def dispatch(counts, topo, members, chunk_bytes, name, device=0):
    """(workload, schedule, collective time in ns) of counts[i][j] chunks from member i to member j."""
    wl = W.Workload(name, topo, W.all_to_all_v(topo.n_npus, members, counts, chunk_bytes))
    s = Synthesizer(wl.topo, wl.coll, tie_seed=wl.tie_seed, device=device)
    try:
        _, ns = s.synthesize()
        return wl, s.schedule(), ns
    finally:
        s.close()


def expert(ops, rows, up, down, e):
    """Expert e's results, in 32 bits, for packed rows."""
    both = ops.matmul(rows, MX(up.codes[e], up.scales[e], up.cols), torch.float32)
    gate, lift = both.chunk(2, dim=1)
    inner = ops.quantize(torch.nn.functional.silu(gate) * lift)
    return ops.matmul(inner, MX(down.codes[e], down.scales[e], down.cols), torch.float32)


def run(tokens=48, hidden=512, inter=256, experts=16, topk=2, seed=0, device=0):
    topo = W.mesh2d(3, 3)
    members = [0, 2, 6, 8]                       # the mesh's corners: their traffic is relayed by NPUs outside the group
    n, per = len(members), experts // len(members)
    ops = Operators(device)
    g = torch.Generator(device=ops.device).manual_seed(seed)

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g, device=ops.device) * scale).to(torch.bfloat16)

    def packed(*shape, scale):
        w = normal(*shape, scale=scale)
        q = ops.quantize(w.view(-1, shape[2]))
        return MX(q.codes.view(*shape[:2], -1), q.scales.view(*shape[:2], -1), shape[2])

    xs = [normal(tokens, hidden) for _ in members]
    router = normal(experts, hidden, scale=hidden ** -0.5)
    up, down = packed(experts, 2 * inter, hidden, scale=hidden ** -0.5), packed(experts, hidden, inter, scale=inter ** -0.5)

    # where each NPU's rows go
    logits = [x.float() @ router.float().t() for x in xs]
    picks = [ops.route(l, topk) for l in logits]
    counts = torch.stack([p[2] for p in picks]).view(n, n, per).sum(dim=2).cpu().numpy()

    # what carries them, with rows of 4-bit values and of 16-bit ones
    row_bytes = sum(mx_bytes(hidden))
    wl, sends, ns = dispatch(counts, topo, members, row_bytes, "rows of 4-bit values", device)
    _, _, ns16 = dispatch(counts, topo, members, 2 * hidden, "rows of 16-bit values", device)

    # the rows that reach each expert, in the order of their senders, and their way back
    payload = [ops.quantize(x) for x in xs]
    ys = [torch.zeros(tokens, hidden, device=ops.device) for _ in members]
    starts = [torch.cat((p[2].new_zeros(1), p[2].cumsum(0))).tolist() for p in picks]
    grads = [torch.zeros_like(p[0]) for p in picks]
    for e in range(experts):
        slots = [p[3][s[e]:s[e + 1]].long() for p, s in zip(picks, starts)]
        rows = MX(torch.cat([q.codes[s // topk] for q, s in zip(payload, slots)]),
                  torch.cat([q.scales[s // topk] for q, s in zip(payload, slots)]), hidden)
        outs = expert(ops, rows, up, down, e).split([s.numel() for s in slots])
        for y, p, grad, s, o in zip(ys, picks, grads, slots, outs):
            y.index_add_(0, s // topk, o * p[0].view(-1)[s, None])
            grad.view(-1)[s] = o.sum(dim=1)      # of the sum of all results, with respect to the weights
    back = [ops.route_backward(l, p[0], p[1], d) for l, p, d in zip(logits, picks, grads)]

    whole = [ops.moe_layer(x, router, up, down, topk).float() for x in xs]
    off = torch.cat(ys) - torch.cat(whole)
    found = {"counts": counts, "workload": wl, "sends": sends, "ns": ns, "ns16": ns16, "row_bytes": row_bytes,
             "off": float(off.norm() / torch.cat(whole).norm()), "gradients": back, "results": ys}
    ops.close()
    return found


def main():
    r = run(hidden=4096, inter=1024)
    print(f"rows from each NPU of the group to each other one:\n{r['counts']}")
    print(f"All-to-Allv of {int(r['counts'].sum() - np.trace(r['counts']))} rows of {r['row_bytes']} bytes: {len(r['sends'])} transfers, "
          f"{r['ns'] / 1e3:.1f} us; with 16-bit rows {r['ns16'] / 1e3:.1f} us")
    print(f"dispatched layer against the whole one (4-bit tokens and inner values against 16-bit ones): {r['off']:.3f} of its norm")
    print(f"router gradients: {len(r['gradients'])} x {tuple(r['gradients'][0].shape)}")


if __name__ == "__main__":
    main()
