"""The counts of the balance loss are made in shared memory that the CTA clears first: no warp counts before all of it is clear."""
import os
import re
from types import SimpleNamespace

import pytest
import torch

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_15383_b200", "csrc")


def test_a_barrier_stands_between_clearing_and_counting():
    """On every way, with sequences and without: a barrier that no branch goes around, behind the last clearing and in front of the first count."""
    with open(os.path.join(CSRC, "gate_loss.cu")) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    body = text[text.index("\nbalance_kernel("):]
    body = body[body.index("{"):body.index("\n}\n")]
    cleared, counted = body.index("n_kept = 0;"), body.index("atomicAdd(")
    assert body.index("hist[e] = 0;") < cleared < counted
    depth, found = 0, False
    for line in body[:counted].splitlines():
        found |= line.strip() == "__syncthreads();" and depth == 1
        if "n_kept = 0;" in line:
            found = False
        depth += line.count("{") - line.count("}")
    assert found


@pytest.mark.gpu
@pytest.mark.parametrize("T,E,k", [(1, 64, 8), (16, 64, 8), (300, 60, 4), (5000, 128, 8), (90, 300, 10), (40, 1000, 700), (12, 3000, 600), (3000, 4096, 3)])
def test_one_sequence_counts_every_choice(T, E, k):
    """Call after call, with and without offsets, behind calls that leave other counts in shared memory."""
    from paper_2608_15383_b200 import binding as B
    g = torch.Generator().manual_seed(T)
    s, gate = SimpleNamespace(d_model=128, num_experts=E, top_k=k), SimpleNamespace(score="softmax", num_groups=1, top_groups=1, group_score="max", renormalise=False, scale=1.0)
    z, ids = torch.randn(T, E, generator=g).cuda(), torch.rand(T, E, generator=g).argsort(1)[:, :k].int().cuda()
    want = torch.bincount(ids.flatten().long(), minlength=E).int()[None]
    offsets = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    other = (ids + 1) % E
    for off in (None, offsets):
        got = []
        for _ in range(20):
            got.append(B.exmoe_balance_loss(s, gate, z, ids, offsets=off))
            B.exmoe_balance_loss(s, gate, z, other, offsets=off)
        torch.cuda.synchronize()
        for losses, counts, sums, kept in got:
            assert torch.equal(counts, want) and kept.tolist() == [T] and torch.equal(sums, got[0][2]) and torch.equal(losses, got[0][0])
