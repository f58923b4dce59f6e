"""Logits far from zero: scores, losses and gradients do not see a number that all of a row's logits have in common.

Bounds.  With d = z - largest, rounded by |d| 2^-24 at most and exact next to the largest, an exponential's argument is off by |d| 2^-23 (this rounding and the product's) and the
exponential by 2 units of 2^-23 besides.  Scores that matter are within 20 of the largest here: 44 2^-23 with a few more for sums of up to 64 terms in pairs, the
reciprocal and the products; REL = 96 2^-23 holds them all, whatever the largest logit is.  A logarithm of a sum is off by REL and by its largest term's last place.
"""
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from oracle import gate_loss as oloss

pytestmark = pytest.mark.gpu
REL = 96 * 2.0 ** -23
FARS = [s * v for v in (100.0, 1e4, 1e5, 1e6, 1e9, 1e10, 1e20, 1e30, 3e37, 2e38) for s in (1, -1)]
FORMS = [("softmax", False), ("softmax", True), ("sigmoid", False), ("sigmoid", True)]


@pytest.fixture(scope="module")
def B():
    from paper_2608_15383_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def gate(score="softmax", renormalise=False):
    return SimpleNamespace(score=score, num_groups=1, top_groups=1, group_score="max", renormalise=renormalise, scale=1.5)


def num(t):
    return None if t is None else t.double().cpu().numpy()


def inputs(T, E, k, seed, far, dtype):
    """Rows near `far`; every fourth one near zero."""
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(T, E, generator=g, dtype=torch.float64)
    z[torch.arange(T) % 4 != 3] += far
    # (what the logits' type keeps of the differences is what the oracle sees too)
    ids = torch.rand(T, E, generator=g).argsort(1)[:, :k].int()
    return z.to(dtype).cuda(), ids.cuda(), g


def check_balance(B, s, g, z, ids):
    losses, counts, sums, kept = B.exmoe_balance_loss(s, g, z, ids)
    want, c, p, n = oloss.balance(num(z), ids.cpu().numpy(), g)
    T = z.shape[0]
    assert np.array_equal(counts.cpu().numpy(), c) and np.array_equal(kept.cpu().numpy(), n)
    rel = REL + (T + 64) * 2.0 ** -24
    assert (np.abs(num(sums) - p) <= rel * p + T * 2.0 ** -126).all(), np.abs(num(sums) / np.maximum(p, 1e-30) - 1).max()
    assert abs(num(losses)[0] - want[0]) <= 2 * rel * want[0]
    lse = np.abs([oloss.log_sum(r) for r in num(z)]).max()
    if lse < 1e18:                                                         # (its square leaves binary32 beyond)
        d = 3 * REL + 2.0 ** -22 * 2 * lse
        assert abs(num(losses)[1] - want[1]) <= d * (2 * lse + d) + rel * want[1]
    else:
        assert float(losses[1]) == float("inf")
    return counts, kept


@pytest.mark.parametrize("far", FARS)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_balance(B, far, score, dtype):
    for T, E, k in ((30, 8, 2), (24, 60, 4), (16, 256, 8), (9, 700, 3), (7, 2000, 5), (2500, 64, 4)):
        z, ids, _ = inputs(T, E, k, T, far, dtype)
        check_balance(B, SimpleNamespace(d_model=128, num_experts=E, top_k=k), gate(score), z, ids)


@pytest.mark.parametrize("far", FARS)
@pytest.mark.parametrize("score,renormalise", FORMS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_backward(B, far, score, renormalise, dtype):
    for T, E, k in ((30, 8, 2), (24, 60, 4), (16, 256, 8), (9, 700, 3), (7, 2000, 5), (12, 40, 20)):
        s, g = SimpleNamespace(d_model=128, num_experts=E, top_k=k), gate(score, renormalise)
        z, ids, rng = inputs(T, E, k, T + 1, far, dtype)
        dw = torch.randn(T, k, generator=rng).cuda()
        _, counts, _, kept = B.exmoe_balance_loss(s, g, z, ids)
        for w, l in ((dw, [0.5, 0.25]), (dw, None), (None, [0.5, 0.0]), (None, [0.5, 0.25])):
            dl = None if l is None else torch.tensor(l, device="cuda")
            got = num(B.exmoe_gate_backward(s, g, z, ids, w, dl, counts, kept))
            want, size = oloss.backward(num(z), ids.cpu().numpy(), g, k, num(w), num(dl), counts.cpu().numpy(), kept.cpu().numpy())
            tol = 4 * REL * size + 1e-35
            tol = tol + torch.finfo(dtype).eps / 2 * (np.abs(want) + tol)
            assert (np.abs(got - want) <= tol).all(), (T, E, l, w is None, (np.abs(got - want) - tol).max())


@pytest.mark.parametrize("mask_value", [-1e9, -1e10, -1e30])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_rows_masked_by_a_finite_value(B, mask_value, score):
    """Experts switched off by a finite constant; a row all of them are off in is an even one and spoils no other."""
    T, E, k = 40, 64, 4
    s, g = SimpleNamespace(d_model=128, num_experts=E, top_k=k), gate(score)
    z, ids, rng = inputs(T, E, k, 5, 0.0, torch.float32)
    z[:, ::3] = mask_value
    z[7] = mask_value
    counts, kept = check_balance(B, s, g, z, ids)
    losses, _, sums, _ = B.exmoe_balance_loss(s, g, z, ids)
    assert torch.isfinite(losses[0]) and torch.isfinite(sums).all()
    one = B.exmoe_balance_loss(s, g, z[7:8], ids[7:8])[2]
    assert torch.allclose(one, torch.full_like(one, 1 / E), rtol=1e-5, atol=0)
    got = B.exmoe_gate_backward(s, g, z, ids, torch.randn(T, k, generator=rng).cuda(), torch.tensor([1.0, 0.001], device="cuda"), counts, kept)
    assert torch.isfinite(got).all()


@pytest.mark.parametrize("far", [0.0, 300.0, -3e4, 1e6, -1e9])
def test_gradients_of_shares_sum_to_nothing(B, far):
    """Softmax weights do not change with what all logits have in common: a row of their gradient sums to 0, up to its terms' roundings."""
    T, E, k = 64, 64, 8
    s, g = SimpleNamespace(d_model=128, num_experts=E, top_k=k), gate()
    z, ids, rng = inputs(T, E, k, 6, far, torch.float32)
    dw = torch.randn(T, k, generator=rng).cuda()
    got = B.exmoe_gate_backward(s, g, z, ids, d_weights=dw).double()
    _, size = oloss.backward(num(z), ids.cpu().numpy(), g, k, num(dw))
    assert (got.sum(1).abs().cpu().numpy() <= 4 * REL * size.sum(1)).all()
