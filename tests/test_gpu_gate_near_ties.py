"""The gate where its first, quick arithmetic cannot decide: ids as in binary64."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from oracle import gate as ogate

pytestmark = pytest.mark.gpu
WEIGHT = 2.0 ** -19             # of a weight from exact logits: 25 roundings of 2^-24 in the sum of exponentials and the quotient, 2^-22 in its own


@pytest.fixture(scope="module")
def B():
    from paper_2608_15383_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def shape(H, E, k):
    return SimpleNamespace(d_model=H, d_ff=128, num_experts=E, top_k=k)


def tie(z, a, b, gap):
    """Balance biases (binary32) under which expert a's choice value is `gap` above expert b's, all others far below."""
    p = ogate.scores(z, "softmax")
    balance = np.full(len(z), -4.0, dtype=np.float32)
    balance[b] = np.float32(p[a] - p[b])
    balance[a] = np.float32(p[b] + float(balance[b]) - p[a] + gap)       # of the size of a rounding of balance[b]: as fine as the gap
    return balance


@pytest.mark.parametrize("E", [3, 60, 64, 100, 128, 200, 256, 300, 512])
def test_softmax_with_balance_bias_on_given_logits(B, E):
    """Choice values p + balance that differ by 1e-9 to 1e-7, of experts whose probabilities p differ by 0.1 and more: a sum of exponentials in
    binary32 (off by 2^-24 of itself and more) puts them in the wrong order."""
    rng = np.random.default_rng(E)
    for i in range(48):
        z = rng.normal(size=E).astype(np.float32)
        a, b = rng.permutation(E)[:2]
        z[a], z[b] = np.log(E) + 1.5 + 0.3 * rng.normal(), np.log(E) + 0.3 * rng.normal()
        gap = float(rng.choice([-1, 1]) * 10.0 ** rng.uniform(-9, -7))
        balance = tie(z.astype(np.float64), a, b, gap)
        for k, gate in ((1, B.Gate()), (2, B.Gate(renormalise=True))):
            ids, w = B.exmoe_gate_logits(shape(0, E, k), gate, torch.from_numpy(z).cuda()[None], balance=torch.from_numpy(balance).cuda())
            ref, ref_w = ogate.choose(z[None], gate, k, balance)
            assert np.array_equal(ids.cpu().numpy(), ref), (i, k, gap)
            np.testing.assert_allclose(w.cpu().numpy(), ref_w, rtol=WEIGHT)


def test_any_binary32_sum_gets_one_of_these_wrong(B):
    """The exact sum of exponentials lies midway between two binary32 numbers: with the upper one expert 2 would win the first, with the
    lower one expert 0 the second."""
    f = float.fromhex
    z = np.array([0.0, f("-0x1.efc2ecp-1"), -30.0])
    for gap in (1e-8, -1e-8):
        balance = np.array([f("-0x1.e8394ep-30"), -1.0, f("0x1.731604p-1")], dtype=np.float32)
        p = ogate.scores(z, "softmax")
        balance[0] = np.float32(p[2] + float(balance[2]) - p[0] + gap)
        for order in ([0, 1, 2], [2, 1, 0], [1, 2, 0]):
            zo, bo = z[order], balance[order]
            ids, w = B.exmoe_gate_logits(shape(0, 3, 1), B.Gate(), torch.tensor(zo[None], dtype=torch.float32).cuda(), balance=torch.from_numpy(bo).cuda())
            ref, ref_w = ogate.choose(zo[None], B.Gate(), 1, bo)
            assert np.array_equal(ids.cpu().numpy(), ref), (gap, order)
            np.testing.assert_allclose(w.cpu().numpy(), ref_w, rtol=WEIGHT)


@pytest.mark.parametrize("T", [1, 40, 400])
def test_softmax_with_balance_bias_on_hidden_rows_of_small_norm(B, T):
    """Logits whose own bound is far below the rounding of the sum of exponentials."""
    rng = np.random.default_rng(T)
    E, H = 4, 64
    for i in range(24):
        x = torch.zeros(T, H)
        x[:, 0] = 2.0 ** -7 * float(rng.uniform(1, 2))
        w = torch.zeros(E, H)
        w[:, 0] = torch.from_numpy(rng.normal(size=E))
        x, w = x.to(torch.bfloat16), w.to(torch.bfloat16)
        z = ogate.logits(x[:1].double().numpy(), w.double().numpy())[0]
        p = ogate.scores(z, "softmax")
        a, b = rng.permutation(E)[:2]
        gap = float(rng.choice([-1, 1]) * abs(p[a] - p[b]) * 10.0 ** rng.uniform(-8.5, -7))
        balance = tie(z, a, b, gap)
        ids, _ = B.exmoe_route_gated(shape(H, E, 1), B.Gate(), x.cuda(), w.cuda(), balance=torch.from_numpy(balance).cuda())
        ref, _ = ogate.choose_token(z, B.Gate(), 1, balance)
        assert (ids.cpu().numpy() == ref).all(), (i, gap)


@pytest.mark.parametrize("E,T", [(128, 1), (128, 30), (100, 3), (128, 300), (60, 700)])
def test_rows_of_tiny_norm_whose_sums_cancel(B, E, T):
    """Logits that come out as 0 in binary32 and are not: c - c + w_e 2^-100, c = 2^-60.  Only a row of zeros, or a router of zeros, has logits that are 0 by themselves."""
    H, k = 64, min(8, E)
    order = torch.from_numpy(np.random.default_rng(E).permutation(128)[:E])
    w = torch.zeros(E, H)
    w[:, 0] = w[:, 2] = 1.0
    w[:, 1] = 1.0 + order / 128.0
    x = torch.zeros(T, H)
    x[:, 0], x[:, 1], x[:, 2] = 2.0 ** -60, 2.0 ** -100, -2.0 ** -60
    if T > 1:
        x[T // 2] = 0.0
    for kw in (dict(), dict(score="sigmoid", renormalise=True)):
        hidden, router, gate = x.to(torch.bfloat16), w.to(torch.bfloat16), B.Gate(**kw)
        ids, weights = B.exmoe_route_gated(shape(H, E, k), gate, hidden.cuda(), router.cuda())
        ref, ref_w = ogate.choose(ogate.logits(hidden.double().numpy(), router.double().numpy()), gate, k)
        assert np.array_equal(ids.cpu().numpy(), ref)
        np.testing.assert_allclose(weights.cpu().numpy(), ref_w, rtol=WEIGHT)
        ids, _ = B.exmoe_route_gated(shape(H, E, k), gate, hidden.cuda(), torch.zeros_like(router).cuda())
        assert (ids.cpu() == torch.arange(k)).all()


@pytest.mark.parametrize("E,T", [(16, 1), (16, 30), (16, 300), (600, 2)])
@pytest.mark.parametrize("hidden_at,router_at", [(70, 60), (100, 100), (-70, -70), (-80, -60), (-100, -30), (-63, -63), (-120, -120)])
def test_products_beyond_binary32(B, E, T, hidden_at, router_at):
    """Products of BF16 numbers that binary32 holds as an infinity, as a subnormal number, or as zero."""
    H, k = 64, 5
    rng = np.random.default_rng(E + T)
    x = torch.from_numpy(rng.uniform(1, 2, (T, H)) * rng.choice([-1, 1], (T, H)) * 2.0 ** hidden_at).to(torch.bfloat16)
    w = torch.from_numpy(rng.uniform(1, 2, (E, H)) * rng.choice([-1, 1], (E, H)) * 2.0 ** router_at).to(torch.bfloat16)
    x[0, 1::2] = 0.0
    z = ogate.logits(x.double().numpy(), w.double().numpy())
    for kw in (dict(), dict(score="sigmoid", renormalise=True), dict(renormalise=True, num_groups=2)):
        gate = B.Gate(**kw)
        ids, weights = B.exmoe_route_gated(shape(H, E, k), gate, x.cuda(), w.cuda())
        ref, ref_w = ogate.choose(z, gate, k)
        assert np.array_equal(ids.cpu().numpy(), ref)
        np.testing.assert_allclose(weights.cpu().numpy(), ref_w, rtol=WEIGHT, atol=2.0 ** -126)
    mask = torch.zeros(T, E)
    mask[torch.from_numpy(rng.random((T, E)) < 0.3)] = -np.inf
    ids, weights = B.exmoe_route_gated(shape(H, E, k), B.Gate(), x.cuda(), w.cuda(), addend=mask.cuda())
    ref, ref_w = ogate.choose(z + mask.double().numpy(), B.Gate(), k)
    assert np.array_equal(ids.cpu().numpy(), ref)
    np.testing.assert_allclose(weights.cpu().numpy(), ref_w, rtol=WEIGHT, atol=2.0 ** -126)


@pytest.mark.parametrize("E,T", [(64, 5), (64, 40), (256, 300)])
def test_rows_of_zeros_with_bias_or_addend(B, E, T):
    """A padded row's logits are its bias or its addend, or the sum of both in 64 bits: ties and neighbours of one binary32 step."""
    H, k = 256, 8
    g = torch.Generator().manual_seed(E + T)
    x, w = torch.randn(T, H, generator=g).to(torch.bfloat16), (torch.randn(E, H, generator=g) * 0.02).to(torch.bfloat16)
    x[1::2] = 0.0
    one = torch.full((E,), 1.0)
    one[::3] += 2.0 ** -23
    for bias, addend in ((one, None), (None, torch.zeros(T, E)), (None, one.flip(0).repeat(T, 1)), (one, torch.zeros(T, E)), (one * 2.0 ** -30, one.repeat(T, 1))):
        for gate in (B.Gate(), B.Gate(score="sigmoid", num_groups=4, top_groups=2, group_score="top2", renormalise=True)):
            cuda = lambda v: None if v is None else v.cuda()
            ids, _ = B.exmoe_route_gated(shape(H, E, k), gate, x.cuda(), w.cuda(), bias=cuda(bias), addend=cuda(addend))
            z = ogate.logits(x.double().numpy(), w.double().numpy(), None if bias is None else bias.double().numpy(), None if addend is None else addend.double().numpy())
            assert np.array_equal(ids.cpu().numpy(), ogate.choose(z, gate, k)[0])
