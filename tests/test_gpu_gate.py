"""The gate on the device against its binary64 oracle: the same experts, always, and weights to binary32 rounding.

Weights: a logit is a sum of H exact products in binary32, in chains of at most H / 64 + 32 additions, each off by 2^-24 of what is
summed at most (2^-23 where the tensor cores truncate), so |dz| <= (H / 64 + 32) 2^-23 S with S = sum |x_i w_i|; a score's relative
error is below 2 |dz| + 8 roundings of 2^-24, a renormalised one's twice that.
"""
import math
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from oracle import gate as ogate
from paper_2608_15383_b200 import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2608_15383_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def shape(H, E, k):
    return SimpleNamespace(d_model=H, d_ff=128, num_experts=E, top_k=k)


def check_weights(w, ref, dz, what=""):
    tol = 2 * (2 * dz + 8 * 2.0 ** -24)
    assert (np.isnan(w) == np.isnan(ref)).all(), what
    ok = ~np.isnan(ref)
    assert (np.abs(w - ref)[ok] <= (tol * np.abs(ref) + 1e-37)[ok]).all(), (what, np.abs(w - ref)[ok].max())


def check_gated(B, s, gate, hidden, w, bias=None, addend=None, balance=None, **k):
    cuda = lambda v: None if v is None else v.cuda()
    ids, weights = B.exmoe_route_gated(s, gate, hidden.cuda(), w.cuda(), bias=cuda(bias), addend=cuda(addend), balance=cuda(balance), **k)
    torch.cuda.synchronize()
    num = lambda v: None if v is None else v.double().numpy()
    z = ogate.logits(num(hidden), num(w), num(bias), num(addend))
    ref_ids, ref_w = ogate.choose(z, gate, s.top_k, num(balance))
    assert ids.dtype == torch.int32 and weights.dtype == torch.float32
    assert np.array_equal(ids.cpu().numpy(), ref_ids), np.flatnonzero((ids.cpu().numpy() != ref_ids).any(1))[:10]
    S = (np.abs(num(hidden)) @ np.abs(num(w)).T).max()
    zs = np.abs(z[np.isfinite(z)]).max() if np.isfinite(z).any() else 0.0
    check_weights(weights.cpu().numpy().astype(np.float64), ref_w, (s.d_model / 64 + 32) * 2.0 ** -23 * S + 3 * 2.0 ** -24 * zs)
    return ids, weights


GATES = [dict(), dict(renormalise=True, scale=2.5), dict(score="sigmoid", renormalise=True),
         dict(score="sigmoid", num_groups=4, top_groups=2, group_score="top2", renormalise=True, scale=2.5),
         dict(num_groups=4, top_groups=3), dict(num_groups=4, top_groups=1, group_score="top2"), dict(score="sigmoid", num_groups=2, top_groups=2)]


@pytest.mark.parametrize("g", range(len(GATES)))
@pytest.mark.parametrize("H,E,k,T", [(256, 8, 2, 16), (2048, 64, 8, 1), (2048, 64, 8, 5), (2048, 60, 4, 24), (512, 16, 4, 333), (1000, 20, 3, 70),
                                     (2048, 64, 8, 400), (1024, 256, 8, 130), (768, 128, 6, 1500), (128, 4, 1, 3), (2048, 256, 8, 700), (64, 12, 2, 260)])
@pytest.mark.parametrize("balanced", [False, True])
def test_gate_matches_oracle(B, g, H, E, k, T, balanced):
    gate = B.Gate(**GATES[g])
    if k > gate.top_groups * (E // gate.num_groups):
        pytest.skip("fewer experts kept than chosen")
    s = shape(H, E, k)
    hidden, w = synth.hidden_states(s, T, 11 + T), synth.router_weights(s, 5)
    balance = torch.randn(E, generator=torch.Generator().manual_seed(1)) * 0.1 if balanced else None
    check_gated(B, s, gate, hidden, w, balance=balance)


@pytest.mark.parametrize("H,E,k,T", [(2048, 64, 8, 40), (2048, 64, 8, 300), (512, 128, 8, 600), (1024, 256, 8, 260), (256, 36, 5, 100), (2048, 256, 8, 30)])
@pytest.mark.parametrize("g", [1, 2, 3, 4, 5])
def test_near_ties_are_decided_as_in_64_bits(B, g, H, E, k, T):
    """Rows of the router's matrix that equal another, or differ from it in one element by one BF16 ulp; equal and nearly equal balance biases."""
    gate = B.Gate(**GATES[g])
    s = shape(H, E, k)
    hidden, w = synth.hidden_states(s, T, 3), synth.router_weights(s, 4)
    for e in range(1, E, 3):
        w[e] = w[e - 1]
        if e % 2:
            w[e, (7 * e) % H] = torch.nextafter(w[e, (7 * e) % H].float(), torch.tensor(9.0)).to(torch.bfloat16) * (1 + 2.0 ** -7)
    for e in range(0, E - E // 4, E // 4):                                 # and whole groups alike
        if e % (E // 2) == 0:
            w[e + E // 4:e + E // 2] = w[e:e + E // 4]
    check_gated(B, s, gate, hidden, w)
    balance = torch.zeros(E)
    balance[::5] = 2.0 ** -26
    check_gated(B, s, gate, hidden, w, balance=balance)


def test_logits_bias_addend_masks_and_nan(B):
    s = shape(512, 24, 4)
    for T in (7, 280, 300):                                                # the last on the tensor cores
        hidden, w = synth.hidden_states(s, T, 8), synth.router_weights(s, 9)
        g = torch.Generator().manual_seed(T)
        bias, addend = torch.randn(24, generator=g), torch.randn(T, 24, generator=g)
        addend[torch.rand(T, 24, generator=g) < 0.3] = -math.inf
        addend[1] = -math.inf                                              # nothing left
        addend[2, 1:] = -math.inf                                          # one expert left
        addend[3, ::2] = torch.finfo(torch.float32).min                    # a mask of the type's lowest value is a number
        addend[4, 5] = math.nan
        addend[5, 6] = math.inf
        for kw in GATES:
            gate = B.Gate(**kw)
            for balance in (None, torch.randn(24, generator=g) * 0.1):
                ids, weights = check_gated(B, s, gate, hidden, w, bias=bias, addend=addend, balance=balance)
                assert weights[1].tolist() == [0.0] * 4 and ids[1].tolist() == [0, 1, 2, 3]


@pytest.mark.parametrize("E,k,G,keep", [(1, 1, 1, 1), (3, 3, 3, 3), (32, 8, 32, 8), (60, 4, 4, 2), (64, 8, 1, 1), (257, 9, 1, 1), (256, 8, 8, 4), (1000, 33, 4, 3),
                                        (4096, 16, 32, 5), (512, 512, 1, 1)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gate_from_logits(B, E, k, G, keep, dtype):
    s = shape(0, E, k)
    for T, score, how, balanced in ((1, "softmax", "max", False), (37, "sigmoid", "top2", True), (130, "softmax", "top2", False), (64, "softmax", "max", True),
                                    (129, "sigmoid", "max", False)):
        g = torch.Generator().manual_seed(E + T)
        wide = torch.randn(T, E + 3, generator=g).to(dtype)
        z = wide[:, 1:E + 1] if T % 2 else wide[:, :E].contiguous()
        z[torch.rand(T, E, generator=g) < 0.05] = -math.inf
        z[0] = -math.inf
        balance = torch.randn(E, generator=g) * 0.1 if balanced else None
        gate = B.Gate(score=score, num_groups=G, top_groups=keep, group_score=how, renormalise=T % 3 != 1, scale=1.5)
        on_gpu = wide.cuda()
        ids, w = B.exmoe_gate_logits(s, gate, on_gpu[:, 1:E + 1] if T % 2 else z.cuda(), balance=None if balance is None else balance.cuda())
        ref_ids, ref_w = ogate.choose(z.double().numpy(), gate, k, None if balance is None else balance.double().numpy())
        assert np.array_equal(ids.cpu().numpy(), ref_ids), (T, score)
        check_weights(w.cpu().numpy().astype(np.float64), ref_w, 0.0, (T, score))


def test_saturated_scores_keep_their_order(B):
    """Sigmoids that are 1 in binary32, and softmax probabilities that are 0, are ordered by their logits."""
    z = torch.tensor([[40.0, 41.0, 60.0, 50.0, 20.0, 18.0], [-200.0, -150.0, -300.0, 5.0, -201.0, -199.0], [-95.0, -96.0, -99.0, -94.0, -97.0, -98.0]])
    s = shape(0, 6, 5)
    for kw in (dict(score="sigmoid"), dict(), dict(renormalise=True), dict(score="sigmoid", renormalise=True)):
        gate = B.Gate(**kw)
        ids, w = B.exmoe_gate_logits(s, gate, z.cuda())
        ref_ids, ref_w = ogate.choose(z.double().numpy(), gate, 5)
        assert np.array_equal(ids.cpu().numpy(), ref_ids)
        np.testing.assert_allclose(w.cpu().numpy(), ref_w, rtol=64 * 2.0 ** -24, atol=2e-38)


@pytest.mark.parametrize("H,E,k", [(2048, 64, 8), (1024, 256, 8), (1000, 20, 3)])
def test_choice_does_not_depend_on_the_batch_size(B, H, E, k):
    s = shape(H, E, k)
    gate = B.Gate(score="sigmoid", num_groups=4, top_groups=2, group_score="top2", renormalise=True)
    hidden, w = synth.hidden_states(s, 1300, 21).cuda(), synth.router_weights(s, 22).cuda()
    balance = torch.randn(E, generator=torch.Generator().manual_seed(2)).cuda() * 0.05
    ids, weights = B.exmoe_route_gated(s, gate, hidden, w, balance=balance)
    for T in (1, 2, 16, 47, 48, 190, 200, 513, 1299):
        i, p = B.exmoe_route_gated(s, gate, hidden[:T], w, balance=balance)
        assert torch.equal(i, ids[:T]), T
        torch.testing.assert_close(p, weights[:T], rtol=2e-5, atol=0)
    again, p = B.exmoe_route_gated(s, gate, hidden, w, balance=balance)
    assert torch.equal(again, ids) and torch.equal(p, weights)             # and the same bits every time


def test_large_strides_and_last_rows_only(B):
    """Rows 2^31 bytes and more apart, and outputs that end where they should."""
    E, T = 64, 5
    big = torch.empty(T * (1 << 29), dtype=torch.bfloat16, device="cuda")
    z = big.as_strided((T, E), (1 << 29, 1))
    z.copy_(torch.randn(T, E, generator=torch.Generator().manual_seed(5)))
    s, gate = shape(0, E, 8), B.Gate(renormalise=True)
    out_i, out_w = torch.full((T + 2, 8), -7, dtype=torch.int32, device="cuda"), torch.full((T + 2, 8), 7.0, device="cuda")
    B.exmoe_gate_logits(s, gate, z, topk_ids=out_i[1:T + 1], topk_weights=out_w[1:T + 1])
    ref, _ = ogate.choose(z.double().cpu().numpy(), gate, 8)
    assert np.array_equal(out_i[1:T + 1].cpu().numpy(), ref)
    assert (out_i[[0, T + 1]] == -7).all() and (out_w[[0, T + 1]] == 7.0).all()


@pytest.mark.parametrize("T", [1, 40, 300])
def test_streams_and_graphs(B, T):
    s, gate = shape(2048, 64, 8), B.Gate(score="sigmoid", renormalise=True)
    w = synth.router_weights(s, 1).cuda()
    batches = [synth.hidden_states(s, T, 30 + i).cuda() for i in range(3)]
    want = [B.exmoe_route_gated(s, gate, h, w) for h in batches]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [B.exmoe_route_gated(s, gate, h, w, stream=side) for h in batches]
    side.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    hidden, graph = batches[0].clone(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ids, weights = B.exmoe_route_gated(s, gate, hidden, w)
        again, _ = B.exmoe_gate_logits(shape(0, 8, 2), gate, weights)
    for i in (1, 2, 0):
        hidden.copy_(batches[i])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(ids, want[i][0]) and torch.equal(weights, want[i][1])


@pytest.mark.parametrize("H,E,k,T", [(128, 16, 4, 20000), (64, 256, 8, 19100), (72, 100, 7, 1000), (64, 512, 32, 300), (64, 513, 5, 60), (64, 300, 33, 40), (8, 40, 2, 500),
                                     (4096, 256, 32, 200), (2048, 512, 8, 30), (104, 65, 1, 290)])
def test_sizes_at_the_edges_of_the_kernels(B, H, E, k, T):
    """Beyond 148 tiles of 128 tokens, K not a multiple of the stages' 64, the largest numbers of experts and choices of each kernel, one more than these."""
    s = shape(H, E, k)
    hidden, w = synth.hidden_states(s, T, 6), synth.router_weights(s, 7)
    check_gated(B, s, B.Gate(renormalise=True), hidden, w)
    check_gated(B, s, B.Gate(score="sigmoid"), hidden, w, balance=torch.randn(E, generator=torch.Generator().manual_seed(3)) * 0.02)


@pytest.mark.parametrize("T", [3, 40, 300])
@pytest.mark.parametrize("E", [40, 256])
def test_every_token_is_a_tie(B, E, T):
    """Equal rows of the router's matrix, rows of zeros, and rows so small that their squares are lost: ties by the lower id, near-ties in 64 bits."""
    s = shape(128, E, 8)
    hidden, w = synth.hidden_states(s, T, 1), synth.router_weights(s, 2)
    for kw in (dict(), dict(score="sigmoid", num_groups=4, top_groups=2, group_score="top2", renormalise=True)):
        gate = B.Gate(**kw)
        for balance in (None, torch.zeros(E)):
            same = w[:1].repeat(E, 1)
            ids, _ = check_gated(B, s, gate, hidden, same, balance=balance)
            assert (ids.cpu() == torch.arange(8)).all()
            zeros = hidden.clone()
            zeros[::2] = 0
            check_gated(B, s, gate, zeros, w, balance=balance)
            check_gated(B, s, gate, hidden, torch.zeros_like(w), balance=balance)
    tiny = (hidden.float() * 2.0 ** -66).to(torch.bfloat16)
    close = w.clone()
    close[1::2] = close[::2]
    close[1::2, 5] = (close[::2, 5].float() * (1 + 2.0 ** -7)).to(torch.bfloat16)
    check_gated(B, s, B.Gate(), tiny, close)


def test_calls_at_once_on_several_streams(B):
    s, gate = shape(512, 64, 8), B.Gate(score="sigmoid", num_groups=4, top_groups=2, renormalise=True)
    w = synth.router_weights(s, 1).cuda()
    batches = [synth.hidden_states(s, T, 60 + T).cuda() for T in (1, 30, 300, 700)]
    want = [B.exmoe_route_gated(s, gate, h, w) for h in batches]
    streams = [torch.cuda.Stream() for _ in batches]
    for st in streams:
        st.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        got = [B.exmoe_route_gated(s, gate, h, w, stream=st) for h, st in zip(batches, streams)]
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert B.exmoe_gate_status() == B.EXMOE_OK


def test_empty_calls_and_refusals(B):
    s, gate = shape(256, 8, 2), B.Gate()
    w = torch.zeros((8, 256), dtype=torch.bfloat16, device="cuda")
    h = torch.zeros((3, 256), dtype=torch.bfloat16, device="cuda")
    ids, p = B.exmoe_route_gated(s, gate, h[:0], w)
    assert ids.shape == (0, 2) and p.shape == (0, 2)
    assert B.exmoe_gate_logits(s, gate, torch.zeros((0, 8), device="cuda"))[0].shape == (0, 2)
    f = torch.zeros
    for bad in (dict(w_router=w[:7]), dict(hidden=h[:, :128].contiguous()), dict(bias=f(7, device="cuda")), dict(addend=f((2, 8), device="cuda")),
                dict(balance=f(8)), dict(topk_ids=f((3, 3), dtype=torch.int32, device="cuda")), dict(topk_weights=f((3, 2), dtype=torch.float64, device="cuda"))):
        with pytest.raises(ValueError):
            B.exmoe_route_gated(**{**dict(shape=s, gate=gate, hidden=h, w_router=w), **bad})
    with pytest.raises(ValueError, match="logits"):
        B.exmoe_gate_logits(s, gate, f((8, 8), device="cuda").t()[:, ::2])
    with pytest.raises(B.ExmoeError) as ei:
        B.exmoe_gate_logits(s, B.Gate(num_groups=3), f((2, 8), device="cuda"))
    assert ei.value.code == B.EXMOE_ERR_SHAPE
