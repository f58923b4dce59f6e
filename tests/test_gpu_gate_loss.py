"""The gate's losses and gradients on the device against the binary64 oracle.

Scores: an exponential is off by 2 units of 2^-23 (the instruction's bound) and by its argument's roundings, |z - largest| 2^-23 at most (the product's, and the
difference's or the shift's): 52 2^-23 as far as 52 below the largest, where a score is e^-52 of the whole; the sum over the experts rounds at most 32 times one after the other, division and products a few times: a score is within
REL = (8 + 52 + 36) 2^-23 of itself, or lost below 2^-126.  Sums of scores have terms of one sign, and a chain of at most rows + 64 additions.
A gradient is a sum of terms whose sizes the oracle gives, each a product of four such factors at most.
"""
import itertools
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from oracle import gate_loss as oloss

pytestmark = pytest.mark.gpu
REL = 96 * 2.0 ** -23
INF = float("inf")


@pytest.fixture(scope="module")
def B():
    from paper_2608_15383_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def shape(E, k):
    return SimpleNamespace(d_model=128, num_experts=E, top_k=k)


def gate(score="softmax", renormalise=False, scale=1.0):
    return SimpleNamespace(score=score, num_groups=1, top_groups=1, group_score="max", renormalise=renormalise, scale=scale)


def num(t):
    return None if t is None else t.double().cpu().numpy()


def inputs(T, E, k, seed, dtype=torch.float32, S=0, masked=0.0, off=0.0, spread=1.0, stride=None):
    g = torch.Generator().manual_seed(seed)
    wide = torch.full((T, stride or E), float("nan"), dtype=dtype)
    wide[:, :E] = (torch.randn(T, E, generator=g) * spread + torch.randn(E, generator=g)).to(dtype)
    z = wide[:, :E]
    if off:
        z[torch.rand(T, E, generator=g) < off] = -INF
    ids = torch.rand(T, E, generator=g).argsort(1)[:, :k].int()
    offsets = None
    if S:
        cuts = torch.sort(torch.randint(0, T + 1, (S + 1,), generator=g)).values
        cuts[0], cuts[-1] = (0, T) if seed % 2 else (min(1, T), max(T - 1, min(1, T)))
        offsets = torch.sort(cuts).values.int()
    mask = torch.rand(T, generator=g) >= masked if masked else None
    dev = lambda t: None if t is None else t.cuda()
    return wide.cuda()[:, :E], dev(ids), dev(mask), dev(offsets), g


def host(t):
    return None if t is None else t.cpu().numpy()


def check_balance(B, s, g, z, ids, mask, offsets):
    losses, counts, sums, kept = B.exmoe_balance_loss(s, g, z, ids, mask=mask, offsets=offsets)
    T = z.shape[0]
    want, c, p, n = oloss.balance(num(z), host(ids), g, host(mask), None if offsets is None else offsets.tolist())
    assert counts.dtype is torch.int32 and np.array_equal(host(counts), c) and np.array_equal(host(kept), n)
    rel = REL + (T + 64) * 2.0 ** -24
    err = np.abs(num(sums) - p)
    assert (err <= rel * p + T * 2.0 ** -126).all(), (err / np.maximum(p, 1e-30)).max()
    got = num(losses)
    assert abs(got[0] - want[0]) <= 2 * rel * want[0] + 1e-37
    # of the tokens that count: the logarithm of the sum is off by 3 REL, and by the roundings of it and of the largest logit
    on = np.ones(T, bool) if mask is None else host(mask)
    if offsets is not None:
        on = on & (np.arange(T) >= int(offsets[0])) & (np.arange(T) < int(offsets[-1]))
    v = num(z)[on]
    lse = np.abs([oloss.log_sum(r) for r in v]).max(initial=0)
    d = 3 * REL + 2.0 ** -22 * (lse + np.abs(np.where(np.isfinite(v), v, 0)).max(initial=0))
    assert abs(got[1] - want[1]) <= d * (2 * lse + d) + rel * want[1]
    return losses, counts, sums, kept


SIZES = [(1, 8, 2), (2, 1, 1), (7, 3, 3), (16, 64, 8), (33, 60, 4), (65, 61, 5), (100, 65, 16), (257, 128, 8), (130, 200, 12), (64, 256, 8), (48, 257, 8), (300, 512, 10),
         (20, 513, 3), (41, 1000, 33), (17, 1024, 600), (9, 1025, 8), (30, 4096, 40)]


@pytest.mark.parametrize("T,E,k", SIZES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_balance_matches_oracle(B, T, E, k, score, dtype):
    for i, (S, masked, off, stride) in enumerate(((0, 0.0, 0.0, None), (3, 0.3, 0.1, E + 4), (1, 0.9, 0.0, E + 1), (T + 3, 0.1, 0.5, None))):
        z, ids, mask, offsets, _ = inputs(T, E, k, 10 * T + i, dtype, S, masked, off, stride=stride)
        check_balance(B, shape(E, k), gate(score), z, ids, mask, offsets)


@pytest.mark.parametrize("T,E,k,S", [(1151, 64, 8, 0), (1152, 64, 8, 1), (5000, 64, 4, 7), (5001, 60, 8, 900), (3000, 256, 8, 2), (4097, 300, 6, 300), (2500, 700, 2, 5), (700, 2048, 4, 40),
                                     (20000, 16, 2, 3)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_many_tokens_and_sequences_across_tiles(B, T, E, k, S, score):
    z, ids, mask, offsets, _ = inputs(T, E, k, T + S, S=S, masked=0.2)
    check_balance(B, shape(E, k), gate(score), z, ids, mask, offsets)


def test_edges_of_sequences(B):
    """Empty sequences before, between and behind; sequences that begin and end at the edges of tiles; no token at all."""
    for T, E in ((2400, 64), (1000, 256), (40, 1500)):
        z, ids, _, _, _ = inputs(T, E, 2, T)
        for cuts in ([0, 0, 0, T, T, T], [0, T // 16, T // 16, T // 8, T], list(range(0, T + 1, 128 if T > 200 else 8)), [5, 5, 6, T - 3], [T, T], [0, 0], [0, T - 1, T, T], [1, T]):
            check_balance(B, shape(E, 2), gate(), z, ids, None, torch.tensor(cuts, dtype=torch.int32, device="cuda"))
    for T in (0, 50):
        z, ids, _, _, _ = inputs(T, 8, 2, 1)
        for S in (1, 5):
            out = B.exmoe_balance_loss(shape(8, 2), gate(), z, ids, mask=torch.zeros(T, dtype=torch.bool, device="cuda"), offsets=torch.zeros(S + 1, dtype=torch.int32, device="cuda"))
            assert all((t == 0).all() for t in out) and out[1].shape == (S, 8)


@pytest.mark.parametrize("cuts", [[0, 50, 40, 100], [-1, 100], [0, 101], [100, 0], [0, -7, 100, 5000000, 3, 100]])
def test_offsets_that_do_not_ascend_are_reported(B, cuts):
    """And nothing is written outside of the outputs.  (The kernel clips what it reads through them: checked on the CPU by reading.)"""
    T, E, S = 100, 16, len(cuts) - 1
    z, ids, _, _, _ = inputs(T, E, 2, 3)
    room = torch.full((3 * S * E,), 7, dtype=torch.int32, device="cuda")
    out = (torch.empty(2, device="cuda"), room[S * E:2 * S * E].view(S, E), torch.empty(S, E, device="cuda"), torch.empty(S, dtype=torch.int32, device="cuda"))
    assert B.exmoe_balance_loss(shape(E, 2), gate(), z, ids, offsets=torch.tensor(cuts, dtype=torch.int32, device="cuda"), out=out) is out
    assert torch.isnan(out[0]).all() and (room[:S * E] == 7).all() and (room[2 * S * E:] == 7).all()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_masked_experts_lowest_values_and_nan_padding(B, score):
    T, E, k = 40, 64, 4
    z, ids, _, _, _ = inputs(T, E, k, 8)
    z[0] = -INF                                                            # no expert left
    z[1] = torch.finfo(torch.float32).min                                  # masked by the type's lowest value: an even row
    z[2, 1:] = torch.finfo(torch.float32).min
    z[3] -= 200                                                            # sigmoids that leave binary32
    z[4] += 300
    z[5, ::2] = -INF
    z[6:9] = float("nan")
    ids[3, 0], ids[4, 1] = -1, E
    mask = torch.ones(T, dtype=torch.bool, device="cuda")
    mask[6:9] = False
    mask[1:3] = False                                                      # (their logarithms' squares leave binary32)
    _, counts, _, kept = check_balance(B, shape(E, k), gate(score), z, ids, mask, None)
    mask[1:3] = True
    sums = B.exmoe_balance_loss(shape(E, k), gate(score), z, ids, mask=mask)[2]
    want = oloss.balance(num(z), host(ids), gate(score), host(mask))[2]
    assert np.allclose(num(sums), want, rtol=1e-4)
    mask[7] = True                                                         # a NaN that counts
    losses, _, sums, _ = B.exmoe_balance_loss(shape(E, k), gate(score), z, ids, mask=mask)
    assert torch.isnan(losses).all() and torch.isnan(sums).all()


def check_backward(B, s, g, z, ids, mask, offsets, dw, dl, counts, kept, out=None):
    got = B.exmoe_gate_backward(s, g, z, ids, d_weights=dw, d_losses=dl, counts=counts, kept=kept, mask=mask, offsets=offsets, out=out)
    assert got.dtype is z.dtype
    want, size = oloss.backward(num(z), host(ids), g, s.top_k, num(dw), num(dl), host(counts), host(kept), host(mask), None if offsets is None else offsets.tolist())
    tol = 4 * REL * size + 1e-35
    tol = tol + torch.finfo(z.dtype).eps / 2 * (np.abs(want) + tol)
    err = np.abs(num(got) - want)
    assert (err <= tol).all(), (err - tol).max()
    return got


@pytest.mark.parametrize("T,E,k", SIZES)
@pytest.mark.parametrize("score,renormalise", [("softmax", False), ("softmax", True), ("sigmoid", False), ("sigmoid", True)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_backward_matches_oracle(B, T, E, k, score, renormalise, dtype):
    s, g = shape(E, k), gate(score, renormalise, 2.5)
    for i, (S, masked, off, stride) in enumerate(((0, 0.0, 0.0, None), (3, 0.3, 0.1, E + 4), (T + 3, 0.1, 0.5, E + 3))):
        z, ids, mask, offsets, rng = inputs(T, E, k, 10 * T + i, dtype, S, masked, off, stride=stride)
        dw = torch.randn(T, k, generator=rng).cuda()
        dl = torch.tensor([0.5, 0.1], device="cuda")
        _, counts, _, kept = B.exmoe_balance_loss(s, g, z, ids, mask=mask, offsets=offsets)
        for w, l in ((dw, dl), (dw, None), (None, dl)):
            check_backward(B, s, g, z, ids, mask, offsets, w, l, counts, kept)


@pytest.mark.parametrize("T,E,k,S", [(5000, 64, 8, 7), (5001, 60, 8, 900), (3000, 256, 8, 2), (1500, 300, 6, 300), (1300, 700, 2, 5), (700, 2048, 4, 40)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_backward_of_many_tokens(B, T, E, k, S, score):
    s, g = shape(E, k), gate(score, True, 1.0)
    z, ids, mask, offsets, rng = inputs(T, E, k, T + S, S=S, masked=0.2)
    _, counts, _, kept = B.exmoe_balance_loss(s, g, z, ids, mask=mask, offsets=offsets)
    check_backward(B, s, g, z, ids, mask, offsets, torch.randn(T, k, generator=rng).cuda(), torch.tensor([2.0, 0.3], device="cuda"), counts, kept)


@pytest.mark.parametrize("score,renormalise", [("softmax", False), ("softmax", True), ("sigmoid", False), ("sigmoid", True)])
@pytest.mark.parametrize("E,k", [(64, 4), (40, 12), (256, 8), (700, 3)])
def test_backward_edges(B, score, renormalise, E, k):
    """Rows without experts, chosen ones that are off or lost beside the row's largest, ids that are named twice or that do not exist, NaN in padding."""
    T = 24
    s, g = shape(E, k), gate(score, renormalise, 1.5)
    z, ids, _, _, rng = inputs(T, E, k, 9)
    z[0] = -INF
    z[1] = torch.finfo(torch.float32).min
    z[2, ids[2].long()] -= 300                                             # chosen by a bias, scores lost
    z[3] -= 200
    z[4] += 300
    z[5, ids[5, :2].long()] = -INF
    z[6, ids[6].long()] = -INF
    z[7:9] = float("nan")
    ids[10, 1] = ids[10, 0]
    ids[11] = ids[11, 0]
    ids[12, 0], ids[13, 2], ids[14, 0] = -1, E, 2 ** 31 - 1
    ids[15] = -5
    mask = torch.ones(T, dtype=torch.bool, device="cuda")
    mask[7:9] = False
    dw = torch.randn(T, k, generator=rng).cuda()
    dl = torch.tensor([1.0, 0.0], device="cuda")
    _, counts, _, kept = B.exmoe_balance_loss(s, g, z, ids, mask=mask)
    for w, l in ((dw, dl), (dw, None), (None, dl)):
        got = check_backward(B, s, g, z, ids, mask, None, w, l, counts, kept)
        assert (got[7:9] == 0).all() and (got[0] == 0).all()
    assert torch.equal(B.exmoe_gate_backward(s, g, z, mask=mask), torch.zeros_like(z))


def test_gradient_against_differences(B):
    """Differences of the device's own losses: off by the losses' roundings over the step, 2 2^-22 / (2 h), and by h^2."""
    T, E, k, h = 6, 8, 2, 2.0 ** -5
    for score in ("softmax", "sigmoid"):
        s, g = shape(E, k), gate(score)
        z, ids, _, _, _ = inputs(T, E, k, 4)
        _, counts, _, kept = B.exmoe_balance_loss(s, g, z, ids)
        dl = torch.tensor([0.6, 0.4], device="cuda")
        got = num(B.exmoe_gate_backward(s, g, z, ids, d_losses=dl, counts=counts, kept=kept))
        for t, e in itertools.product(range(T), range(E)):
            v = []
            for sign in (1, -1):
                y = z.clone()
                y[t, e] += sign * h
                v.append(float((B.exmoe_balance_loss(s, g, y, ids)[0].double() * dl).sum()))
            assert abs(got[t, e] - (v[0] - v[1]) / (2 * h)) <= 2.0 ** -21 * 8 / h + h * h


def test_strides_and_what_lies_between(B):
    T, E, k = 70, 60, 4
    s, g = shape(E, k), gate("sigmoid", True)
    for dtype, shift, width in itertools.product((torch.float32, torch.bfloat16), (0, 4, 3), (72, 71)):
        z, ids, mask, offsets, rng = inputs(T, E, k, 5, dtype, S=3, masked=0.2)
        dw, dl = torch.randn(T, k, generator=rng).cuda(), torch.tensor([1.0, 0.1], device="cuda")
        _, counts, _, kept = B.exmoe_balance_loss(s, g, z, ids, mask=mask, offsets=offsets)
        want = B.exmoe_gate_backward(s, g, z, ids, dw, dl, counts, kept, mask, offsets)
        wide = torch.full((T + 1, width), 3.0, dtype=dtype, device="cuda")
        view = wide[:T, shift:shift + E]
        assert B.exmoe_gate_backward(s, g, z, ids, dw, dl, counts, kept, mask, offsets, out=view) is view
        assert torch.allclose(view.float(), want.float(), rtol=2e-2 if dtype is torch.bfloat16 else 1e-5, atol=1e-7)
        assert (wide[:, :shift] == 3).all() and (wide[:, shift + E:] == 3).all() and (wide[T] == 3).all()


def test_rows_far_apart(B):
    """Rows 2^30 bytes and more apart: offsets beyond 32 bits."""
    T, E, k = 5, 16, 2
    z, ids, _, _, rng = inputs(T, E, k, 6)
    big = torch.empty(T << 28, device="cuda")
    far, out = (big[at:].as_strided((T, E), (1 << 28, 1)) for at in (0, 64))
    far.copy_(z)
    s, g, dw, dl = shape(E, k), gate(), torch.randn(T, k, generator=rng).cuda(), torch.tensor([1.0, 0.1], device="cuda")
    a, b = B.exmoe_balance_loss(s, g, z, ids), B.exmoe_balance_loss(s, g, far, ids)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    B.exmoe_gate_backward(s, g, far, ids, dw, dl, a[1], a[3], out=out)
    assert torch.equal(out, B.exmoe_gate_backward(s, g, z, ids, dw, dl, a[1], a[3]))


@pytest.mark.parametrize("T,E,S", [(300, 64, 3), (9000, 64, 0), (6000, 256, 50)])
def test_streams_graphs_and_the_same_bits(B, T, E, S):
    k = 4
    s, g = shape(E, k), gate("softmax", True)
    z, ids, mask, offsets, rng = inputs(T, E, k, 7, S=S, masked=0.1)
    dw, dl = torch.randn(T, k, generator=rng).cuda(), torch.tensor([1.0, 0.1], device="cuda")

    def step(stream=None):
        out = B.exmoe_balance_loss(s, g, z, ids, mask, offsets, stream=stream)
        return out + (B.exmoe_gate_backward(s, g, z, ids, dw, dl, out[1], out[3], mask, offsets, stream=stream),)
    want = step()
    torch.cuda.synchronize()
    for _ in range(3):
        assert all(torch.equal(x, y) for x, y in zip(step(), want))
    streams = [torch.cuda.Stream() for _ in range(4)]
    outs = [step(st) for st in streams for _ in range(3)]                  # at once
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for out in outs for x, y in zip(out, want))
    graph, st = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(st):
        step()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=st):
            out = step()
    for i in range(3):
        if i == 2:
            z.copy_(z.flip(0).clone())
            want = None
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out, want or step()))


def test_refusals(B):
    T, E, k = 8, 16, 2
    z, ids, _, _, rng = inputs(T, E, k, 2)
    s, g = shape(E, k), gate()
    losses, counts, sums, kept = B.exmoe_balance_loss(s, g, z, ids)
    dl, dw = torch.ones(2, device="cuda"), torch.ones(T, k, device="cuda")
    for call in (lambda: B.exmoe_balance_loss(s, g, z, ids.long()), lambda: B.exmoe_balance_loss(s, g, z, ids[:, :1]), lambda: B.exmoe_balance_loss(s, g, z.double(), ids),
                 lambda: B.exmoe_balance_loss(s, g, z[:, :8], ids), lambda: B.exmoe_balance_loss(s, g, z, ids, mask=torch.ones(T, device="cuda")),
                 lambda: B.exmoe_balance_loss(s, g, z, ids, mask=torch.ones(T - 1, dtype=torch.bool, device="cuda")), lambda: B.exmoe_balance_loss(s, g, z, ids[:4]),
                 lambda: B.exmoe_balance_loss(s, g, z, None), lambda: B.exmoe_balance_loss(s, g, z, ids, offsets=torch.zeros(1, dtype=torch.int32, device="cuda")),
                 lambda: B.exmoe_balance_loss(s, g, z, ids, offsets=torch.zeros(2, dtype=torch.int64, device="cuda")), lambda: B.exmoe_balance_loss(s, g, z.t().contiguous().t(), ids),
                 lambda: B.exmoe_balance_loss(s, g, z, ids, out=(losses, counts, sums)), lambda: B.exmoe_balance_loss(s, g, z, ids, out=(losses, counts, sums, kept[:0])),
                 lambda: B.exmoe_gate_backward(s, g, z, None, d_weights=dw), lambda: B.exmoe_gate_backward(s, g, z, ids, d_weights=dw[:, :1]),
                 lambda: B.exmoe_gate_backward(s, g, z, ids, d_losses=dl), lambda: B.exmoe_gate_backward(s, g, z, ids, d_losses=dl[:1], counts=counts, kept=kept),
                 lambda: B.exmoe_gate_backward(s, g, z, ids, d_losses=dl, counts=counts[:, :8], kept=kept), lambda: B.exmoe_gate_backward(s, g, z, out=z.bfloat16())):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(B.ExmoeError):
        B.exmoe_gate_backward(s, g, z, out=z)                              # in place
    with pytest.raises(B.ExmoeError):
        B.exmoe_balance_loss(shape(E, 17), g, z, torch.zeros(T, 17, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("S,E", [(1, 8), (3, 60), (20, 64), (40, 256)])
def test_results_are_tensors_of_their_own(B, S, E):
    """Few small results or many: shapes, types and strides of theirs, and what is written to one is in no other."""
    T, k = 64, 2
    z, ids, _, offsets, _ = inputs(T, E, k, 11, S=S)
    want = [t.clone() for t in B.exmoe_balance_loss(shape(E, k), gate(), z, ids, offsets=offsets)]
    for i in range(4):
        got = B.exmoe_balance_loss(shape(E, k), gate(), z, ids, offsets=offsets)
        assert [tuple(t.shape) for t in got] == [(2,), (S, E), (S, E), (S,)] and all(t.is_contiguous() and t.data_ptr() % 16 == 0 for t in got)
        assert [t.dtype for t in got] == [torch.float32, torch.int32, torch.float32, torch.int32]
        got[i].fill_(7)
        assert all(torch.equal(g, w) for j, (g, w) in enumerate(zip(got, want)) if j != i)
        assert not any(t.requires_grad for t in got) and torch.equal(got[i].cpu() + 0, torch.full_like(want[i], 7).cpu())
