"""Products with an epilogue on the device against the binary64 oracle.

With M = |x| |W|^T + |bias|, a product's binary32 sum is off by SUM(K) M: the matrix instructions sum 16 products at a time and round (or
truncate) by at most 5.25 units of 2^-23 of what has been summed; a chain has at most 512 / 16 of them in front of a binary32 result, K / 16 in front of a
BF16 one, and the chains are added in at most K / 512 + 64 further roundings.  An activation changes by at most 1.13 of its argument's error and
is itself off by (8 + 2 |v|) 2^-23 of the value (exp's bound), plus what is lost below 2^-100.  Then a product, a sum and the rounding to the output's type.
"""
import itertools

import numpy as np
import pytest
import torch

from oracle import linear as olinear

pytestmark = pytest.mark.gpu
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")


@pytest.fixture(scope="module")
def B():
    from paper_2608_15383_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def num(t):
    return None if t is None else t.double().cpu().numpy()


def normal(g, std, *size, dtype=torch.bfloat16):
    return (torch.randn(*size, generator=g) * std).to(dtype).cuda()


def inputs(T, K, N, seed, gated=False, bias=True, residual=True, dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(seed)
    f = lambda *s: normal(g, 1.0, *s, dtype=torch.float32)
    return dict(x=normal(g, 1.0, T, K), w=normal(g, K ** -0.5, N, K), bias=f(N) if bias else None, w_up=normal(g, K ** -0.5, N, K) if gated else None,
                bias_up=f(N) if gated and bias else None, residual=normal(g, 1.0, T, N, dtype=dtype) if residual else None)


def check(out, i, act, rows=slice(None)):
    dtype, K = out.dtype, i["x"].shape[1]
    x, res, got = i["x"][rows], None if i["residual"] is None else i["residual"][rows], num(out[rows])
    chain = K / 16 if dtype is torch.bfloat16 else min(K, 512) / 16
    SUM = (5.25 * (chain + 1) + K / 512 + 64) * 2.0 ** -23
    e = SUM * olinear.magnitude(num(x), num(i["w"]), num(i["bias"]))
    v = olinear.apply(num(x), num(i["w"]), num(i["bias"]))
    a = olinear.activate(v, act)
    err = 1.13 * e + (8 + 2 * np.abs(v)) * 2.0 ** -23 * (np.abs(a) + e) + 2.0 ** -100 if act != "none" else e
    ref = a
    if i["w_up"] is not None:
        u = olinear.apply(num(x), num(i["w_up"]), num(i["bias_up"]))
        eu = SUM * olinear.magnitude(num(x), num(i["w_up"]), num(i["bias_up"]))
        err = np.abs(u) * err + np.abs(a) * eu + err * eu
        ref = a * u
        err = err + 2.0 ** -24 * (np.abs(ref) + err)
    if res is not None:
        ref = ref + num(res)
        err = err + 2.0 ** -24 * (np.abs(ref) + err)
    err = err + torch.finfo(dtype).eps / 2 * (np.abs(ref) + err) + 1e-37
    assert np.isfinite(got).all()
    assert (np.abs(got - ref) <= err).all(), ((np.abs(got - ref) - err).max(), np.abs(got - ref).max())


def some_rows(T):
    return slice(None) if T <= 300 else sorted({*range(0, T, max(1, T // 150)), *range(T - 3, T), 127, 128, 255, 256})


SIZES = [(1, 8, 1), (1, 2048, 2048), (1, 4096, 33), (2, 16, 7), (3, 40, 16), (5, 64, 100), (7, 1408, 60), (8, 256, 24), (9, 512, 130), (15, 72, 129), (16, 1024, 64), (17, 2048, 257), (24, 136, 40),
         (31, 264, 1000), (32, 512, 512), (33, 2048, 60), (45, 5632, 96), (63, 64, 128), (64, 1024, 1024), (65, 128, 200), (100, 1416, 333), (127, 200, 300), (128, 512, 256), (129, 520, 264),
         (200, 2048, 1), (250, 2048, 60), (257, 576, 513), (300, 64, 2049), (500, 1000, 700), (777, 1408, 1025), (1025, 256, 136), (2000, 512, 640), (4100, 128, 520)]


@pytest.mark.parametrize("T,K,N", SIZES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("gated", [False, True])
def test_products_match_oracle(B, T, K, N, dtype, gated):
    for n, (bias, residual) in enumerate(((True, True), (False, False))):
        act = ACTS[(T + N + n + 2 * gated) % 5]
        i = inputs(T, K, N, T + K + n, gated, bias, residual, dtype)
        out = B.exmoe_linear(**i, activation=act, out_dtype=dtype)
        assert out.dtype is dtype and tuple(out.shape) == (T, N)
        check(out, i, act, some_rows(T))


@pytest.mark.parametrize("T,K,N", [(4097, 72, 700), (9000, 64, 300), (2600, 576, 1290), (1100, 1096, 4000), (3300, 512, 2049), (20000, 8, 257), (5000, 2048, 1000)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("gated", [False, True])
def test_many_tokens(B, T, K, N, dtype, gated):
    """Calls that fill the chip with tiles of 256 x 256, partly empty ones at both edges."""
    for act, bias in (("silu", True), ("none", False)):
        i = inputs(T, K, N, T + N, gated, bias, bias, dtype)
        check(B.exmoe_linear(**i, activation=act, out_dtype=dtype), i, act, some_rows(T))
    assert B.exmoe_linear_status() == B.EXMOE_OK


@pytest.mark.parametrize("T", [1, 12, 40, 200, 600, 12000])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("gated", [False, True])
def test_every_activation(B, T, act, gated):
    i = inputs(T, 256, 192, T, gated, dtype=torch.float32)
    i["bias"] = torch.linspace(-120, 120, 192).cuda()                      # over the activations' whole range
    check(B.exmoe_linear(**i, activation=act), i, act, some_rows(T))
    assert torch.equal(B.exmoe_linear(**i, activation=act), B.exmoe_linear(**i, activation=ACTS.index(act)))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("T,N,shift", [(1, 64, 0), (9, 64, 1), (20, 61, 3), (70, 96, 8), (150, 130, 2), (300, 256, 5), (700, 384, 0)])
def test_strides_in_place_and_what_lies_between(B, T, N, shift, dtype, gated):
    """Column ranges of wider matrices for x, w and w_up; residual and out column ranges of one buffer, at any offset, in place; what lies around keeps its values."""
    K = 200
    i = inputs(T, K, N, 7, gated, dtype=dtype)
    want = B.exmoe_linear(**i, activation="silu")
    for name, rows, at in (("x", T, 8), ("w", N, 16), ("w_up", N, 24)):
        if i[name] is not None:
            wide = torch.full((rows, K + 40), float("nan"), dtype=torch.bfloat16, device="cuda")
            wide[:, at:at + K] = i[name]
            i[name] = wide[:, at:at + K]
    wide = torch.full((T + 1, N + 16), 3.0, dtype=dtype, device="cuda")
    view = wide[:T, shift:shift + N]
    view.copy_(i["residual"])
    out = B.exmoe_linear(**{**i, "residual": view}, activation="silu", out=view)
    assert out is view and torch.equal(view, want)
    assert (wide[:, :shift] == 3.0).all() and (wide[:, shift + N:] == 3.0).all() and (wide[T] == 3.0).all()
    other = torch.full((T, 2 * N + 32), 5.0, dtype=dtype, device="cuda")
    other[:, :N] = i["residual"]
    B.exmoe_linear(**{**i, "residual": other[:, :N]}, activation="silu", out=other[:, N + 16:2 * N + 16])
    assert torch.equal(other[:, N + 16:2 * N + 16], want) and torch.equal(other[:, :N], i["residual"]) and (other[:, N:N + 16] == 5.0).all() and (other[:, 2 * N + 16:] == 5.0).all()


@pytest.mark.parametrize("T", [5, 40])
def test_rows_far_apart(B, T):
    """Rows 2^28 bytes apart: offsets beyond 32 bits."""
    K, N = 64, 40
    i = inputs(T, K, N, 4)
    want = B.exmoe_linear(**i)
    big = torch.empty(T << 27, dtype=torch.bfloat16, device="cuda")
    far = [big[at:].as_strided((T, w), (1 << 27, 1)) for at, w in ((0, K), (64, N), (128, N))]
    far[0].copy_(i["x"])
    far[1].copy_(i["residual"])
    assert torch.equal(B.exmoe_linear(far[0], i["w"], i["bias"], residual=far[1], out=far[2]), want)
    del far
    w = big[:].as_strided((min(N, T), K), (1 << 27, 1))
    w.copy_(i["w"][:min(N, T)])
    assert torch.equal(B.exmoe_linear(i["x"], w), B.exmoe_linear(i["x"], i["w"][:min(N, T)].contiguous()))


@pytest.mark.parametrize("T", [1, 16, 100, 1000])
def test_infinities_and_nan_stay_in_their_rows(B, T):
    i = inputs(T, 128, 96, 5, residual=False)
    want = B.exmoe_linear(**i)
    i["x"][T // 2, 3] = float("inf")
    i["x"][0, 5] = float("nan")
    out = B.exmoe_linear(**i)
    keep = [t for t in range(T) if t not in (0, T // 2)]
    assert torch.equal(out[keep], want[keep]) and torch.isnan(out[0]).all()
    if T > 1:
        assert not torch.isfinite(out[T // 2].float()).any()


def test_one_row_without_distance_and_empty_calls(B):
    i = inputs(1, 64, 24, 1)
    x = i["x"].as_strided((1, 64), (3, 1))                                 # a single row's distance is nobody's business
    assert torch.equal(B.exmoe_linear(x, i["w"], i["bias"]), B.exmoe_linear(i["x"], i["w"], i["bias"]))
    empty = B.exmoe_linear(i["x"][:0], i["w"], out_dtype=torch.float32)
    assert tuple(empty.shape) == (0, 24) and empty.dtype is torch.float32


@pytest.mark.parametrize("T", [1, 30, 300])
def test_streams_and_graphs(B, T):
    """A shared expert's two products: at once on several streams, captured, replayed with other inputs in the same place."""
    g = torch.Generator().manual_seed(T)
    H, F = 256, 512
    x, routed, w, u, d = normal(g, 1.0, T, H), normal(g, 1.0, T, H), normal(g, 0.05, F, H), normal(g, 0.05, F, H), normal(g, 0.05, H, F)

    def block(stream=None):
        act = B.exmoe_linear(x, w, w_up=u, activation="silu", stream=stream)
        return B.exmoe_linear(act, d, residual=routed, stream=stream)
    want = block()
    torch.cuda.synchronize()
    outs = [block(st) for st in [torch.cuda.Stream() for _ in range(4)] for _ in range(3)]
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    graph, st = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(st):
        block()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=st):
            out = block()
    for n in range(3):
        if n == 2:
            x.copy_(x.flip(0).clone() * 0.5)
            want = block()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_refusals(B):
    i = inputs(4, 64, 24, 1, gated=True)
    x, w, u, b, r = i["x"], i["w"], i["w_up"], i["bias"], i["residual"]
    for call in (lambda: B.exmoe_linear(x.float(), w), lambda: B.exmoe_linear(x, w.float()), lambda: B.exmoe_linear(x[:, :32], w), lambda: B.exmoe_linear(x, w, b[:8]),
                 lambda: B.exmoe_linear(x, w, b.bfloat16()), lambda: B.exmoe_linear(x, w, w_up=u[:8]), lambda: B.exmoe_linear(x, w, bias_up=b),
                 lambda: B.exmoe_linear(x, w, activation="tanh"), lambda: B.exmoe_linear(x, w, residual=r[:, :8]), lambda: B.exmoe_linear(x, w, residual=r, out_dtype=torch.float32),
                 lambda: B.exmoe_linear(x, w, out_dtype=torch.float16), lambda: B.exmoe_linear(x, w, out=r.t()), lambda: B.exmoe_linear(x.cpu(), w),
                 lambda: B.exmoe_linear(x, w, residual=r, out=r.float()), lambda: B.exmoe_linear(x.view(2, 2, 64), w)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: B.exmoe_linear(x[:, :60], w[:, :60]), lambda: B.exmoe_linear(x, w, activation=7), lambda: B.exmoe_linear(x, w, out=x[:, :24]),
                 lambda: B.exmoe_linear(x, w[:, :24].contiguous().new_zeros(24, 68)[:, :64])):
        with pytest.raises(B.ExmoeError):
            call()


def test_router_tuning_step_and_block(B):
    """A sparse block with a shared expert and a step of its router's training, as a program runs them: logits, choice, routed experts, shared expert on
    top, losses, gradient on the logits; against the oracles at every joint."""
    from oracle import gate as ogate
    from oracle import gate_loss as oloss
    from paper_2608_15383_b200 import synth

    import helpers
    s, T, F = synth.TINY, 96, 640
    ora, bank = helpers.make_layer(s, 11)
    cache = B.Cache(s, [bank], s.num_experts, T)
    g = torch.Generator().manual_seed(12)
    x, wr = normal(g, 1.0, T, s.d_model), normal(g, 0.05, s.num_experts, s.d_model)
    w, u, d = normal(g, 0.06, F, s.d_model), normal(g, 0.06, F, s.d_model), normal(g, 0.04, s.d_model, F)
    gate = B.Gate(score="sigmoid", renormalise=True, scale=2.0)
    offsets = torch.tensor([0, 30, 96], dtype=torch.int32, device="cuda")
    logits = B.exmoe_linear(x, wr, out_dtype=torch.float32)
    check(logits, dict(x=x, w=wr, bias=None, w_up=None, bias_up=None, residual=None), "none")
    ids, weights = B.exmoe_gate_logits(s, gate, logits)
    y = cache.forward(0, x, ids, weights)
    act = B.exmoe_linear(x, w, w_up=u, activation="silu")
    check(act, dict(x=x, w=w, bias=None, w_up=u, bias_up=None, residual=None), "silu")
    out = B.exmoe_linear(act, d, residual=y)
    check(out, dict(x=act, w=d, bias=None, w_up=None, bias_up=None, residual=y), "none")
    losses, counts, sums, kept = B.exmoe_balance_loss(s, gate, logits, ids, offsets=offsets)
    want = oloss.balance(num(logits), ids.cpu().numpy(), gate, None, offsets.tolist())
    np.testing.assert_allclose(num(losses), want[0], rtol=1e-5)
    assert np.array_equal(counts.cpu().numpy(), want[1]) and int(counts.sum()) == T * s.top_k
    assert np.array_equal(ids.cpu().numpy(), ogate.choose(num(logits), gate, s.top_k)[0])
    dw = normal(g, 1.0, T, s.top_k, dtype=torch.float32)
    dl = torch.tensor([0.01, 0.001], device="cuda")
    dz = B.exmoe_gate_backward(s, gate, logits, ids, dw, dl, counts, kept, offsets=offsets)
    ref, size = oloss.backward(num(logits), ids.cpu().numpy(), gate, s.top_k, num(dw), num(dl), want[1], want[3], None, offsets.tolist())
    assert (np.abs(num(dz) - ref) <= 4 * 96 * 2.0 ** -23 * size + 2.0 ** -24 * np.abs(ref) + 1e-35).all()
    assert cache.status() == B.EXMOE_OK
    cache.close()
