"""Low-rank adapters on the device against the binary64 oracle.

An output is base + scale * sum_j b_j v_j, v_j = sum_i a_ji x_i.  With M = |scale| |B| (|A| |x|) the binary32 sums are off by
(K / 64 + r + 64) 2^-23 M at most (chains of that many additions, truncated ones among them), an inner product kept as two BF16 numbers by
2^-16 of it, as three by 2^-24; base + product rounds once more in binary32 and once to the output's type.
"""
import numpy as np
import pytest
import torch

from oracle import gate as ogate
from oracle import lora as olora
from paper_2608_15383_b200 import synth

import helpers

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2608_15383_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def normal(g, std, *size, dtype=torch.bfloat16):
    return (torch.randn(*size, generator=g) * std).to(dtype)


def num(t):
    return None if t is None else t.double().cpu().numpy()


def check(out, x, a, b, scale, ids, base, rows=slice(None)):
    got, dtype = num(out), out.dtype
    x, ids, base = x[rows], ids[rows], None if base is None else base[rows]
    got = got[rows]
    ref = olora.apply(num(x), num(a), num(b), num(scale), ids.cpu().numpy(), num(base))
    M = olora.magnitude(num(x), num(a), num(b), num(scale), ids.cpu().numpy())
    kept = 2.0 ** -16 if dtype is torch.bfloat16 else 2.0 ** -24
    unit = torch.finfo(dtype).eps / 2
    tol = ((a.shape[2] / 64 + a.shape[1] + 64) * 2.0 ** -23 + kept) * M
    tol = tol + 2.0 ** -24 * (np.abs(ref) + tol)
    tol = tol + unit * (np.abs(ref) + tol) + 1e-37
    assert np.isfinite(got).all()
    assert (np.abs(got - ref) <= tol).all(), (np.abs(got - ref) - tol).max()
    none = (ids.cpu().numpy() < 0) | (ids.cpu().numpy() >= a.shape[0])
    assert np.array_equal(got[none], 0 * got[none] if base is None else num(base)[none])      # untouched, to the bit


def inputs(T, n, r, K, N, seed, dtype=torch.bfloat16, ids=None, base=True):
    g = torch.Generator().manual_seed(seed)
    x, a, b = normal(g, 1.0, T, K), normal(g, 0.05, n, r, K), normal(g, 0.05, n, N, r)
    scale = torch.rand(n, generator=g) * 3 - 1
    if ids is None:
        ids = torch.randint(-1, n, (T,), generator=g)
    return x.cuda(), a.cuda(), b.cuda(), scale.cuda(), ids.int().cuda(), normal(g, 1.0, T, N, dtype=dtype).cuda() if base else None


CASES = [(1, 1, 8, 128, 128), (1, 8, 16, 2048, 2048), (2, 3, 8, 8, 1), (5, 4, 64, 1024, 2048), (16, 16, 16, 512, 200), (33, 5, 24, 1408, 60), (64, 32, 16, 2048, 2048),
         (65, 1, 8, 264, 31), (130, 7, 128, 512, 1000), (200, 200, 8, 256, 256), (333, 3, 16, 2048, 5632), (700, 12, 32, 1920, 1030), (1000, 1, 16, 1000, 64),
         (2050, 40, 8, 256, 512)]


@pytest.mark.parametrize("T,n,r,K,N", CASES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_adapters_match_oracle(B, T, n, r, K, N, dtype):
    for base in (True, False):
        x, a, b, scale, ids, y = inputs(T, n, r, K, N, T + r, dtype, base=base)
        plan = B.exmoe_lora_plan(ids, n)
        out = B.exmoe_lora(plan, x, a, b, scale, base=y, out_dtype=dtype)
        assert out.dtype is dtype and tuple(out.shape) == (T, N)
        check(out, x, a, b, scale, ids, y)
        assert B.exmoe_lora_plan_status(plan) == B.EXMOE_OK


@pytest.mark.parametrize("T,n,r,K,N", [(1300, 2, 64, 256, 264), (1500, 3, 128, 392, 200), (1200, 200, 32, 128, 72), (600, 1, 128, 520, 1), (650, 40, 64, 64, 130),
                                       (8, 1024, 128, 8, 1000), (3000, 5, 24, 1032, 33), (1, 1, 128, 4096, 4096), (5000, 1, 16, 4096, 16)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_every_rank_with_every_tile(B, T, n, r, K, N, dtype):
    """Tiles of 16, 32 and 64 rows with ranks of each kernel, clusters of one to eight CTAs, K and N of less than a step."""
    x, a, b, scale, ids, y = inputs(T, n, r, K, N, T + N, dtype)
    rows = list(range(0, T, 1 + T // 300)) + [T - 1]
    check(B.exmoe_lora(B.exmoe_lora_plan(ids, n), x, a, b, scale, base=y), x, a, b, scale, ids, y, rows)


def test_rows_far_apart(B):
    """Rows of x, base and out 2^30 bytes apart: offsets beyond 32 bits."""
    T, n, r, K, N = 5, 2, 8, 64, 40
    x, a, b, scale, ids, y = inputs(T, n, r, K, N, 4, ids=torch.tensor([1, 0, -1, 1, 0]))
    big = torch.empty(T << 29, dtype=torch.bfloat16, device="cuda")
    far = [big[at:].as_strided((T, w), (1 << 29, 1)) for at, w in ((0, K), (64, N), (128, N))]
    far[0].copy_(x)
    far[1].copy_(y)
    far[2].fill_(7.0)
    out = B.exmoe_lora(B.exmoe_lora_plan(ids, n), far[0], a, b, scale, base=far[1], out=far[2])
    assert torch.equal(out, B.exmoe_lora(B.exmoe_lora_plan(ids, n), x, a, b, scale, base=y))


@pytest.mark.parametrize("T,n,r,K,N", [(3, 2, 16, 256, 136), (40, 6, 8, 512, 77), (150, 2, 64, 1024, 1024), (600, 9, 16, 640, 384)])
def test_results_depend_on_the_own_row_only(B, T, n, r, K, N):
    """In another order, and with other rows and adapters around them: the same bits.  Alone: the same value."""
    x, a, b, scale, ids, y = inputs(T, n, r, K, N, 5)
    out = B.exmoe_lora(B.exmoe_lora_plan(ids, n), x, a, b, scale, base=y)

    def call(x, ids, y):
        return B.exmoe_lora(B.exmoe_lora_plan(ids.contiguous(), n), x.contiguous(), a, b, scale, base=y.contiguous())
    back = list(range(T - 1, -1, -1))
    assert torch.equal(call(x[back], ids[back], y[back]).view(torch.int16), out[back].view(torch.int16))
    others = inputs(T, n, r, K, N, 6)
    keep = torch.arange(T, device="cuda") % 3 == 1
    mixed = [torch.where(keep.view(-1, *[1] * (u.dim() - 1)), u, v) for u, v in ((x, others[0]), (ids, others[4]), (y, others[5]))]
    assert torch.equal(call(*mixed)[keep].view(torch.int16), out[keep].view(torch.int16))
    for rows in ([T // 2], list(range(0, T, 3))):
        check(call(x[rows], ids[rows], y[rows]), x[rows], a, b, scale, ids[rows], y[rows])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,N,shift", [(9, 64, 0), (70, 96, 8), (70, 61, 3), (300, 256, 1)])
def test_strides_in_place_and_what_lies_between(B, T, N, shift, dtype):
    """x a column range of wider rows; base and out column ranges of one buffer, at an offset that is no multiple of 16 bytes too, in
    place; the columns around them, and the rows behind the last, keep what they held."""
    n, r, K = 3, 16, 256
    x, a, b, scale, ids, y = inputs(T, n, r, K, N, 7, dtype)
    wide_x = torch.full((T, K + 24), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide_x[:, 8:K + 8] = x
    plan = B.exmoe_lora_plan(ids, n)
    want = B.exmoe_lora(plan, x, a, b, scale, base=y)
    wide = torch.full((T + 1, N + 16), 3.0, dtype=dtype, device="cuda")
    wide[:T, shift:shift + N] = y
    view = wide[:T, shift:shift + N]
    out = B.exmoe_lora(plan, wide_x[:, 8:K + 8], a, b, scale, base=view, out=view)
    assert out is view and torch.equal(view, want)
    assert (wide[:, :shift] == 3.0).all() and (wide[:, shift + N:] == 3.0).all() and (wide[T] == 3.0).all()
    other = torch.full((T, 2 * N + 32), 5.0, dtype=dtype, device="cuda")
    other[:, :N] = y
    B.exmoe_lora(plan, x, a, b, scale, base=other[:, :N], out=other[:, N + 16:2 * N + 16])
    assert torch.equal(other[:, N + 16:2 * N + 16], want) and torch.equal(other[:, :N], y) and (other[:, N:N + 16] == 5.0).all() and (other[:, 2 * N + 16:] == 5.0).all()


def test_no_adapters_one_adapter_and_bad_ids(B):
    for T in (1, 64, 65, 300):
        n, r, K, N = 4, 8, 128, 96
        for ids in (torch.full((T,), -1), torch.full((T,), 2), torch.arange(T) % 6 - 1, torch.tensor([-2, 4, 1 << 30, -(1 << 31), 0, 3]).repeat(T)[:T]):
            x, a, b, scale, ids, y = inputs(T, n, r, K, N, 9, ids=ids)
            plan = B.exmoe_lora_plan(ids, n)
            check(B.exmoe_lora(plan, x, a, b, scale, base=y), x, a, b, scale, ids, y)
            check(B.exmoe_lora(plan, x, a, b, scale), x, a, b, scale, ids, None)
            bad = bool(((ids < -1) | (ids >= n)).any())
            assert B.exmoe_lora_plan_status(plan) == (B.EXMOE_ERR_BAD_ADAPTER_ID if bad else B.EXMOE_OK)


def test_infinities_stay_in_their_rows(B):
    x, a, b, scale, ids, y = inputs(100, 4, 16, 256, 128, 3)
    want = B.exmoe_lora(B.exmoe_lora_plan(ids, 4), x, a, b, scale, base=y)
    rows = [3, 17, 64]
    x[3, 5], x[17, 0] = float("inf"), float("nan")
    y[64, 2] = float("-inf")
    out = B.exmoe_lora(B.exmoe_lora_plan(ids, 4), x, a, b, scale, base=y)
    keep = [t for t in range(100) if t not in rows]
    assert torch.equal(out[keep], want[keep])
    for t in rows[:2]:
        assert ids[t] < 0 or not torch.isfinite(out[t]).any()
    assert out[64, 2] == float("-inf") and torch.equal(out[64, 3:], want[64, 3:])


def test_plan_of_many_tokens_and_adapters(B):
    for T, n in ((20000, 1024), (5000, 1000), (40000, 3)):
        x, a, b, scale, ids, y = inputs(T, n, 8, 64, 40, 13)
        out = B.exmoe_lora(B.exmoe_lora_plan(ids, n), x, a, b, scale, base=y)
        rows = list(range(0, T, 37)) + list(range(T - 70, T))
        check(out, x, a, b, scale, ids, y, rows)


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 1023, 1024])
@pytest.mark.parametrize("T", [1, 33, 1023, 1025, 8193])
def test_plan_at_its_edges(B, T, n):
    """Steps of 32 tokens, 32 warps, 1024 threads and the steps kept in registers, each with one more and one less; ids in any order and in runs."""
    x, a, b, scale, ids, y = inputs(T, n, 8, 64, 40, 3 * n + T)
    for order in (ids, ids.sort().values):
        plan = B.exmoe_lora_plan(order, n)
        check(B.exmoe_lora(plan, x, a, b, scale, base=y), x, a, b, scale, order, y, sorted({*range(0, T, max(1, T // 40)), T - 1}))
        assert B.exmoe_lora_plan_status(plan) == B.EXMOE_OK


def test_a_plan_serves_its_own_sizes_only(B):
    x, a, b, scale, ids, y = inputs(10, 4, 8, 64, 32, 1)
    plan = B.exmoe_lora_plan(ids, 4)
    with pytest.raises(ValueError, match="plan"):
        B.exmoe_lora(plan, x[:9], a, b, scale, base=y[:9])
    other = torch.zeros_like(plan)                                         # never planned: nothing is written, and it says so
    out = torch.full_like(y, 2.0)
    B.exmoe_lora(other, x, a, b, scale, base=y, out=out)
    assert (out == 2.0).all() and B.exmoe_lora_plan_status(other) == B.EXMOE_ERR_STATE
    assert B.exmoe_lora_plan(ids, 4, plan=other) is other
    check(B.exmoe_lora(other, x, a, b, scale, base=y), x, a, b, scale, ids, y)
    empty = B.exmoe_lora_plan(ids[:0], 4)
    assert B.exmoe_lora(empty, x[:0], a, b, scale).shape == (0, 32) and B.exmoe_lora_plan_status(empty) == B.EXMOE_OK


def test_status_of_what_is_no_plan_is_refused(B):
    with pytest.raises(ValueError, match="plan"):
        B.exmoe_lora_plan_status(torch.zeros(15, dtype=torch.int32, device="cuda"))


def test_refusals(B):
    x, a, b, scale, ids, y = inputs(10, 4, 8, 64, 32, 1)
    plan = B.exmoe_lora_plan(ids, 4)
    good = dict(plan=plan, x=x, a=a, b=b, scale=scale, base=y)
    for bad in (dict(x=x.float()), dict(x=x.t()), dict(a=a[:, :, :56].contiguous()), dict(b=b[:3]), dict(scale=scale[:3]), dict(scale=scale.double()), dict(base=y[:9]),
                dict(base=y.half()), dict(out=y[:, :31]), dict(out=torch.empty((10, 32), device="cuda")), dict(out_dtype=torch.float32), dict(base=None, out_dtype=torch.float16)):
        with pytest.raises(ValueError):
            B.exmoe_lora(**{**good, **bad})
    with pytest.raises(B.ExmoeError) as ei:
        B.exmoe_lora(plan, x, a[:, :4].contiguous(), b[:, :, :4].contiguous(), scale)
    assert ei.value.code == B.EXMOE_ERR_SHAPE
    with pytest.raises(B.ExmoeError) as ei:                                # rows that start off a 16-byte boundary
        B.exmoe_lora(plan, torch.zeros((10, 68), dtype=torch.bfloat16, device="cuda")[:, :64], a, b, scale)
    assert ei.value.code == B.EXMOE_ERR_ARG
    square = normal(torch.Generator().manual_seed(1), 1.0, 4, 64, 8).cuda()
    with pytest.raises(B.ExmoeError) as ei:                                # out may not be x
        B.exmoe_lora(plan, x, a, square, scale, out=x)
    assert ei.value.code == B.EXMOE_ERR_ARG


@pytest.mark.parametrize("T", [1, 40, 500])
def test_streams_graphs_and_one_plan_for_many_layers(B, T):
    n, r, K, N = 5, 16, 512, 320
    sets = [inputs(T, n, r, K, N, 40 + i) for i in range(3)]
    ids = sets[0][4]
    plan = B.exmoe_lora_plan(ids, n)
    want = [B.exmoe_lora(plan, x, a, b, s, base=y) for x, a, b, s, _, y in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    got = []
    for st, (x, a, b, s, _, y) in zip(streams, sets):                      # a plan is only read: calls may overlap
        st.wait_stream(torch.cuda.current_stream())
        got.append(B.exmoe_lora(plan, x, a, b, s, base=y, stream=st))
    torch.cuda.synchronize()
    for u, v in zip(want, got):
        assert torch.equal(u, v)
    static, graph = ids.clone(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p = B.exmoe_lora_plan(static, n)
        outs = [B.exmoe_lora(p, x, a, b, s, base=y) for x, a, b, s, _, y in sets]
    for new in (ids, sets[1][4], torch.full_like(ids, -1), sets[2][4]):
        static.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        for o, (x, a, b, s, _, y) in zip(outs, sets):
            check(o, x, a, b, s, new, y, list(range(0, T, 1 + T // 50)))


def test_adapters_beside_the_router_and_the_block(B):
    """A step as a serving program makes it: corrections of the router's logits, the gate, the experts, corrections of the block's output."""
    shape, T, n = synth.MID, 30, 4
    ora, bank = helpers.make_layer(shape, seed=77)
    g = torch.Generator().manual_seed(2)
    hidden, w = synth.hidden_states(shape, T, 3), synth.router_weights(shape, 4)
    E, H = shape.num_experts, shape.d_model
    ids = torch.randint(-1, n, (T,), generator=g).int()
    ar, br, ab, bb = normal(g, 0.05, n, 8, H), normal(g, 0.05, n, E, 8), normal(g, 0.02, n, 16, H), normal(g, 0.02, n, H, 16)
    scale = torch.rand(n, generator=g) + 1
    gate = B.Gate(score="sigmoid", num_groups=4, top_groups=2, group_score="top2", renormalise=True)
    cache = B.Cache(shape, [bank], E, max_tokens=T)
    h, graph = hidden.cuda(), torch.cuda.CUDAGraph()
    dev = [v.cuda() for v in (ids, ar, br, ab, bb, scale, w)]

    def step():
        i, ar, br, ab, bb, s, w = dev
        plan = B.exmoe_lora_plan(i, n)
        top, p = B.exmoe_route_gated(shape, gate, h, w, addend=B.exmoe_lora(plan, h, ar, br, s, out_dtype=torch.float32))
        y = cache.forward(0, h, top, p)
        return top, p, y, B.exmoe_lora(plan, h, ab, bb, s, base=y)
    eager = step()
    with torch.cuda.graph(graph):
        captured = step()
    graph.replay()
    torch.cuda.synchronize()
    for u, v in zip(eager, captured):
        assert torch.equal(u, v)
    top, p, y, out = eager
    add = olora.apply(num(hidden), num(ar), num(br), num(scale), ids.numpy())
    want, weights = ogate.choose(ogate.logits(num(hidden), num(w), None, add), gate, shape.top_k)
    assert np.array_equal(top.cpu().numpy(), want)
    np.testing.assert_allclose(p.cpu().numpy(), weights, rtol=1e-4)
    ref, rounded = ora.forward(hidden, top.cpu(), p.cpu())
    helpers.check_output(y, ref, rounded, "block")
    check(out, h, dev[3], dev[4], dev[5], dev[0], y)
    cache.close()
