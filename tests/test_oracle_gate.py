"""The gate's and the adapters' oracles against closed forms, brute force and torch."""
import itertools
import math
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from oracle import gate as ogate
from oracle import lora as olora
from oracle import router as orouter


def gate(**k):
    return SimpleNamespace(**{**dict(score="softmax", num_groups=1, top_groups=1, group_score="max", renormalise=False, scale=1.0), **k})


def test_softmax_without_anything_is_the_router():
    rng = np.random.default_rng(0)
    h, w = rng.normal(size=(5, 32)), rng.normal(size=(12, 32))
    ids, p, z = orouter.route(h, w, 4)
    got, weights = ogate.choose(ogate.logits(h, w), gate(), 4)
    assert np.array_equal(got, ids)
    np.testing.assert_allclose(weights, p, rtol=1e-12)


def test_closed_forms():
    z = np.log([1.0, 2.0, 3.0, 4.0])
    ids, w = ogate.choose_token(z, gate(renormalise=True, scale=2.5), 2)
    assert ids.tolist() == [3, 2]
    np.testing.assert_allclose(w, [2.5 * 4 / 7, 2.5 * 3 / 7])
    ids, w = ogate.choose_token(z, gate(score="sigmoid"), 2)              # 1 / (1 + 1 / v)
    np.testing.assert_allclose(w, [4 / 5, 3 / 4])
    ids, w = ogate.choose_token(z, gate(score="sigmoid"), 2, balance=[1.0, 0.0, 0.0, 0.0])
    assert ids.tolist() == [0, 3]                                         # 1/2 + 1, 4/5
    np.testing.assert_allclose(w, [1 / 2, 4 / 5])                         # the bias enters no weight


def test_groups():
    z = [3.0, 0.0, 2.0, 1.9]                                              # groups (0, 1) and (2, 3)
    assert ogate.choose_token(z, gate(num_groups=2), 2)[0].tolist() == [0, 1]
    top2 = gate(score="sigmoid", num_groups=2, group_score="top2")        # 0.95 + 0.5 against 0.88 + 0.87
    assert ogate.choose_token(z, top2, 2)[0].tolist() == [2, 3]
    one = gate(num_groups=4, top_groups=2, group_score="top2")            # groups of one expert: its own value
    assert ogate.choose_token(z, one, 2)[0].tolist() == [0, 2]
    assert ogate.choose_token([0.0] * 4, gate(num_groups=2), 1)[0].tolist() == [0]   # equal groups: the lower


def test_masks_and_nan():
    inf = -np.inf
    g = gate(num_groups=2, group_score="top2", renormalise=True)
    ids, w = ogate.choose_token([inf, 1.0, inf, inf], g, 2)
    assert ids.tolist() == [1, 0] and w.tolist() == [1.0, 0.0]            # a masked expert comes last, with weight zero
    ids, w = ogate.choose_token([inf] * 4, g, 2)
    assert ids.tolist() == [0, 1] and w.tolist() == [0.0, 0.0]
    ids, w = ogate.choose_token([math.nan, inf, 0.0, 1.0], gate(score="sigmoid"), 4, balance=[9.0, 9.0, 0.0, 0.0])
    assert ids.tolist() == [3, 2, 1, 0] and math.isnan(w[3])
    assert np.isnan(ogate.choose_token([math.nan, 0.0], gate(), 1)[1]).all()


def test_choice_maximises_over_all_subsets():
    rng = np.random.default_rng(1)
    for _ in range(50):
        z, bias = rng.normal(size=12), rng.normal(size=12) * 0.3
        g = gate(score="sigmoid", num_groups=4, top_groups=2, group_score="top2")
        ids, _ = ogate.choose_token(z, g, 3, bias)
        c = ogate.scores(z, "sigmoid") + bias
        value = [sum(sorted(c[3 * i:3 * i + 3])[-2:]) for i in range(4)]
        groups = max(itertools.combinations(range(4), 2), key=lambda p: sum(value[i] for i in p))
        allowed = [e for e in range(12) if e // 3 in groups]
        best = max(itertools.combinations(allowed, 3), key=lambda p: sum(c[list(p)]))
        assert sorted(ids.tolist()) == sorted(best)


def test_adapters_against_torch():
    g = torch.Generator().manual_seed(3)
    x, a, b = (torch.randn(*s, generator=g, dtype=torch.float64) for s in ((6, 16), (3, 8, 16), (3, 10, 8)))
    scale, ids, base = torch.tensor([1.0, 2.0, -0.5], dtype=torch.float64), torch.tensor([0, 2, -1, 1, 7, 0]), torch.randn(6, 10, generator=g, dtype=torch.float64)
    want = base.clone()
    for i in range(3):
        rows = ids == i
        want[rows] += scale[i] * torch.nn.functional.linear(torch.nn.functional.linear(x[rows], a[i]), b[i])
    np.testing.assert_allclose(olora.apply(x.numpy(), a.numpy(), b.numpy(), scale.numpy(), ids.numpy(), base.numpy()), want.numpy(), rtol=1e-12, atol=1e-12)
    assert olora.groups(ids.numpy(), 3) == [(0, [0, 5]), (1, [3]), (2, [1]), (-1, [2, 4])]


@pytest.fixture(scope="module")
def B():
    from paper_2608_15383_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def test_gate_refusals(B):
    """Everything that is refused is refused before a device is touched."""
    from ctypes import byref
    L, p = B.lib(), 1 << 20                                               # an aligned address that is never used

    def route(shape=(64, 128, 8, 2, 128), g=(0, 1, 1, 0, 0, 1.0), hidden=p, T=1):
        return L.exmoe_route_gated(byref(B.exmoe_shape(*shape)), byref(B.exmoe_gate(*g)), hidden, p, None, None, None, T, p, p, None)
    assert route(T=0) == B.EXMOE_OK
    assert route(T=-1) == B.EXMOE_ERR_ARG
    for g in ((2, 1, 1, 0, 0, 1.0), (0, 1, 1, 2, 0, 1.0), (0, 1, 1, 0, 2, 1.0)):
        assert route(g=g) == B.EXMOE_ERR_ARG, g
    for g in ((0, 3, 1, 0, 0, 1.0), (0, 0, 1, 0, 0, 1.0), (0, 2, 3, 0, 0, 1.0), (0, 2, 0, 0, 0, 1.0), (0, 8, 1, 0, 0, 1.0)):
        assert route(g=g) == B.EXMOE_ERR_SHAPE, g                         # the last: top_k 2 of one group of one expert
    assert route((64, 128, 64, 2, 128), (0, 64, 32, 0, 0, 1.0)) == B.EXMOE_ERR_SHAPE            # more than 32 groups
    for shape in ((60, 128, 8, 2, 128), (0, 128, 8, 2, 128), (64, 128, 0, 1, 128), (64, 128, 4097, 2, 128), (64, 128, 8, 0, 128), (64, 128, 8, 9, 128),
                  (102400, 128, 8, 2, 128)):
        assert route(shape) == B.EXMOE_ERR_SHAPE, shape
    assert route(hidden=None) == B.EXMOE_ERR_ARG and route(hidden=p + 8) == B.EXMOE_ERR_ARG

    def logits(type=0, ld=8, T=2, at=p):
        return L.exmoe_gate_logits(byref(B.exmoe_shape(0, 0, 8, 2, 0)), byref(B.exmoe_gate(0, 1, 1, 0, 0, 1.0)), at, type, ld, None, T, p, p, None)
    assert logits(T=0) == B.EXMOE_OK
    assert logits(type=2) == logits(ld=7) == logits(ld=-8) == logits(at=None) == logits(T=-1) == B.EXMOE_ERR_ARG


def test_adapter_refusals(B):
    from ctypes import byref, c_size_t
    L, p = B.lib(), 1 << 30
    n = c_size_t()
    assert L.exmoe_lora_plan_bytes(10, 1025, byref(n)) == L.exmoe_lora_plan_bytes(10, 0, byref(n)) == B.EXMOE_ERR_SHAPE
    assert L.exmoe_lora_plan_bytes(-1, 4, byref(n)) == L.exmoe_lora_plan_bytes(1, 4, None) == B.EXMOE_ERR_ARG
    assert L.exmoe_lora_plan(None, 5, 4, p, None) == L.exmoe_lora_plan(p, 5, 4, None, None) == L.exmoe_lora_plan(p, 5, 4, p + 4, None) == B.EXMOE_ERR_ARG
    assert L.exmoe_lora_plan_status(None) == B.EXMOE_ERR_ARG

    MB = 1 << 20
    good = dict(shape=(4, 64, 32, 8), plan=p, x=p + MB, ld_x=64, a=p + 2 * MB, b=p + 3 * MB, scale=p + 4 * MB, T=16, base=p + 5 * MB, ld_base=32,
                out=p + 6 * MB, ld_out=32, type=1)

    def lora(**k):
        c = {**good, **k}
        return L.exmoe_lora(byref(B.exmoe_lora_shape(*c["shape"])), c["plan"], c["x"], c["ld_x"], c["a"], c["b"], c["scale"], c["T"], c["base"], c["ld_base"],
                            c["out"], c["ld_out"], c["type"], None)
    assert lora(T=0) == B.EXMOE_OK
    for shape in ((0, 64, 32, 8), (1025, 64, 32, 8), (4, 60, 32, 8), (4, 0, 32, 8), (4, 64, 0, 8), (4, 64, 32, 4), (4, 64, 32, 0), (4, 64, 32, 136)):
        assert lora(shape=shape) == B.EXMOE_ERR_SHAPE, shape
    for bad in (dict(T=-1), dict(type=2), dict(plan=None), dict(x=None), dict(a=None), dict(b=None), dict(scale=None), dict(out=None), dict(ld_x=56),
                dict(ld_x=68), dict(ld_out=31), dict(ld_base=31), dict(x=p + MB + 8), dict(a=p + 2 * MB + 8), dict(b=p + 3 * MB + 2), dict(plan=p + 8),
                dict(out=p + MB), dict(out=p + MB + 64 * 2 * 16 - 2), dict(out=p + 2 * MB), dict(out=p + 3 * MB), dict(out=p + 4 * MB), dict(out=p),
                dict(out=p + 5 * MB + 2), dict(out=p + 5 * MB, ld_out=40)):
        assert lora(**bad) == B.EXMOE_ERR_ARG, bad
    # column ranges of the same wider rows overlap where they share a column
    for shift in (-33 * 2, -2, 2, 62 * 2):
        assert lora(base=p + 5 * MB + 128, ld_base=64, out=p + 5 * MB + 128 + shift, ld_out=64, shape=(4, 64, 34, 8)) == B.EXMOE_ERR_ARG, shift


def test_sizes_beyond_32_bits_are_refused(B):
    """Row and column counts whose rounding up or grid would pass 32 bits; nothing is read."""
    from ctypes import byref, c_size_t
    L, p, many = B.lib(), 1 << 30, (1 << 29) + 1
    gate = byref(B.exmoe_gate(0, 1, 1, 0, 0, 1.0))
    assert L.exmoe_route_gated(byref(B.exmoe_shape(8, 128, 8, 2, 128)), gate, p, p, None, None, None, many, p, p, None) == B.EXMOE_ERR_ARG
    assert L.exmoe_gate_logits(byref(B.exmoe_shape(0, 0, 8, 2, 0)), gate, p, 0, 8, None, many, p, p, None) == B.EXMOE_ERR_ARG
    n = c_size_t()
    assert L.exmoe_lora_plan_bytes(many, 4, byref(n)) == L.exmoe_lora_plan(p, many, 4, p, None) == B.EXMOE_ERR_ARG
    assert L.exmoe_lora_plan_bytes(many - 1, 1024, byref(n)) == B.EXMOE_OK and n.value == 4 * (16 + 4 * ((many - 1) // 64 + 1025) + many - 1)
    for shape, T, want in (((1, 8, 8, 8), many, B.EXMOE_ERR_ARG), ((1, (1 << 30) + 8, 8, 8), 1, B.EXMOE_ERR_SHAPE), ((1, 8, (1 << 30) + 1, 8), 1, B.EXMOE_ERR_SHAPE)):
        ld = max(shape[1:3])
        assert L.exmoe_lora(byref(B.exmoe_lora_shape(*shape)), p, p, ld, p, p, p, T, None, 0, p + (1 << 40), ld, 1, None) == want, shape


def test_binding_refuses_host_tensors(B):
    z = torch.zeros((2, 8))
    shape, g = SimpleNamespace(d_model=64, d_ff=128, num_experts=8, top_k=2), B.Gate()
    with pytest.raises(ValueError, match="logits"):
        B.exmoe_gate_logits(shape, g, z)
    with pytest.raises(ValueError, match="hidden"):
        B.exmoe_route_gated(shape, g, z, z)
    with pytest.raises(ValueError, match="softmax"):
        B.exmoe_gate_logits(shape, B.Gate(score="tanh"), z)
    with pytest.raises(ValueError, match="adapter_ids"):
        B.exmoe_lora_plan(torch.zeros(4, dtype=torch.int32), 4)
    with pytest.raises(ValueError, match="plan"):
        B.exmoe_lora(torch.zeros(4, dtype=torch.int32), z, z, z, z)
