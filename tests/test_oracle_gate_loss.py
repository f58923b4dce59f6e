"""The oracles of the gate's losses and gradients and of the products with an epilogue: closed forms, differences, torch; and what the entry
points refuse before they touch a device."""
import itertools
import math
from ctypes import byref, c_size_t
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from oracle import gate as ogate
from oracle import gate_loss as oloss
from oracle import linear as olinear


def gate(**k):
    return SimpleNamespace(**{**dict(score="softmax", num_groups=1, top_groups=1, group_score="max", renormalise=False, scale=1.0), **k})


def test_an_even_load_has_loss_one():
    """Scores of 1 / E and every expert chosen equally often: E / (k T^2) * E * (k T / E) * (T / E) = 1."""
    E, k, T = 8, 2, 12
    ids = np.arange(T * k).reshape(T, k) % E
    for score in ("softmax", "sigmoid"):
        losses, counts, sums, kept = oloss.balance(np.full((T, E), 0.7), ids, gate(score=score))
        np.testing.assert_allclose(losses, [1.0, (0.7 + math.log(E)) ** 2])
        assert (counts == 3).all() and kept.tolist() == [T]
        np.testing.assert_allclose(sums, np.full((1, E), T / E))


def test_all_on_one_expert():
    E, T = 4, 5
    z = np.full((T, E), -np.inf)
    z[:, 2] = 3.0
    losses, counts, sums, _ = oloss.balance(z, np.full((T, 1), 2), gate())
    np.testing.assert_allclose(losses, [E, 9.0])
    assert counts.tolist() == [[0, 0, T, 0]] and sums.tolist() == [[0, 0, T, 0]]


def test_sequences_masks_and_rows_without_experts():
    rng = np.random.default_rng(0)
    z, ids = rng.normal(size=(9, 5)), rng.integers(0, 5, (9, 2))
    z[4] = -np.inf
    ids[3, 1] = 7                                                          # not counted
    mask = np.array([1, 1, 0, 1, 1, 1, 1, 0, 1], bool)
    losses, counts, sums, kept = oloss.balance(z, ids, gate(), mask, [0, 2, 2, 7, 8])
    assert kept.tolist() == [2, 0, 4, 0] and counts.sum(1).tolist() == [4, 0, 7, 0]
    np.testing.assert_allclose(sums.sum(1), [2, 0, 3, 0])
    a = oloss.balance(z[:2], ids[:2], gate())[0]
    b = oloss.balance(z[[3, 4, 5, 6]], ids[[3, 4, 5, 6]], gate())[0]
    np.testing.assert_allclose(losses, [(a[0] + b[0]) / 2, (2 * a[1] + 4 * b[1]) / 6])
    assert oloss.balance(z, ids, gate(), np.zeros(9, bool))[0].tolist() == [0.0, 0.0]


@pytest.mark.parametrize("score,renormalise", list(itertools.product(("softmax", "sigmoid"), (False, True))))
def test_gradient_against_differences(score, renormalise):
    rng = np.random.default_rng(1)
    T, E, k = 7, 6, 3
    g = gate(score=score, renormalise=renormalise, scale=2.5)
    z = rng.normal(size=(T, E)) * 2
    z[0, 2] = z[3, 5] = -np.inf
    z[6] = -np.inf
    ids = np.stack([rng.permutation(E)[:k] for _ in range(T)])
    ids[1, 0] = E + 3                                                      # has no weight
    ids[2] = [4, 4, 1]                                                     # twice
    mask, offsets = np.array([1, 1, 1, 0, 1, 1, 1], bool), [0, 3, 3, 6]
    dw, dl = rng.normal(size=(T, k)), np.array([0.7, 0.3])
    _, counts, _, kept = oloss.balance(z, ids, g, mask, offsets)

    def value(z):
        w = sum((dw[t] * oloss.weights(z[t], ids[t], g)).sum() for t in range(T) if mask[t])
        sums = np.stack([sum([oloss.shares(z[t], score == "sigmoid") for t in range(a, b) if mask[t]], np.zeros(E)) for a, b in oloss.sequences(T, offsets)])
        some = kept > 0
        bal = np.mean(E / (k * kept[some].astype(float) ** 2) * (counts * sums)[some].sum(1))
        sq = np.mean([oloss.log_sum(z[t]) ** 2 for t in range(6) if mask[t]])
        return w + dl[0] * bal + dl[1] * sq
    got, size = oloss.backward(z, ids, g, k, dw, dl, counts, kept, mask, offsets)
    assert (np.abs(got) <= size * (1 + 1e-12) + 1e-300).all() and (got[3] == 0).all() and (got[6] == 0).all()
    h = 1e-5
    for t, e in itertools.product(range(T), range(E)):
        if not np.isneginf(z[t, e]):
            up, dn = z.copy(), z.copy()
            up[t, e] += h
            dn[t, e] -= h
            # the second-order term of the difference: h^2 / 6 of a third derivative, below 10 here
            np.testing.assert_allclose(got[t, e], (value(up) - value(dn)) / (2 * h), atol=10 * h * h + 1e-10)
        else:
            assert got[t, e] == 0


def test_weights_are_the_gates():
    rng = np.random.default_rng(2)
    for score, renormalise in itertools.product(("softmax", "sigmoid"), (False, True)):
        g = gate(score=score, renormalise=renormalise, scale=1.5)
        z = rng.normal(size=8)
        ids, w = ogate.choose_token(z, g, 3)
        np.testing.assert_allclose(oloss.weights(z, np.asarray(ids), g), w, rtol=1e-12)
    g = gate(score="sigmoid", renormalise=True)                            # sigmoids that binary64 loses keep their shares
    np.testing.assert_allclose(oloss.weights(np.array([-1000.0, -1001.0, 5.0]), np.array([0, 1]), g), [1 / (1 + math.exp(-1)), 1 / (1 + math.exp(1))])


@pytest.mark.parametrize("activation", ["none", "relu", "gelu", "gelu_tanh", "silu"])
def test_products(activation):
    g = torch.Generator().manual_seed(3)
    x, w, u, r = (torch.randn(*s, generator=g, dtype=torch.float64) for s in ((5, 16), (7, 16), (7, 16), (5, 7)))
    b, bu = (torch.randn(7, generator=g, dtype=torch.float64) for _ in range(2))
    f = {"none": lambda v: v, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu,
         "gelu_tanh": lambda v: torch.nn.functional.gelu(v, approximate="tanh")}[activation]
    np.testing.assert_allclose(olinear.apply(x, w, b, activation=activation), f(x @ w.T + b), rtol=1e-12, atol=1e-14)
    np.testing.assert_allclose(olinear.apply(x, w, None, u, bu, activation, r), r + f(x @ w.T) * (x @ u.T + bu), rtol=1e-12, atol=1e-14)
    assert (olinear.magnitude(x, w, b) >= np.abs(olinear.apply(x, w, b)) - 1e-12).all()


# ---- refusals: addresses that are never used
@pytest.fixture(scope="module")
def B():
    from paper_2608_15383_b200 import binding, build
    build.build()
    binding.lib()
    return binding


P, MB = 1 << 40, 1 << 32


def linear(B, K=64, N=32, act=0, x=P, ld_x=64, w=P + MB, ld_w=64, bias=P + 2 * MB, w_up=None, ld_up=0, bias_up=None, T=16, res=P + 3 * MB, ld_res=32, out=P + 4 * MB,
           ld_out=32, type=1):
    return B.lib().exmoe_linear(byref(B.exmoe_linear_shape(K, N, act)), x, ld_x, w, ld_w, bias, w_up, ld_up, bias_up, T, res, ld_res, out, ld_out, type, None)


def test_products_refuse(B):
    A, S = B.EXMOE_ERR_ARG, B.EXMOE_ERR_SHAPE
    assert linear(B, T=0) == B.EXMOE_OK
    assert linear(B, K=60) == S and linear(B, K=0) == S and linear(B, N=0) == S and linear(B, K=-8) == S
    for bad in (dict(act=5), dict(act=-1), dict(type=2), dict(T=-1), dict(T=(1 << 29) + 1), dict(x=None), dict(w=None), dict(out=None), dict(ld_x=56), dict(ld_x=68),
                dict(ld_w=56), dict(ld_w=68), dict(ld_out=31), dict(ld_res=31), dict(bias_up=P + 5 * MB), dict(w_up=P + 5 * MB, ld_up=63),
                dict(w_up=P + 5 * MB, ld_up=56), dict(x=P + 8), dict(w=P + MB + 2), dict(w_up=P + 5 * MB + 8, ld_up=64), dict(bias=P + 2), dict(res=P + 3 * MB + 1),
                dict(out=P + 4 * MB + 1), dict(w_up=P + 5 * MB, ld_up=64, bias_up=P + 6 * MB + 1)):
        assert linear(B, **bad) == A, bad
    for off in (1, 2, 3):
        assert linear(B, type=0, out=P + 4 * MB + off) == A and linear(B, type=0, res=P + 3 * MB + off) == A


def test_products_refuse_overlap(B):
    A = B.EXMOE_ERR_ARG
    for name in ("x", "w", "bias", "res"):
        assert linear(B, **{name: P + 4 * MB + 16}) == A, name
    assert linear(B, w_up=P + 4 * MB + 16, ld_up=64) == A and linear(B, w_up=P + 7 * MB, ld_up=64, bias_up=P + 4 * MB + 16) == A
    assert linear(B, res=P + 4 * MB, ld_res=40) == A                       # in place with other rows
    assert linear(B, res=P + 4 * MB + 2, ld_res=32) == A


def loss(B, shape=(0, 0, 8, 2, 0), g=(0, 1, 1, 0, 0, 1.0), z=P, type=0, ld=8, ids=P + MB, mask=None, off=None, S=1, T=4, losses=P + 2 * MB, counts=P + 3 * MB,
         sums=P + 4 * MB, kept=P + 5 * MB, scratch=P + 6 * MB):
    return B.lib().exmoe_balance_loss(byref(B.exmoe_shape(*shape)), byref(B.exmoe_gate(*g)), z, type, ld, ids, mask, off, S, T, losses, counts, sums, kept, scratch, None)


def back(B, shape=(0, 0, 8, 2, 0), g=(0, 1, 1, 0, 0, 1.0), z=P, type=0, ld=8, ids=P + MB, dw=P + 2 * MB, dl=P + 3 * MB, counts=P + 4 * MB, kept=P + 5 * MB, mask=None,
         off=None, S=1, T=4, dz=P + 6 * MB, ld_dz=8):
    return B.lib().exmoe_gate_backward(byref(B.exmoe_shape(*shape)), byref(B.exmoe_gate(*g)), z, type, ld, ids, dw, dl, counts, kept, mask, off, S, T, dz, ld_dz, None)


def test_losses_and_gradients_refuse(B):
    A, S = B.EXMOE_ERR_ARG, B.EXMOE_ERR_SHAPE
    assert back(B, T=0) == B.EXMOE_OK
    for call in (loss, back):
        for bad in ((0, 0, 0, 2, 0), (0, 0, 4097, 2, 0), (0, 0, 8, 0, 0), (0, 0, 8, 9, 0)):
            assert call(B, shape=bad) == S, bad
        for bad in ((2, 1, 1, 0, 0, 1.0), (0, 1, 1, 2, 0, 1.0), (0, 1, 1, 0, 2, 1.0)):
            assert call(B, g=bad) == A, bad
        assert call(B, g=(0, 3, 1, 0, 0, 1.0)) == S
        for bad in (dict(type=2), dict(ld=7), dict(ld=-8), dict(T=-1), dict(T=(1 << 29) + 1), dict(S=0), dict(S=2), dict(S=-1), dict(z=None), dict(ids=None),
                    dict(counts=None), dict(kept=None), dict(z=P + 2), dict(type=1, z=P + 1), dict(ids=P + MB + 2), dict(off=P + 9 * MB + 1), dict(counts=P + 4 * MB + 2),
                    dict(kept=P + 5 * MB + 1)):
            assert call(B, **bad) == A, (call, bad)
    for bad in (dict(losses=None), dict(sums=None), dict(T=5000, scratch=None), dict(losses=P + 2 * MB + 2), dict(sums=P + 4 * MB + 1), dict(scratch=P + 6 * MB + 4)):
        assert loss(B, **bad) == A, bad
    for bad in (dict(dz=None), dict(ld_dz=7), dict(dz=P + 6 * MB + 2), dict(dw=P + 2), dict(dl=P + 3 * MB + 1)):
        assert back(B, **bad) == A, bad
    for name in ("z", "ids", "dw", "dl", "counts", "kept", "mask", "off"):
        assert back(B, **{name: P + 6 * MB + 16}) == A, name


def test_scratch(B):
    n = c_size_t()
    for T, E in ((0, 1), (1, 8), (100, 64), (100000, 256), (1 << 29, 4096)):
        assert B.lib().exmoe_balance_scratch_bytes(byref(B.exmoe_shape(0, 0, E, 1, 0)), T, byref(n)) == B.EXMOE_OK and n.value < 64 << 20 and (n.value > 0) == (T >= 100000)
    assert B.lib().exmoe_balance_scratch_bytes(byref(B.exmoe_shape(0, 0, 8, 1, 0)), -1, byref(n)) == B.EXMOE_ERR_ARG
    assert B.lib().exmoe_balance_scratch_bytes(byref(B.exmoe_shape(0, 0, 5000, 1, 0)), 4, byref(n)) == B.EXMOE_ERR_SHAPE
    assert B.lib().exmoe_balance_scratch_bytes(byref(B.exmoe_shape(0, 0, 8, 1, 0)), 4, None) == B.EXMOE_ERR_ARG


def test_python_refuses_host_tensors_and_wrong_names(B):
    s, g, z, i = SimpleNamespace(d_model=128, num_experts=8, top_k=2), gate(), torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int32)
    for call in (lambda: B.exmoe_balance_loss(s, g, z, i), lambda: B.exmoe_gate_backward(s, g, z, i)):
        with pytest.raises(ValueError, match="logits"):
            call()
    with pytest.raises(ValueError, match="x: need"):
        B.exmoe_linear(torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(4, 8, dtype=torch.bfloat16))


def test_losses_refuse_overlap(B):
    """What is written overlaps neither an input nor one another."""
    at = dict(losses=P + 10 * MB, counts=P + 11 * MB, sums=P + 12 * MB, kept=P + 13 * MB)
    inputs = dict(z=P + 14 * MB, ids=P + 15 * MB, mask=P + 16 * MB, off=P + 17 * MB)
    for name in at:
        for other, where in {**at, **inputs}.items():
            if other != name:
                assert loss(B, **{**at, **inputs, name: where}) == B.EXMOE_ERR_ARG, (name, other)
    for other in {**at, **inputs}.values():
        assert loss(B, **{**at, **inputs, "T": 5000, "scratch": other}) == B.EXMOE_ERR_ARG, other
