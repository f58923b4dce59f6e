"""The activations by themselves: x = 0, so that the argument is the bias, exactly, and binary32 results.  Bounds in units u = 2^-23 of binary32's last place:

silu       exp(-v) is off by (2 + 1.173 |v|) u of itself (the instruction's bound), the sum by half, the quotient by 2.  Below 2^-126 it is lost: |v| exp(v) 2 at most
           from -87 on, 2^-118.
gelu_tanh  y = sqrt(2 / pi) (v + 0.044715 v^3) is off by 3 u of itself (five roundings and two constants'), which exp(-2 y) sees 2 |y| times; then as silu with 2 y.
gelu       |v| Phi(-|v|), Phi by a polynomial f(t) that is off by 7.5e-8 at most (Abramowitz and Stegun, 7.1.26), t = 1 / (1 + p |v|) off by 3.5 u of itself (the
           denominator's two roundings and the quotient's two units) and f by 4 u besides (five steps and five constants), half of both times exp(-v^2 / 2); that
           off by (2 + 1.173 v^2 / 2) u and by the argument's rounding, v^2 / 2 half u.  That is a bound on Phi, not relative to it: far below 0 what is left is 7.5e-8 |v|.
And the products and sums at the end, 2 u of the value.
"""
import numpy as np
import pytest
import torch

from oracle import linear as olinear

pytestmark = pytest.mark.gpu
U = 2.0 ** -23


@pytest.fixture(scope="module")
def B():
    from paper_2608_15383_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def bound(v, act):
    a = np.abs(v)
    size = np.abs(olinear.activate(v, act))
    if act == "silu":
        return (2 + 1.173 * a + 0.5 + 2 + 2) * U * size + 2.0 ** -118
    if act == "gelu_tanh":
        y = np.abs(np.sqrt(2 / np.pi) * (v + 0.044715 * v ** 3))
        # the last term is the oracle's: its tanh is half a unit of 2^-53 off near -1, and the 1 that it is added to leaves nothing else (0.5 v of two such halves)
        return (2 + (2 * 1.173 + 2 * 3) * y + 0.5 + 2 + 2) * U * size + 2.0 ** -100 + a * 2.0 ** -53
    if act == "gelu":
        t = 1 / (1 + 0.3275911 * a / np.sqrt(2))
        coefficients = (0.254829592, -0.284496736, 1.421413741, -1.453152027, 1.061405429)
        f = sum(c * t ** (i + 1) for i, c in enumerate(coefficients))
        slope = sum((i + 1) * c * t ** (i + 1) for i, c in enumerate(coefficients))      # t f'(t)
        e = np.exp(-v * v / 2)
        return a * (7.5e-8 + 0.5 * e * (3.5 * np.abs(slope) + 4 + (2 + 1.673 * v * v / 2) * f) * U) + 2 * U * (size + a * 0.5 * e * f) + 2.0 ** -100
    return np.zeros_like(v)


@pytest.mark.parametrize("T", [1, 16, 40, 3000])                           # few tokens, clusters, pairs
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("gated", [False, True])
def test_arguments_that_are_exact(B, T, act, gated):
    g = torch.Generator().manual_seed(T)
    v = torch.cat([torch.linspace(-12, 12, 3001), torch.linspace(-130, 130, 521), torch.randn(500, generator=g) * 1e-3, torch.tensor([0.0, -0.0, 1e-30, -1e-30, 1e30, -1e4])])
    N = len(v)
    x, w = torch.zeros(T, 8, dtype=torch.bfloat16, device="cuda"), torch.randn(N, 8, generator=g).bfloat16().cuda()
    up = torch.full((N,), 1.5)
    out = B.exmoe_linear(x, w, v.cuda(), w_up=w if gated else None, bias_up=up.cuda() if gated else None, activation=act, out_dtype=torch.float32)
    assert torch.equal(out, out[:1].expand(T, N))
    v = v.double().numpy()
    with np.errstate(over="ignore"):
        want, tol = olinear.activate(v, act), bound(v, act)
    if gated:
        want, tol = 1.5 * want, 1.5 * tol + 2.0 ** -24 * np.abs(1.5 * want)
    err = np.abs(out[0].double().cpu().numpy() - want)
    at = np.argmax(err - tol)
    assert (err <= tol).all(), (v[at], err[at], tol[at])
