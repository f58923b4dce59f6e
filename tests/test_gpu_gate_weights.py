"""Weights of the gate from hidden states of N(0, 1) and routers of N(0, 0.02): as close to the binary64 oracle as the forms' sums are for such inputs.

A logit's partial sums are normal variables of at most its own deviation, s = 0.02 sqrt(H), and roundings have signs of their own, so that errors add up in squares; six
deviations are allowed (1e-9 for a comparison).  Few tokens: 10 + H / 256 additions of 2^-24 each.  Tensor cores: 10.5 units of 2^-24 for each of a chain's 8 MMAs (these may
all have one sign) of what 128 products come to, 0.02 sqrt(128), in H / 128 chains.  More than 512 experts: binary64.  A weight is off by twice a logit's error relative to
itself, renormalised or not, and by 28 roundings: 25 of a sum of exponentials, its own, the quotient and the scale.
"""
import math
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from oracle import gate as ogate

pytestmark = pytest.mark.gpu
UNIT = 2.0 ** -24


@pytest.fixture(scope="module")
def B():
    from paper_2608_15383_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def logit_error(T, H, E):
    if E > 512:
        return 0.0
    few = math.sqrt(10 + H / 256) * 0.02 * math.sqrt(H)
    many = math.sqrt(H / 128) * 8 * 10.5 * 0.02 * math.sqrt(128)
    return 6 * UNIT * (few if T <= 40 or E > 256 else few + many)


@pytest.mark.parametrize("H,E,k,T", [(2048, 64, 8, 1), (2048, 64, 8, 40), (2048, 60, 4, 700), (4096, 256, 8, 16), (4096, 256, 8, 400), (1024, 128, 6, 500), (2048, 384, 8, 60),
                                     (1024, 600, 8, 9)])
@pytest.mark.parametrize("kw", [dict(), dict(renormalise=True, scale=2.5), dict(score="sigmoid"), dict(score="sigmoid", num_groups=4, top_groups=2, group_score="top2", renormalise=True)])
def test_weights(B, H, E, k, T, kw):
    g = torch.Generator().manual_seed(H + E + T)
    hidden, w = torch.randn(T, H, generator=g).to(torch.bfloat16), (torch.randn(E, H, generator=g) * 0.02).to(torch.bfloat16)
    gate = B.Gate(**kw)
    ids, weights = B.exmoe_route_gated(SimpleNamespace(d_model=H, num_experts=E, top_k=k), gate, hidden.cuda(), w.cuda())
    ref, ref_w = ogate.choose(ogate.logits(hidden.double().numpy(), w.double().numpy()), gate, k)
    assert np.array_equal(ids.cpu().numpy(), ref)
    np.testing.assert_allclose(weights.cpu().numpy(), ref_w, rtol=2 * logit_error(T, H, E) + 28 * UNIT)


@pytest.mark.parametrize("E,k", [(8, 8), (40, 5), (100, 9), (256, 32), (500, 16)])
def test_sigmoids_below_binary32_are_renormalised(B, E, k):
    """Sigmoids that binary32 holds as subnormal numbers or as 0 have weights relative to the largest of them.  Exponentials (2^-22 each), a sum of 32 and a quotient in binary32,
    or all in binary64: below 48 units."""
    g = torch.Generator().manual_seed(E)
    z = torch.stack([-low - torch.rand(E, generator=g) * span for low in (0.0, 10.0, 17.0, 19.0, 40.0, 62.0, 85.0, 95.0, 150.0, 600.0) for span in (1.0, 30.0, 80.0)])
    for dtype in (torch.float32, torch.bfloat16):
        for kw in (dict(), dict(num_groups=2 if E % 2 == 0 and 2 * k <= E else 1)):
            gate = B.Gate(score="sigmoid", renormalise=True, scale=2.5, **kw)
            ids, w = B.exmoe_gate_logits(SimpleNamespace(num_experts=E, top_k=k), gate, z.to(dtype).cuda())
            ref, ref_w = ogate.choose(z.to(dtype).double().numpy(), gate, k)
            assert np.array_equal(ids.cpu().numpy(), ref)
            np.testing.assert_allclose(w.cpu().numpy(), ref_w, rtol=48 * UNIT, atol=1e-30)
