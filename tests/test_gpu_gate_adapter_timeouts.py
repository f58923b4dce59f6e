"""Waits of the gate's and the adapters' kernels that run out: the kernel returns, says so, and the next call is right.

No fault is caused: a barrier asks for an arrival that nobody makes, with a budget of about a millisecond."""
from ctypes import byref

import numpy as np
import pytest
import torch

from oracle import gate as ogate
from oracle import lora as olora
from paper_2608_15383_b200 import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2608_15383_b200 import binding, build
    build.build()
    binding.lib()
    return binding


@pytest.mark.parametrize("T,H,E", [(300, 1024, 16), (130, 4096, 64), (3000, 2048, 40)])
def test_gate(B, T, H, E):
    s = synth.Shape(H, 128, E, 4)
    hidden, w = synth.hidden_states(s, T, 1), synth.router_weights(s, 2)
    x, r = hidden.cuda(), w.cuda()
    ids, weights = torch.empty((T, 4), dtype=torch.int32, device="cuda"), torch.empty((T, 4), device="cuda")
    c = B.exmoe_shape(H, 128, E, 4, 128)
    assert B.exmoe_gate_status() == B.EXMOE_OK
    rc = B.lib().exmoe_debug_gate_timeout(byref(c), byref(B.exmoe_gate(0, 1, 1, 0, 0, 1.0)), x.data_ptr(), r.data_ptr(), T, ids.data_ptr(), weights.data_ptr(),
                                          torch.cuda.current_stream().cuda_stream)
    assert rc == B.EXMOE_OK
    assert B.exmoe_gate_status() == B.EXMOE_ERR_TIMEOUT                    # reported once, and cleared
    assert B.exmoe_gate_status() == B.EXMOE_OK
    got, _ = B.exmoe_route_gated(s, B.Gate(), x, r)
    ref, _ = ogate.choose(ogate.logits(hidden.double().numpy(), w.double().numpy()), B.Gate(), 4)
    assert np.array_equal(got.cpu().numpy(), ref) and B.exmoe_gate_status() == B.EXMOE_OK


@pytest.mark.parametrize("T,r", [(5, 16), (5, 64), (40, 8), (100, 40)])    # parts of v in one hop, and in two
def test_adapters(B, T, r):
    n, K, N = 2, 512, 640
    g = torch.Generator().manual_seed(T)
    x, a, b = (torch.randn(*size, generator=g).to(torch.bfloat16).cuda() for size in ((T, K), (n, r, K), (n, N, r)))
    scale, ids = torch.ones(n, device="cuda"), (torch.arange(T) % 3 - 1).int().cuda()
    plan = B.exmoe_lora_plan(ids, n)
    want = B.exmoe_lora(plan, x, a, b, scale)
    wide = torch.full((T + 2, N), 7.0, dtype=torch.bfloat16, device="cuda")
    out = wide[1:T + 1]
    rc = B.lib().exmoe_debug_lora_timeout(byref(B.exmoe_lora_shape(n, K, N, r)), plan.data_ptr(), x.data_ptr(), a.data_ptr(), b.data_ptr(), scale.data_ptr(), T,
                                          out.data_ptr(), torch.cuda.current_stream().cuda_stream)
    assert rc == B.EXMOE_OK
    assert B.exmoe_lora_plan_status(plan) == B.EXMOE_ERR_TIMEOUT
    left = out == 7.0
    assert left[ids >= 0].any() and torch.equal(out[~left], want[~left])   # an output is right or left as it was
    assert (wide[[0, T + 1]] == 7.0).all()
    assert B.exmoe_lora_plan(ids, n, plan=plan) is plan and B.exmoe_lora_plan_status(plan) == B.EXMOE_OK
    assert torch.equal(B.exmoe_lora(plan, x, a, b, scale), want) and B.exmoe_lora_plan_status(plan) == B.EXMOE_OK
    ref = olora.apply(*(v.double().cpu().numpy() for v in (x, a, b, scale)), ids.cpu().numpy())
    assert np.abs(want.double().cpu().numpy() - ref).max() <= 2.0 ** -7 * np.abs(ref).max()


def test_refusals(B):
    p, f = 1 << 30, B.lib().exmoe_debug_lora_timeout
    assert f(byref(B.exmoe_lora_shape(2, 64, 64, 72)), p, p << 1, p << 2, p << 3, p << 4, 5, p << 5, None) == B.EXMOE_ERR_SHAPE
    assert f(byref(B.exmoe_lora_shape(2, 64, 64, 8)), p, p << 1, p << 2, p << 3, p << 4, 0, p << 5, None) == B.EXMOE_ERR_ARG
    f, gate = B.lib().exmoe_debug_gate_timeout, byref(B.exmoe_gate(0, 1, 1, 0, 0, 1.0))
    assert f(byref(B.exmoe_shape(512, 128, 16, 4, 128)), gate, p, p << 1, 300, p << 2, p << 3, None) == B.EXMOE_ERR_SHAPE
    assert f(byref(B.exmoe_shape(1024, 128, 65, 4, 128)), gate, p, p << 1, 300, p << 2, p << 3, None) == B.EXMOE_ERR_SHAPE
    assert f(byref(B.exmoe_shape(1024, 128, 16, 4, 128)), gate, p, p << 1, 0, p << 2, p << 3, None) == B.EXMOE_ERR_ARG
