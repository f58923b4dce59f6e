"""Waits of exmoe_linear's tensor-core kernels that run out: the kernel returns, says so, writes nothing outside of its result, and the next call is right.

No fault is caused: a barrier asks for an arrival that nobody makes, with a budget of about a millisecond."""
from ctypes import byref

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2608_15383_b200 import binding, build
    build.build()
    binding.lib()
    return binding


@pytest.mark.parametrize("T,K,N", [(20, 1024, 200), (64, 2048, 2048), (300, 1024, 130), (1500, 1088, 1000), (5000, 1024, 2048)])     # clusters and pairs
def test_a_wait_that_runs_out(B, T, K, N):
    g = torch.Generator().manual_seed(T)
    x, w = ((torch.randn(*size, generator=g) * 0.1).to(torch.bfloat16).cuda() for size in ((T, K), (N, K)))
    want = B.exmoe_linear(x, w)
    wide = torch.full((T + 2, N), 7.0, dtype=torch.bfloat16, device="cuda")
    assert B.exmoe_linear_status() == B.EXMOE_OK
    rc = B.lib().exmoe_debug_linear_timeout(byref(B.exmoe_linear_shape(K, N, 0)), x.data_ptr(), w.data_ptr(), T, wide[1:T + 1].data_ptr(), torch.cuda.current_stream().cuda_stream)
    assert rc == B.EXMOE_OK
    assert B.exmoe_linear_status() == B.EXMOE_ERR_TIMEOUT                  # reported once, and cleared
    assert B.exmoe_linear_status() == B.EXMOE_OK
    assert (wide[[0, T + 1]] == 7.0).all()
    for _ in range(2):
        assert torch.equal(B.exmoe_linear(x, w), want)
    assert B.exmoe_linear_status() == B.EXMOE_OK


def test_refusals(B):
    p, f = 1 << 40, B.lib().exmoe_debug_linear_timeout
    for K, N, T, rc in ((512, 64, 100, B.EXMOE_ERR_SHAPE), (1024, 64, 16, B.EXMOE_ERR_SHAPE), (1024, 64, 0, B.EXMOE_ERR_ARG), (1020, 64, 100, B.EXMOE_ERR_SHAPE)):
        assert f(byref(B.exmoe_linear_shape(K, N, 0)), p, p + (1 << 32), T, p + (1 << 33), None) == rc
