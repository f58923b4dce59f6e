"""Products over a long K, of inputs of one sign, where truncations add up: sums are made of chains of bounded length.

A chain of n MMAs is off by 5.25 n units of 2^-23 of its sum at most (each sums 16 products and truncates); chains, and warps' parts, are added in binary32, half a unit of 2^-23 each.
"""
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


def inputs(T, K, N, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.rand(n, K, generator=g, device="cuda").add_(0.01).bfloat16() for n in (T, N, N)]


def exact(x, w):
    y = torch.zeros(x.shape[0], w.shape[0], dtype=torch.float64, device="cuda")
    for k in range(0, x.shape[1], 32768):
        y += x[:, k:k + 32768].double() @ w[:, k:k + 32768].double().t()
    return y


def check(out, want, rel):
    tol = rel + torch.finfo(out.dtype).eps / 2 * (1 + rel)
    err = (out.double() / want - 1).abs().max().item()
    assert err <= tol, (err, tol)


@pytest.mark.parametrize("T,K,N", [(1200, 16384, 512), (1200, 16392, 512), (1200, 262144, 512), (700, 262144 + 24, 300)])
@pytest.mark.parametrize("gated", [False, True])
def test_bf16_results_of_many_tokens(B, T, K, N, gated):
    """No chain is longer than 1024 MMAs."""
    x, w, u = inputs(T, K, N, K + T)
    rel = (5.25 * 1024 + K / 16384 / 2 + 1) * 2.0 ** -23
    want = exact(x, w)
    if gated:
        want, rel = want * exact(x, u), 2 * rel + rel * rel + 2.0 ** -23
    check(B.exmoe_linear(x, w, w_up=u if gated else None), want, rel)
    assert B.exmoe_linear_status() == B.EXMOE_OK


@pytest.mark.parametrize("T,K,N", [(1, 8200, 40), (5, 16384, 64), (8, 262144, 64), (16, 262144 + 40, 33), (3, 1 << 20, 64), (12, 1 << 20, 2500)])
@pytest.mark.parametrize("gated", [False, True])
def test_fp32_results_of_few_tokens(B, T, K, N, gated):
    """No chain is longer than 32 MMAs; a warp has an eighth of K at most, and 16 parts are added at most."""
    x, w, u = inputs(T, K, N, K + T)
    rel = (5.25 * 32 + K / 16 / 32 / 8 / 2 + 1 + 8) * 2.0 ** -23
    want = exact(x, w)
    if gated:
        want, rel = want * exact(x, u), 2 * rel + rel * rel + 2.0 ** -23
    check(B.exmoe_linear(x, w, w_up=u if gated else None, out_dtype=torch.float32), want, rel)


@pytest.mark.parametrize("T,K,N", [(2, 65536, 64), (8, 65544, 64), (5, 131080, 2500), (16, 1 << 20, 64)])
@pytest.mark.parametrize("gated", [False, True])
def test_bf16_results_of_few_tokens(B, T, K, N, gated):
    """No chain is longer than 1024 MMAs."""
    x, w, u = inputs(T, K, N, K + T)
    rel = (5.25 * 1024 + K / 16 / 32 / 8 / 2 + 1 + 8) * 2.0 ** -23
    want = exact(x, w)
    if gated:
        want, rel = want * exact(x, u), 2 * rel + rel * rel + 2.0 ** -23
    check(B.exmoe_linear(x, w, w_up=u if gated else None), want, rel)


def test_a_wait_of_long_chains_that_runs_out(B):
    """The form of pairs that adds chains gives up as the others do: the call returns and says so, writes nothing outside of its result, and the next one is right."""
    T, K, N = 1200, 16448, 512
    x, w, _ = inputs(T, K, N, 1)
    want = B.exmoe_linear(x, w)
    wide = torch.full((T + 2, N), 7.0, dtype=torch.bfloat16, device="cuda")
    assert B.exmoe_linear_status() == B.EXMOE_OK
    rc = B.lib().exmoe_debug_linear_timeout(byref(B.exmoe_linear_shape(K, N, 0)), x.data_ptr(), w.data_ptr(), T, wide[1:T + 1].data_ptr(), torch.cuda.current_stream().cuda_stream)
    assert rc == B.EXMOE_OK
    assert B.exmoe_linear_status() == B.EXMOE_ERR_TIMEOUT and B.exmoe_linear_status() == B.EXMOE_OK
    assert (wide[[0, T + 1]] == 7.0).all()
    assert torch.equal(B.exmoe_linear(x, w), want)
