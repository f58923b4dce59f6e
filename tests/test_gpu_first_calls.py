"""Products, losses and gradients where a process calls them for the first time inside a capture, and where calls of different forms overlap."""
import subprocess
import sys
from types import SimpleNamespace

import pytest
import torch

pytestmark = pytest.mark.gpu

CAPTURED = """
import torch
from types import SimpleNamespace
from paper_2608_15383_b200 import binding as B
T, E = {T}, 64
s, g = SimpleNamespace(d_model=128, num_experts=E, top_k=4), SimpleNamespace(score="sigmoid", num_groups=1, top_groups=1, group_score="max", renormalise=True, scale=1.0)
rng = torch.Generator().manual_seed(T)
x, w, u = (torch.randn(*n, generator=rng).bfloat16().cuda() for n in ((T, 256), (E, 256), (E, 256)))
ids = torch.rand(T, E, generator=rng).argsort(1)[:, :4].int().cuda()
dw, dl = torch.ones(T, 4, device="cuda"), torch.ones(2, device="cuda")
offsets = torch.tensor([0, T // 3, T], dtype=torch.int32).cuda()
def step():
    z = B.exmoe_linear(x, w, w_up=u, activation="silu", out_dtype=torch.float32)
    out = B.exmoe_balance_loss(s, g, z, ids, offsets=offsets)
    return (z,) + out + (B.exmoe_gate_backward(s, g, z, ids, dw, dl, out[1], out[3], offsets=offsets),)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    got = step()
graph.replay()
torch.cuda.synchronize()
want = step()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.isfinite(got[1]).all() and int(got[2].sum()) == 4 * T
assert B.exmoe_linear_status() == B.EXMOE_OK
print("captured", T)
"""


@pytest.mark.parametrize("T", [1, 40, 3000])
def test_first_calls_in_a_capture(T):
    p = subprocess.run([sys.executable, "-c", CAPTURED.format(T=T)], capture_output=True, text=True, timeout=300)
    assert p.returncode == 0 and f"captured {T}" in p.stdout, p.stderr[-2000:]


@pytest.fixture(scope="module")
def B():
    from paper_2608_15383_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def test_forms_overlap(B):
    """Every form of the products, the loss and the gradient on streams of their own, at once: the bits of calls one after the other."""
    rng = torch.Generator().manual_seed(1)
    normal = lambda *n: torch.randn(*n, generator=rng).bfloat16().cuda()
    s = SimpleNamespace(d_model=128, num_experts=64, top_k=4)
    g = SimpleNamespace(score="softmax", num_groups=1, top_groups=1, group_score="max", renormalise=False, scale=1.0)
    w, u, down = normal(1408, 1024), normal(1408, 1024), normal(1024, 1408)
    z, ids = torch.randn(9000, 64, generator=rng).cuda(), torch.rand(9000, 64, generator=rng).argsort(1)[:, :4].int().cuda()
    dl = torch.ones(2, device="cuda")

    def products(T):
        x, y = normal(T, 1024), normal(T, 1024)

        def run(stream):
            act = B.exmoe_linear(x, w, w_up=u, activation="gelu", stream=stream)
            return (B.exmoe_linear(act, down, residual=y, stream=stream),)
        return run

    def gate(stream):
        out = B.exmoe_balance_loss(s, g, z, ids, stream=stream)
        return out + (B.exmoe_gate_backward(s, g, z, None, None, dl, out[1], out[3], stream=stream),)
    calls = [products(1), products(12), products(33), products(64), products(700), products(3000), gate]
    want = []
    for call in calls:
        want.append(call(None))
        torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    outs = [(i, call(st)) for _ in range(20) for i, (call, st) in enumerate(zip(calls, streams))]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for i, out in outs for a, b in zip(out, want[i]))
    assert B.exmoe_linear_status() == B.EXMOE_OK


@pytest.mark.parametrize("T", [7, 100, 1500])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_one_matrix_in_several_places(B, T, dtype):
    """x as the weights, the same matrix for both factors: inputs may be one another."""
    rng = torch.Generator().manual_seed(T)
    x = torch.randn(T, 64, generator=rng).bfloat16().cuda()
    assert torch.equal(B.exmoe_linear(x, x, w_up=x, out_dtype=dtype), B.exmoe_linear(x.clone(), x.clone(), w_up=x.clone(), out_dtype=dtype))


def test_pairs_with_rows_far_apart(B):
    """Results and residuals beyond 32 bits of bytes and of elements, on pairs of CTAs."""
    T, K, N = 1200, 2048, 300
    rng = torch.Generator().manual_seed(3)
    x, w, r = (torch.randn(*n, generator=rng).bfloat16().cuda() for n in ((T, K), (N, K), (T, N)))
    big = torch.empty(T << 22, dtype=torch.bfloat16, device="cuda")
    res, out = (big[at:].as_strided((T, N), (1 << 22, 1)) for at in (0, 512))
    res.copy_(r)
    B.exmoe_linear(x, w, residual=res, out=out)
    assert torch.equal(out, B.exmoe_linear(x, w, residual=r)) and torch.equal(res, r)
