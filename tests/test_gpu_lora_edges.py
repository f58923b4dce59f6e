"""Low-rank adapters where the definition gives infinities, and rows that are one only."""
import numpy as np
import pytest
import torch

from oracle import lora as olora

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2608_15383_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def normal(g, std, *size, dtype=torch.bfloat16):
    return (torch.randn(*size, generator=g) * std).to(dtype)


@pytest.mark.parametrize("r", [8, 16, 24, 40, 72, 128])
@pytest.mark.parametrize("T,dtype", [(1, torch.bfloat16), (20, torch.float32), (700, torch.bfloat16), (1300, torch.float32)])
def test_infinities_as_the_definition_gives_them(B, r, T, dtype):
    """An infinity in x makes the inner products infinite, and an output infinite where these all add up with one sign, NaN where they do not: whatever the rank is
    rounded up to."""
    n, K, N = 3, 64, 48
    g = torch.Generator().manual_seed(r + T)
    x, a, b = normal(g, 1.0, T, K), normal(g, 0.05, n, r, K), normal(g, 0.05, n, N, r)
    a[:, :, 7] = a[:, :, 7].abs() + 0.01
    b = torch.where(b == 0, torch.ones_like(b), b)
    b[:, ::2] = b[:, ::2].abs()
    b[:, 2::4] *= -1
    scale, ids = torch.tensor([1.0, -2.0, 0.5]), torch.randint(-1, n, (T,), generator=g).int()
    rows = sorted({0, T // 3, T - 1})
    ids[rows[0]], ids[rows[-1]] = 1, 2
    x[rows[0], 7] = float("inf")
    x[rows[-1], 7] = float("-inf")
    with np.errstate(invalid="ignore"):
        ref = olora.apply(x.double().numpy(), a.double().numpy(), b.double().numpy(), scale.double().numpy(), ids.numpy())
    out = B.exmoe_lora(B.exmoe_lora_plan(ids.cuda(), n), x.cuda(), a.cuda(), b.cuda(), scale.cuda(), out_dtype=dtype).double().cpu().numpy()
    assert np.isinf(ref).any() and np.isnan(ref[:, 1::2]).any()
    assert np.array_equal(np.isnan(out), np.isnan(ref))
    assert np.array_equal(np.where(np.isinf(out), np.sign(out), 0), np.where(np.isinf(ref), np.sign(ref), 0))


def test_one_row_in_place_whatever_its_distance_to_the_next(B):
    """A single row has no row behind it: base and out are the same where their addresses are."""
    g = torch.Generator().manual_seed(1)
    n, r, K, N = 2, 8, 64, 40
    x, a, b, scale = normal(g, 1.0, 1, K).cuda(), normal(g, 0.1, n, r, K).cuda(), normal(g, 0.1, n, N, r).cuda(), torch.ones(n, device="cuda")
    wide = normal(g, 1.0, 1, 2 * N).cuda()
    plan = B.exmoe_lora_plan(torch.zeros(1, dtype=torch.int32, device="cuda"), n)
    want = B.exmoe_lora(plan, x, a, b, scale, base=wide[:, :N])
    out = wide.as_strided((1, N), (N, 1))
    assert B.exmoe_lora(plan, x, a, b, scale, base=wide[:, :N], out=out) is out
    assert torch.equal(out, want)
