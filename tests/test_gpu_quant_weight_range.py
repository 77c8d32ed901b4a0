"""V rows whose sizes differ by a hundred octaves, and rows of zeros among them: every key counts for the normaliser by its
score alone, whatever its V."""

import pytest
import torch

import paper_2606_00144_gb300 as bd
from tests import quant_reference as ref
from tests.test_gpu_quant_attn import BF, check_draft, check_verify, run_draft, run_verify
from tests.test_gpu_quant_attn_long import run

pytestmark = pytest.mark.gpu


def sized(v, case, size):
    """v [.., rows, d] with some rows of zeros or far smaller than the others, which are 2^size."""
    v = v * 2.0 ** size
    rows = v.shape[-2]
    if case == "zeros between":
        v[..., ::2, :] = 0
    elif case == "zeros first":
        v[..., :rows // 2, :] = 0
    elif case == "zeros last":
        v[..., rows // 2:, :] = 0
    elif case == "small first":
        v[..., :rows // 2, :] *= 2.0 ** -120
    elif case == "small between":
        v[..., ::2, :] *= 2.0 ** -120
    return v


CASES = ["zeros between", "zeros first", "zeros last", "small first", "small between"]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n", [(1, 1), (4, 6), (4, 21)])
@pytest.mark.parametrize("long", [False, True])
@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("size", [40, 90])
def test_verify(d, G, n, long, case, size):
    t = 777
    g = torch.Generator().manual_seed(n)
    k, v = (torch.randn(2, 1, t + n, d, generator=g) for _ in range(2))
    tensors = [x for y in (k, sized(v, case, size)) for x in ref.quantise(y.to(BF))]
    q = torch.randn(2, G, n, d, generator=g).to(BF)
    o, lse = run(tensors, q, [t, t], n) if long else run_verify(tensors, q, t, n)
    check_verify(tensors, q, [t, t], n, o, lse, case)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [4, 16])
@pytest.mark.parametrize("budget", [200, 6000])
@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("size", [40, 90])
def test_draft(d, G, budget, case, size):
    t, j = budget + 100, 2
    g = torch.Generator().manual_seed(G)
    k, v = (torch.randn(1, 1, t + j + 1, d, generator=g) for _ in range(2))
    tensors = [x for y in (k, sized(v, case, size)) for x in ref.quantise(y.to(BF))]
    q = torch.randn(1, G, d, generator=g).to(BF)
    idx = torch.randperm(t, generator=g)[:budget].sort().values.int().view(1, 1, budget)
    count = torch.full((1, 1), budget, dtype=torch.int32)
    o, lse, status = run_draft(tensors, q, t, idx, count, j)
    assert status == 0
    check_draft(tensors, q, [t], idx, count, j, o, lse)


@pytest.mark.parametrize("n", [1, 4])
def test_a_long_cache_of_zeros_under_scores_that_grow(n):
    """V all zeros, so many keys to a CTA, each just short of what raises a maximum, that a sum in units of the largest
    weight over V's exponent leaves fp32."""
    units, t, d = 160, 40_000, 64
    codes = torch.full((1, units, t + n, d // 2), 0x88, dtype=torch.uint8, device="cuda")
    codes[:, :, 512:, 0] = 0x8f                              # element 0 is 7 but in the first tiles, where it is 0
    ones = torch.ones(1, units, t + n, d // 32, dtype=BF, device="cuda")
    cache = bd.QuantCache(codes, ones, torch.full_like(codes, 0x88), torch.zeros_like(ones))
    q = torch.zeros(1, units, n, d, device="cuda").to(BF)
    q[..., 0] = 6.25                                         # 6.25 * 7 / 8 nats: 7.89 in log2 units
    shape = cache.shape(units, t)
    ws = bd.Workspace(bd.bd_workspace_size(shape, bd.BD_OP_QUANT_VERIFY, 0, n))
    o, lse = torch.full_like(q, 7.0), torch.zeros(1, units, n, device="cuda")
    bd.bd_quant_verify_attn(shape, q, n, cache, o, lse, ws)
    assert ws.status() == 0
    assert (o == 0).all()
    late = t - 512 + 1 + torch.arange(n, device="cuda").double()
    want = torch.log(512 + late * torch.exp(torch.tensor(6.25 * 7 / 8, dtype=torch.float64)).item())
    assert (lse.double() - want).abs().max() < 1e-4
