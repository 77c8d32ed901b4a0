"""A V row with one group that is not a number, among V of any size: the row's other groups are finite and right."""

import math

import pytest
import torch

import paper_2606_00144_gb300 as bd
from tests import quant_reference as ref
from tests.test_gpu_quant_attn import BF, run_verify_nan
from tests.test_gpu_quant_attn_long import room, widened
from tests.test_gpu_quant_hidden_nan import run_lens

pytestmark = pytest.mark.gpu


def check_healthy(tensors, group, q, rows, visible, o, lse, what):
    """All channels but the group's against 64 bits, the group's NaN."""
    d = q.shape[-1]
    k = ref.values(tensors[0][rows], tensors[1][rows])
    scales = tensors[3][rows].clone()
    scales[scales.isnan()] = 0
    v = ref.values(tensors[2][rows], scales)
    wo, wl, spread = ref.attend(q.reshape(-1, d), k, v, visible)
    o, lse = o.reshape(-1, d).cpu(), lse.reshape(-1).cpu()
    g = slice(32 * group, 32 * group + 32)
    assert o[:, g].isnan().all(), what
    keep = [c for c in range(d) if not g.start <= c < g.stop]
    ref.check(o[:, keep], lse, wo[:, keep], wl, spread[:, keep], v.abs().max(), what)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n", [(1, 1), (4, 6), (8, 8), (4, 21)])
@pytest.mark.parametrize("long", [False, True])
@pytest.mark.parametrize("size", [0, 10, -40])
def test_verify(d, G, n, long, size):
    t, group = 300, 1
    g = torch.Generator().manual_seed(n + size)
    k, v = (torch.randn(2, 1, t + n, d, generator=g) for _ in range(2))
    tensors = [x for y in (k, v * 2.0 ** size) for x in ref.quantise(y.to(BF))]
    q = torch.randn(2, G, n, d, generator=g).to(BF)
    tensors[3][:, 0, 45, group] = math.nan                   # a context row: every query sees it
    if long:
        cap = room(G * n, d) + n
        o, lse = run_lens(widened(tensors, cap), q, cap - n, n, torch.tensor([t, t], dtype=torch.int32, device="cuda"))
    else:
        o, lse = run_verify_nan(tensors, q, t, n)
    visible = torch.arange(t + n)[None, :] <= (t + torch.arange(n).repeat(G))[:, None]
    for i in range(2):
        check_healthy([x[i, 0] for x in tensors], group, q[i], slice(0, t + n), visible, o[i], lse[i], f"seq {i}")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [4, 16])
@pytest.mark.parametrize("size", [0, 10, -40])
def test_draft(d, G, size):
    t, j, budget, group = 400, 2, 200, 0
    g = torch.Generator().manual_seed(G + size)
    k, v = (torch.randn(1, 1, t + j + 1, d, generator=g) for _ in range(2))
    tensors = [x for y in (k, v * 2.0 ** size) for x in ref.quantise(y.to(BF))]
    q = torch.randn(1, G, d, generator=g).to(BF)
    idx = torch.randperm(t, generator=g)[:budget].sort().values.int().view(1, 1, budget)
    tensors[3][0, 0, int(idx[0, 0, 77]), group] = math.nan
    cache = bd.QuantCache(*(x.cuda() for x in tensors))
    shape = cache.shape(G, t)
    ws = bd.Workspace(bd.bd_workspace_size(shape, bd.BD_OP_QUANT_DRAFT, budget, j + 1))
    o, lse = torch.empty_like(q, device="cuda"), torch.empty(q.shape[:2], device="cuda")
    bd.bd_quant_draft_attn(shape, q.cuda(), cache, idx.cuda(), torch.full((1, 1), budget, dtype=torch.int32, device="cuda"),
                           budget, j, o, lse, ws)
    rows = torch.cat([idx[0, 0].long(), t + torch.arange(j + 1)])
    check_healthy([x[0, 0] for x in tensors], group, q[0], rows, torch.ones(G, len(rows), dtype=torch.bool), o[0], lse[0], "draft")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n", [(1, 1), (4, 6), (4, 21)])
@pytest.mark.parametrize("long", [False, True])
def test_a_row_of_next_to_no_weight(d, G, n, long):
    """A context row that is NaN is seen by every query, also where another part of the context has all the weight."""
    t, group = 2000, 1
    g = torch.Generator().manual_seed(n)
    k, v = (torch.randn(2, 1, t + n, d, generator=g) * 0.1 for _ in range(2))
    k[:, :, 1700, 0] = 40.0
    q = torch.randn(2, G, n, d, generator=g) * 0.1
    q[..., 0] = 100.0                                        # 4000 / sqrt(d): hundreds of nats above the others
    tensors = [x for y in (k, v) for x in ref.quantise(y.to(BF))]
    q = q.to(BF)
    tensors[3][:, 0, 45, group] = math.nan
    if long:
        cap = room(G * n, d) + n
        o, lse = run_lens(widened(tensors, cap), q, cap - n, n, torch.tensor([t, t], dtype=torch.int32, device="cuda"))
    else:
        o, lse = run_verify_nan(tensors, q, t, n)
    visible = torch.arange(t + n)[None, :] <= (t + torch.arange(n).repeat(G))[:, None]
    for i in range(2):
        check_healthy([x[i, 0] for x in tensors], group, q[i], slice(0, t + n), visible, o[i], lse[i], f"seq {i}")
