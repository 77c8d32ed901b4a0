"""A block row whose V is not a number: the queries before it do not see it, and their outputs are what they would be
without it; the queries that see it have NaN in that group's channels alone."""

import math

import pytest
import torch

import paper_2606_00144_gb300 as bd
from tests import quant_reference as ref
from tests.test_gpu_quant_attn import BF, make_cache, run_verify_nan
from tests.test_gpu_quant_attn_long import room, widened

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n", [(1, 6), (4, 6), (8, 4), (8, 8), (4, 21), (8, 21)])
@pytest.mark.parametrize("long", [False, True])
@pytest.mark.parametrize("t", [127, 300])
def test_queries_before_it_are_untouched(d, G, n, long, t):
    tensors = make_cache(2, 1, t + n, d, seed=n)
    q = torch.randn(2, G, n, d, generator=torch.Generator().manual_seed(n)).to(BF)
    clean = [x.clone() for x in tensors]
    bad = {0: (3, 1), 1: (1, 0)}                             # sequence: the block's row, its group
    for i, (row, group) in bad.items():
        tensors[3][i, 0, t + row, group] = math.nan
        tensors[2][i, 0, t + row, 16 * group:16 * group + 16] = 0x88
        clean[3][i, 0, t + row, group] = 0                   # (what a query that does not see the row makes of it)
    if long:
        cap = room(G * n, d) + n
        seq = torch.tensor([t, t], dtype=torch.int32, device="cuda")
        o, lse = run_lens(widened(tensors, cap), q, cap - n, n, seq)
    else:
        o, lse = run_verify_nan(tensors, q, t, n)
    o, lse = o.cpu(), lse.cpu()
    for i, (row, group) in bad.items():
        g = slice(32 * group, 32 * group + 32)
        assert o[i, :, row:, g].isnan().all()
        assert torch.isfinite(o[i, :, :row]).all()
        o[i, :, row:, g] = 0
    # every other number, against 64 bits (the queries that see the row: its group alone is left out)
    for i, (row, group) in bad.items():
        k = ref.values(clean[0][i, 0], clean[1][i, 0])
        v = ref.values(clean[2][i, 0], clean[3][i, 0])
        visible = torch.arange(t + n)[None, :] <= (t + torch.arange(n).repeat(G))[:, None]
        wo, wl, spread = ref.attend(q[i].reshape(G * n, d), k, v, visible)
        wo = wo.reshape(G, n, d)
        wo[:, row:, 32 * group:32 * group + 32] = 0
        ref.check(o[i].reshape(G * n, d), lse[i].reshape(-1), wo.reshape(G * n, d), wl, spread, v.abs().max(), f"seq {i}")


def run_lens(tensors, q, t, n, seq):
    cache = bd.QuantCache(*(x.cuda() for x in tensors))
    shape = cache.shape(q.shape[1], t, seq)
    ws = bd.Workspace(bd.bd_workspace_size(shape, bd.BD_OP_QUANT_VERIFY, 0, n))
    o, lse = torch.empty_like(q, device="cuda"), torch.empty(q.shape[:3], device="cuda")
    bd.bd_quant_verify_attn(shape, q.cuda(), n, cache, o, lse, ws)
    torch.cuda.synchronize()
    return o, lse


@pytest.mark.parametrize("long", [False, True])
def test_an_infinity_in_a_drafted_row(long):
    """The way it comes about: a written row holds an infinity; tokens before it must not change."""
    b, h_kv, G, n, d, t = 1, 2, 4, 6, 128, 250
    cap = (room(G * n, d) if long else t) + n
    g = torch.Generator().manual_seed(5)
    k, v = (torch.randn(b, h_kv, t + n, d, generator=g).to(BF) for _ in range(2))
    q = torch.randn(b, h_kv * G, n, d, generator=g).to(BF)
    seq = torch.tensor([t], dtype=torch.int32, device="cuda")
    v[0, 1, t + 2, 70] = math.inf
    cache = bd.QuantCache.empty(b, h_kv, cap, d)
    bd.bd_quant_write(cache.shape(h_kv * G, 0), k.cuda(), v.cuda(), cache)
    shape = cache.shape(h_kv * G, cap - n, seq)
    ws = bd.Workspace(bd.bd_workspace_size(shape, bd.BD_OP_QUANT_VERIFY, 0, n))
    o, lse = torch.empty_like(q, device="cuda"), torch.empty(q.shape[:3], device="cuda")
    bd.bd_quant_verify_attn(shape, q.cuda(), n, cache, o, lse, ws)
    assert ws.status() == 0
    o = o.cpu()
    assert o[0, G:, 2:, 64:96].isnan().all()
    o[0, G:, 2:, 64:96] = 0
    v[0, 1, t + 2, 64:96] = 0                                # (what a query that does not see the row makes of it)
    tensors = [x for y in (k, v) for x in ref.quantise(y)]
    visible = torch.arange(t + n)[None, :] <= (t + torch.arange(n).repeat(G))[:, None]
    for h in range(h_kv):
        hs = slice(h * G, (h + 1) * G)
        wo, wl, spread = ref.attend(q[0, hs].reshape(G * n, d), ref.values(tensors[0][0, h], tensors[1][0, h]),
                                    ref.values(tensors[2][0, h], tensors[3][0, h]), visible)
        if h == 1:
            wo = wo.reshape(G, n, d)
            wo[:, 2:, 64:96] = 0
        ref.check(o[0, hs].reshape(G * n, d), lse[0, hs].reshape(-1), wo.reshape(G * n, d), wl, spread, v[0, h].abs().max().double(), f"head {h}")
