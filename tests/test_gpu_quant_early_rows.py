"""Drafter passes whose newest row is written by the kernel just before them, with BD_DRAFT_VIEW_READY: the pass reads the
view while that kernel runs, and the drafted row after it, although their scales share cache lines."""

import pytest
import torch

import paper_2606_00144_gb300 as bd
from tests.test_gpu_quant_attn import BF

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("t", [509, 1003, 2048])
@pytest.mark.parametrize("b,h_kv,budget", [(1, 2, 64), (8, 8, 64), (2, 2, 500)])
def test_the_row_just_written_is_the_one_read(d, t, b, h_kv, budget):
    gamma, G, turns = 3, 4, 12
    h_q, cap = h_kv * G, t + gamma                           # no room past the drafted rows: the next unit's first row follows
    g = torch.Generator("cuda").manual_seed(t)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda").to(BF)

    cache = bd.QuantCache.empty(b, h_kv, cap, d)
    bd.bd_quant_write(cache.shape(h_q, 0), randn(b, h_kv, cap, d), randn(b, h_kv, cap, d), cache)
    # the first positions, the last ones and every third in between
    pos = torch.cat([torch.arange(8), torch.arange(8, t, 3)[:budget - 24], torch.arange(t - 16, t)]).int()
    idx = torch.full((b, h_kv, budget), -1, dtype=torch.int32, device="cuda")
    idx[..., :len(pos)] = pos.cuda()
    count = torch.full((b, h_kv), len(pos), dtype=torch.int32, device="cuda")
    shape = cache.shape(h_q, t)
    ws = bd.Workspace(bd.bd_workspace_size(shape, bd.BD_OP_QUANT_DRAFT, budget, gamma))
    o = [[torch.empty(b, h_q, d, dtype=BF, device="cuda") for _ in range(gamma)] for _ in range(2)]
    lse = [[torch.empty(b, h_q, device="cuda") for _ in range(gamma)] for _ in range(2)]
    behind = [cache.shape(h_q, t + j) for j in range(gamma)]
    for turn in range(turns):
        # (sizes that differ from turn to turn: a stale scale shows)
        rows = [[randn(b, h_kv, 1, d) * 2.0 ** ((turn + j) % 5) for _ in range(2)] for j in range(gamma)]
        q = [randn(b, h_q, d) for _ in range(gamma)]
        torch.cuda.synchronize()
        for j in range(gamma):
            bd.bd_quant_write(behind[j], *rows[j], cache)
            bd.bd_quant_draft_attn(shape, q[j], cache, idx, count, budget, j, o[0][j], lse[0][j], ws,
                                   flags=bd.BD_DRAFT_VIEW_READY)
        torch.cuda.synchronize()
        for j in range(gamma):
            bd.bd_quant_draft_attn(shape, q[j], cache, idx, count, budget, j, o[1][j], lse[1][j], ws)
            torch.cuda.synchronize()
            assert torch.equal(o[0][j], o[1][j]) and torch.equal(lse[0][j], lse[1][j]), (turn, j)
    assert ws.status() == 0
