"""Drafter passes over a paged cache whose newest row is appended by the kernel just before them, with BD_DRAFT_VIEW_READY and in a
drafter's order (row, pass, row, pass): the pass reads the view while that kernel runs, and the drafted rows after it, although
they lie in one page; against the same pass run after everything, and the last of them against 64 bits."""

import pytest
import torch

import paper_2606_00144_gb300 as bd
from tests import paged_reference as ref

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("t,page", [(509, 16), (1003, 512), (2048, 64)])
@pytest.mark.parametrize("b,h_kv,budget", [(1, 2, 64), (8, 8, 64), (2, 2, 500), (1, 1, 900)])
@pytest.mark.parametrize("graph", [False, True])
def test_the_row_just_appended_is_the_one_read(d, t, page, b, h_kv, budget, graph):
    gamma, G, turns = 3, 4, 8
    h_q, cap, budget = h_kv * G, t + gamma, min(budget, t)
    pool = ref.Pool([cap] * b, h_kv, page, d, seed=t, cap=cap)
    K, V, table = pool.cuda()
    cache, rope = bd.PagedCache(K, V), bd.Rope.of_base(d)
    g = torch.Generator("cuda").manual_seed(t)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda").to(BF)

    # the first positions, the last ones (in the drafted rows' pages) and some in between
    pos = torch.cat([torch.arange(8), torch.arange(8, t - 16)[::max(1, (t - 24) // (budget - 24))][:budget - 24], torch.arange(t - 16, t)]).int()
    idx = torch.full((b, h_kv, budget), -1, dtype=torch.int32, device="cuda")
    idx[..., :len(pos)] = pos.cuda()
    count = torch.full((b, h_kv), len(pos), dtype=torch.int32, device="cuda")
    shape = cache.shape(b, h_q, t, cap)
    behind = [cache.shape(b, h_q, t + j, cap) for j in range(gamma)]
    ws = bd.Workspace(bd.bd_workspace_size(shape, bd.BD_OP_PAGED_DRAFT, budget, gamma))
    o, late_o = (torch.empty(gamma, b, h_q, d, dtype=BF, device="cuda") for _ in range(2))
    lse, late_lse = (torch.empty(gamma, b, h_q, device="cuda") for _ in range(2))
    rows = torch.empty(gamma, 2, b, h_kv, 1, d, dtype=BF, device="cuda")        # keys and values
    q = torch.empty(gamma, b, h_q, 1, d, dtype=BF, device="cuda")
    q_rot = torch.empty_like(q)

    def drafter():
        for j in range(gamma):
            bd.bd_paged_append(behind[j], q[j], rows[j, 0], rows[j, 1], rope, cache, table, q_rot[j])
            # (the queries of the pass are the append's as well)
            bd.bd_paged_draft_attn(shape, q_rot[j].view(b, h_q, d), cache, table, idx, count, budget, j, o[j], lse[j], ws,
                                   flags=bd.BD_DRAFT_VIEW_READY)

    def fill(turn):                          # sizes that differ from turn to turn: a stale row shows
        rows.copy_(randn(*rows.shape) * 2.0 ** (turn % 3))
        q.copy_(randn(*q.shape))

    fill(0)
    drafter()
    run = drafter
    if graph:
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured):
            drafter()
        run = captured.replay
    for turn in range(turns):
        fill(turn)
        torch.cuda.synchronize()
        run()
        torch.cuda.synchronize()
        for j in range(gamma):               # (the rows of later passes are there by now, and not seen by this one)
            bd.bd_paged_draft_attn(shape, q_rot[j].view(b, h_q, d), cache, table, idx, count, budget, j, late_o[j], late_lse[j], ws)
        torch.cuda.synchronize()
        assert torch.equal(o, late_o) and torch.equal(lse, late_lse), turn
    assert ws.status() == 0
    pool.k, pool.v = K.cpu(), V.cpu()
    for i in {0, b - 1}:
        for h in {0, h_kv - 1}:
            hs = slice(h * G, (h + 1) * G)
            for j in range(gamma):
                k, v, there = pool.unit(i, h, torch.cat([pos.long(), t + torch.arange(j + 1)]))
                freq = 10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)
                want = ref.rotate(rows[j, 0, i, h].cpu(), torch.tensor([t + j]), freq, False)
                assert ((k[-1] - want[0]).abs() <= ref.rotate_tolerance(rows[j, 0, i, h].cpu(), want, freq, False)[0]).all()
                ref.check(o[j, i, hs], lse[j, i, hs], *ref.attend(q_rot[j, i, hs, 0].cpu(), k, v, there[None, :].expand(G, -1)), f"pass {j}")
