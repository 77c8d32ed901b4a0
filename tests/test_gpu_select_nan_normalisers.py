"""A selection that computes its window's normalisers itself (window_lse NULL), with BD_SELECT_NAN_HIDDEN: keys that hold NaN
have no part in them, so the other keys' scores, and what is kept, are as without those keys; against 64 bits.  A verify block's
rows, and a selection's without the flag, stay as they were."""

import math

import numpy as np
import pytest
import torch

import oracle
import paper_2606_00144_gb300 as bd
from tests.parity import check_selection

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,W", [(1, 8), (4, 8), (4, 16), (4, 32)])        # 8 and 32 (four copies), 64 (two), 128 rows (one)
@pytest.mark.parametrize("lens", [[3001], [1500, 130, 2999]])
@pytest.mark.parametrize("bad", ["some", "a tile", "most"])
def test_nan_keys_have_no_part(d, G, W, lens, bad):
    b, h_kv, budget, sink, recent, t_cap = len(lens), 2, 100, 4, 16, max(lens) + 5
    g = torch.Generator().manual_seed(d + W + G)
    k = torch.full((b, h_kv, t_cap, d), math.nan, dtype=BF)
    q = torch.randn(b, h_kv * G, W, d, generator=g).to(BF)
    gone = torch.zeros(b, h_kv, t_cap, dtype=torch.bool)
    for i, t in enumerate(lens):
        k[i, :, :t] = torch.randn(h_kv, t, d, generator=g).to(BF)
        gone[i, 0, slice(5, t, 97) if bad == "some" else slice(0, t // 2) if bad == "a tile" else slice(0, t - 1)] = True
        gone[i, 1, t - W // 2] = True            # hidden from some rows of the window as it is
    k[gone] = math.nan
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda") if b > 1 else None
    step = bd.SpecStep(b, h_kv * G, h_kv, d, max(lens), t_cap, budget, sink, recent, W, 1, seq_lens=seq)
    bd.bd_select_budget(step.shape, k.cuda(), q.cuda(), None, W, budget, sink, recent, 1, step.idx, step.count, step.ws,
                        flags=bd.BD_SELECT_NAN_HIDDEN)
    assert step.ws.status() == 0
    for i, t in enumerate(lens):
        for h in range(h_kv):
            x = q[i, h * G:(h + 1) * G].double() @ torch.where(gone[i, h, :t, None], 0.0, k[i, h, :t].double()).T / math.sqrt(d)
            seen = (torch.arange(t)[None, :] <= (t - W + torch.arange(W))[:, None]) & ~gone[i, h, None, :t]
            x = torch.where(seen, x, -math.inf)
            lse = torch.logsumexp(x, -1, keepdim=True)
            score = torch.where(seen, torch.exp(x - lse), 0.0).sum((0, 1)).numpy()
            keep = oracle.select_from_scores(score, t, budget, sink, recent, 1)
            idx = np.full((1, budget), -1)
            idx[0, :keep.size] = keep
            check_selection(step.idx[i, h], step.count[i, h:h + 1], idx, [keep.size], score, t, budget, sink, recent, what=f"{i} {h}")


@pytest.mark.parametrize("d", [64, 128])
def test_a_verify_blocks_normalisers_keep_their_nan(d):
    """bd_verify_attn without an output runs the same kernel: a row that sees a NaN is -inf there, as before."""
    t, n = 700, 4
    k = torch.randn(1, 2, t + n, d, device="cuda").to(BF)
    k[0, 0, 300] = math.nan
    q, lse = torch.randn(1, 2, n, d, device="cuda").to(BF), torch.empty(1, 2, n, device="cuda")
    shape = bd.make_shape(1, 2, 2, d, t, t + n)
    bd.bd_verify_attn(shape, q, n, k, None, None, lse, bd.Workspace(bd.bd_workspace_size(shape, bd.BD_OP_VERIFY, 1, n)))
    assert (lse[0, 0] == -math.inf).all() and torch.isfinite(lse[0, 1]).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("W", [8, 32])
def test_the_flag_changes_nothing_where_there_is_no_nan(d, W):
    b, h_kv, G, t, budget = 3, 2, 4, 4097, 300
    k, q = (torch.randn(b, h, n, d, device="cuda").to(BF) for h, n in ((h_kv, t), (h_kv * G, W)))
    step = bd.SpecStep(b, h_kv * G, h_kv, d, t, t, budget, 4, 64, W, 0)
    step.select(k, q)
    plain = step.idx.clone()
    for flags in (bd.BD_SELECT_NAN_HIDDEN, bd.BD_SELECT_NAN_HIDDEN | bd.BD_SELECT_WINDOW_READY):
        step.idx.fill_(-7)
        torch.cuda.synchronize()
        bd.bd_select_budget(step.shape, k, q, None, W, budget, 4, 64, 1, step.idx, step.count, step.ws, flags=flags)
        assert torch.equal(step.idx, plain) and step.ws.status() == 0
