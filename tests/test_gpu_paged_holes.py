"""The selection and the window's normalisers over a paged cache of which pages are not there (given back behind a sliding window,
or anywhere): both are over the keys that are there, as the attentions are, each against 64 bits."""

import math

import numpy as np
import pytest
import torch

import oracle
import paper_2606_00144_gb300 as bd
from tests import paged_reference as ref
from tests.parity import check_selection, f64

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
SINK, RECENT, W = 4, 16, 8


def holes(kind, table, lens, page):
    """Entries of the table that go: behind a window but for the first page, here and there, or a whole sequence but its end."""
    table = table.clone()
    for i, t in enumerate(lens):
        last = (t - RECENT - W) // page              # (the recent positions and the window's own stay)
        if kind == "window":
            table[i, 1:max(1, (t - 100) // page)] = -1
        elif kind == "scattered":
            table[i, 1:last:3] = -1 - i
        elif kind == "all":
            table[i, :last] = -1
    return table


def setting(lens, h_kv, G, d, page, kind, seed=0, away_by=0.0):
    """away_by: how far the window's queries point away from the keys, so that scores are below those of a key of zeros."""
    b, cap = len(lens), max(lens) + 8
    pool = ref.Pool([t + 8 for t in lens], h_kv, page, d, seed=seed, cap=cap)
    g = torch.Generator().manual_seed(seed + 1)
    q = torch.randn(b, h_kv * G, W, d, generator=g)
    if away_by:
        away = torch.nn.functional.normalize(torch.randn(d, generator=g), dim=0)
        pool.k = (pool.k.float() + 4 * away).to(BF)
        q -= away_by * away
    pool.table = holes(kind, pool.table, lens, page)
    return pool, q.to(BF)


def expected(pool, q, lens, i, h, G):
    """Normalisers [G, W] and scores [t] of one (sequence, KV head), 64 bits, absent keys hidden."""
    t, d = lens[i], q.shape[-1]
    k, _, there = pool.unit(i, h, torch.arange(t))
    x = (q[i, h * G:(h + 1) * G].double() @ torch.where(there[:, None], k, 0.0).T) / math.sqrt(d)        # [G, W, t]
    seen = (torch.arange(t)[None, :] <= (t - W + torch.arange(W))[:, None]) & there[None, :]
    x = torch.where(seen, x, -math.inf)
    lse = torch.logsumexp(x, -1)
    return lse, torch.where(seen, torch.exp(x - lse[..., None]), 0.0).sum((0, 1)), there


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 4])
@pytest.mark.parametrize("lens", [[1500], [1201, 777, 1500]])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("kind", ["none", "window", "scattered", "all"])
@pytest.mark.parametrize("chunk", [1, 8])
def test_select_and_normalisers(d, G, lens, page, kind, chunk):
    h_kv, budget, b = 2, 100, len(lens)
    pool, q = setting(lens, h_kv, G, d, page, kind, seed=d + G + page, away_by=6.0)
    K, V, table = pool.cuda()
    cache = bd.PagedCache(K, V)
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda") if b > 1 else None
    step = bd.PagedSpecStep(b, h_kv * G, h_kv, d, max(lens), pool.cap, budget, SINK, RECENT, W, gamma=2, chunk=chunk, seq_lens=seq)
    dev = q.cuda()
    lse = step.window_lse(cache, table, dev)
    want = [[expected(pool, q, lens, i, h, G) for h in range(h_kv)] for i in range(b)]
    for i in range(b):
        for h in range(h_kv):
            wl = want[i][h][0]
            # (as in paged_reference.check: sum |q k| log2(e) / sqrt(d) is about 20 for these rows, within its 80)
            assert ((lse[i, h * G:(h + 1) * G].cpu().double() - wl).abs() <= 8e-5 + 1e-5 * wl.abs()).all()
    for given in (lse, None):
        step.idx.fill_(-7)
        step.select(cache, table, dev, given)
        assert step.ws.status() == 0
        for i, t in enumerate(lens):
            for h in range(h_kv):
                _, score, there = want[i][h]
                keep = oracle.select_from_scores(score.numpy(), t, budget, SINK, RECENT, chunk)
                idx = np.full((1, budget), -1)
                idx[0, :keep.size] = keep
                check_selection(step.idx[i, h], step.count[i, h:h + 1], idx, [keep.size], score.numpy(), t, budget, SINK, RECENT,
                                chunk, what=f"{kind} seq {i} head {h}")
                if chunk == 1:       # nothing absent in the middle is kept while something that is there is left
                    kept = step.idx[i, h].cpu().long()
                    middle = kept[(kept >= SINK) & (kept < t - RECENT)]
                    assert there[middle].sum() == min(len(middle), int(there[SINK:t - RECENT].sum()))


@pytest.mark.parametrize("d,page", [(64, 16), (128, 32)])
def test_a_windowed_step(d, page):
    """run(): the selection, the passes and the block of a step behind a window, against 64 bits."""
    lens, h_kv, G, gamma, budget = [900, 1300], 2, 4, 2, 64
    pool, q = setting(lens, h_kv, G, d, page, "window", seed=5)
    K, V, table = pool.cuda()
    cache = bd.PagedCache(K, V)
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
    step = bd.PagedSpecStep(2, h_kv * G, h_kv, d, max(lens), pool.cap, budget, SINK, RECENT, W, gamma=gamma, seq_lens=seq)
    g = torch.Generator().manual_seed(3)
    q_draft, q_verify = torch.randn(gamma, 2, h_kv * G, d, generator=g).to(BF), torch.randn(2, h_kv * G, gamma + 1, d, generator=g).to(BF)
    step.run(cache, table, q.cuda(), q_draft.cuda(), q_verify.cuda())
    assert step.ws.status() == 0
    for i, t in enumerate(lens):
        for h in range(h_kv):
            hs = slice(h * G, (h + 1) * G)
            view = step.idx[i, h, :int(step.count[i, h])].long().cpu()
            assert len(view) == budget
            for j in range(gamma):
                k, v, there = pool.unit(i, h, torch.cat([view, t + torch.arange(j + 1)]))
                assert there.all()                          # a whole view: sinks and recent positions are there
                ref.check(step.draft_o[j, i, hs], step.draft_lse[j, i, hs],
                          *ref.attend(q_draft[j, i, hs], k, v, there[None, :].expand(G, -1)), f"draft {j}")
            rows = torch.arange(t + gamma + 1)
            k, v, there = pool.unit(i, h, rows)
            visible = (rows[None, :] <= (t + torch.arange(gamma + 1).repeat(G))[:, None]) & there[None, :]
            ref.check(step.verify_o[i, hs].reshape(-1, d), step.verify_lse[i, hs].reshape(-1),
                      *ref.attend(q_verify[i, hs].reshape(-1, d), k, v, visible), "verify")


def test_a_window_that_sees_nothing():
    """Every page gone: the normalisers are -inf, every score 0, and the lowest positions of the middle are kept."""
    lens, d, page, budget = [300, 260], 64, 16, 40
    pool, q = setting(lens, 1, 2, d, page, "none")
    pool.table[0] = -1
    K, V, table = pool.cuda()
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
    step = bd.PagedSpecStep(2, 2, 1, d, 300, pool.cap, budget, SINK, RECENT, W, gamma=1, seq_lens=seq)
    cache = bd.PagedCache(K, V)
    lse = step.window_lse(cache, table, q.cuda())
    assert (lse[0] == -math.inf).all() and torch.isfinite(lse[1]).all()
    step.select(cache, table, q.cuda())
    assert step.ws.status() == 0
    assert step.idx[0, 0].tolist() == [*range(budget - RECENT), *range(300 - RECENT, 300)]
    _, score, _ = expected(pool, q, lens, 1, 0, 2)
    keep = oracle.select_from_scores(score.numpy(), 260, budget, SINK, RECENT, 1)
    check_selection(step.idx[1], step.count[1], keep[None], [budget], score.numpy(), 260, budget, SINK, RECENT)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("layout", ["heads", "rows"])
def test_keys(d, layout):
    """Rows that are there as they lie, NaN for absent pages (an entry past the pool's end is one), nothing past a length."""
    lens, page, h_kv = [200, 0, 77], 16, 2
    pool = ref.Pool([max(t, 1) for t in lens], h_kv, page, d, seed=2, cap=208, layout=layout)
    pool.table[0, 3] = -1
    pool.table[0, 5] = pool.k.shape[0]
    pool.table[2, 0] = -(2**31)
    K, V, table = pool.cuda()
    cache = bd.PagedCache(K, V)
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
    out = torch.full((3, h_kv, 203, d), 7.0, dtype=BF, device="cuda")[:, :, 2:202]
    bd.bd_paged_keys(cache.shape(3, h_kv, 200, 208, seq), cache, table, out)
    for i, t in enumerate(lens):
        for h in range(h_kv):
            k, _, there = pool.unit(i, h, torch.arange(t))
            got = out[i, h].cpu().double()
            assert torch.equal(got[:t][there], k[there]) and got[:t][~there].isnan().all() and (got[t:] == 7).all()
    bd.bd_paged_keys(cache.shape(3, h_kv, 200, 208, seq), cache, table, out[:, :, :0])
    assert f64(out[1]).min() == 7


def test_normalisers_in_a_graph_and_on_another_stream():
    """A captured selection follows the table; on another stream the call's own memory belongs to that stream."""
    lens, h_kv, G, d, page, budget = [700, 512], 2, 4, 128, 16, 64
    pool, q = setting(lens, h_kv, G, d, page, "window", seed=8)
    K, V, table = pool.cuda()
    cache, dev = bd.PagedCache(K, V), q.cuda()
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
    step = bd.PagedSpecStep(2, h_kv * G, h_kv, d, 700, pool.cap, budget, SINK, RECENT, W, gamma=1, seq_lens=seq)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    step.select(cache, table, dev, stream=side)
    side.synchronize()
    want = step.idx.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.select(cache, table, dev)
    other = holes("scattered", pool.table, lens, page).cuda()
    first = table.clone()
    for entries in (first, other, first):
        table.copy_(entries)
        step.idx.zero_()
        graph.replay()
        torch.cuda.synchronize()
        pool.table = entries.cpu()
        for i, t in enumerate(lens):
            for h in range(h_kv):
                _, score, _ = expected(pool, q, lens, i, h, G)
                keep = oracle.select_from_scores(score.numpy(), t, budget, SINK, RECENT, 1)
                check_selection(step.idx[i, h], step.count[i, h:h + 1], keep[None], [budget], score.numpy(), t, budget, SINK, RECENT)
    assert torch.equal(step.idx, want) and step.ws.status() == 0
