"""Verify blocks (one query to the longest) and drafter passes over a paged cache on the GPU against 64 bits, at the lengths,
pages, masks and values where a kernel can go wrong."""

import math

import pytest
import torch

import paper_2606_00144_gb300 as bd
from tests import paged_reference as ref

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def queries(b, h_q, n, d, seed=0, size=1.0):
    return (torch.randn(b, h_q, n, d, generator=torch.Generator().manual_seed(seed)) * size).to(BF)


def run_verify(pool, q, t, n, seq=None, ws_n=None, stream=None, status=0):
    K, V, table = pool.cuda()
    cache = bd.PagedCache(K, V)
    lens = None if seq is None else torch.tensor(seq, dtype=torch.int32, device="cuda")
    shape = cache.shape(q.shape[0], q.shape[1], t, pool.cap, lens)
    ws = bd.Workspace(bd.bd_workspace_size(shape, bd.BD_OP_PAGED_VERIFY, 0, ws_n or n))
    o = torch.full(q.shape, 7.0, dtype=BF, device="cuda")
    lse = torch.full(q.shape[:3], 7.0, device="cuda")
    dq = q.cuda()
    torch.cuda.synchronize()
    bd.bd_paged_verify_attn(shape, dq, n, cache, table, o, lse, ws, stream)
    torch.cuda.synchronize()
    first, first_lse = o.clone(), lse.clone()
    bd.bd_paged_verify_attn(shape, dq, n, cache, table, o, lse, ws, stream)     # the workspace is left as it was
    torch.cuda.synchronize()
    assert ws.status() == status
    assert torch.equal(first.view(torch.int16), o.view(torch.int16)) and torch.equal(first_lse.view(torch.int32), lse.view(torch.int32))
    return o.cpu(), lse.cpu()


def check_verify(pool, q, lens, n, o, lse, what=""):
    b, h_q, _, d = q.shape
    h_kv = pool.k.shape[1]
    G = h_q // h_kv
    for i in range(b):
        rows = torch.arange(lens[i] + n)
        for h in range(h_kv):
            k, v, there = pool.unit(i, h, rows)
            hs = slice(h * G, (h + 1) * G)
            visible = (rows[None, :] <= (lens[i] + torch.arange(n).repeat(G))[:, None]) & there[None, :]
            want = ref.attend(q[i, hs].reshape(G * n, d), k, v, visible)
            ref.check(o[i, hs].reshape(G * n, d), lse[i, hs].reshape(-1), *want, f"{what} seq {i} head {h}")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n", [(1, 1), (4, 1), (4, 2), (8, 2), (4, 6), (1, 17), (8, 4), (8, 5), (3, 21), (8, 21), (8, 25), (16, 3)])
@pytest.mark.parametrize("t,page", [(0, 16), (1, 32), (15, 16), (16, 16), (63, 64), (127, 128), (130, 16), (300, 256), (700, 32)])
def test_verify_lengths(d, G, n, t, page):
    b, h_kv = 2, 2
    pool = ref.Pool([t + n] * b, h_kv, page, d, seed=t + 7 * n, cap=t + n + 3, layout=("heads", "rows", "both")[(t + n) % 3])
    q = queries(b, h_kv * G, n, d, n)
    o, lse = run_verify(pool, q, t, n)
    check_verify(pool, q, [t] * b, n, o, lse)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n", [(4, 1), (4, 6), (8, 21), (1, 6)])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("lens", [[0, 1, 2, 700], [513, 0, 129, 128], [2500, 31, 2499, 64], [3, 3, 3, 3]])
def test_verify_unequal_lengths(d, G, n, page, lens):
    b, h_kv = len(lens), 2
    pool = ref.Pool([t + n for t in lens], h_kv, page, d, seed=sum(lens), cap=max(lens) + n + 1)
    q = queries(b, h_kv * G, n, d, n)
    o, lse = run_verify(pool, q, max(lens), n, lens)
    check_verify(pool, q, lens, n, o, lse)


@pytest.mark.parametrize("b,h_kv,G,n,t,d,page", [
    (1, 1, 4, 6, 40000, 128, 16), (1, 2, 8, 1, 33001, 64, 64), (5, 4, 4, 6, 2049, 128, 32), (40, 8, 4, 6, 260, 128, 16),
    (40, 8, 1, 1, 517, 64, 16), (2, 2, 8, 96, 300, 128, 16), (1, 1, 8, 96, 5000, 64, 128), (3, 4, 8, 21, 2100, 128, 16),
    (1, 1, 8, 32, 900, 128, 32), (2, 1, 8, 33, 900, 64, 16),
])
def test_verify_many_and_long(b, h_kv, G, n, t, d, page):
    """Units that span many CTAs, more units than CTAs, 768 query rows a KV head."""
    pool = ref.Pool([t + n] * b, h_kv, page, d, seed=n)
    q = queries(b, h_kv * G, n, d, n)
    o, lse = run_verify(pool, q, t, n, ws_n=min(768 // G, n + 3) if n < 96 else n)
    check_verify(pool, q, [t] * b, n, o, lse)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n", [(4, 1), (4, 6), (8, 21)])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_pages_that_are_not_there(d, G, n, page):
    """Pages behind a window are gone, whole sequences' pages, pages inside a tile, the block's own; a query that sees nothing."""
    lens = [777, 64, 5, 300, 0]
    pool = ref.Pool([t + n for t in lens], 2, page, d, seed=n, cap=max(lens) + n)
    pool.table[0, 1:5] = torch.tensor([-1, -2, -2**31, -1], dtype=torch.int32)[:pool.table[0, 1:5].numel()]
    pool.table[1, :-(-(64 + n) // page)] = -1                      # nothing left at all
    pool.table[2, 0] = -1                                          # the first queries' rows
    pool.table[3, 300 // page] = -1                                # the first rows of the block
    q = queries(len(lens), 2 * G, n, d, n)
    o, lse = run_verify(pool, q, max(lens), n, lens)
    check_verify(pool, q, lens, n, o, lse)
    assert (lse[1] == -math.inf).all() and (o[1] == 0).all()


@pytest.mark.parametrize("d,n", [(64, 1), (128, 6), (128, 21)])
def test_entries_past_the_pool_are_recorded_and_hidden(d, n):
    t = 200
    pool = ref.Pool([t + n] * 2, 2, 16, d, seed=n)
    pool.table[0, 3] = len(pool.k)
    pool.table[1, 0] = 2**31 - 1
    q = queries(2, 8, n, d, n)
    o, lse = run_verify(pool, q, t, n, status=-1)
    check_verify(pool, q, [t] * 2, n, o, lse)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 6])
@pytest.mark.parametrize("G", [4, 8])
@pytest.mark.parametrize("case", ["large v", "sharp", "zero rows", "offset v", "late peak", "tiny q"])
def test_verify_sizes_of_values(d, n, G, case):
    t = 777
    pool = ref.Pool([t + n], 2, 32, d, seed=11)
    q = queries(1, 2 * G, n, d, 11).float()
    if case == "large v":
        pool.v = (pool.v.float() * 2.0 ** 60).to(BF)
    elif case == "sharp":
        q *= 8
    elif case == "zero rows":
        pool.k[:, :, ::3] = 0
        pool.v[:, :, ::2] = 0
        q[:, 0] = 0
    elif case == "offset v":
        pool.v = (pool.v.float() * 0.05 + 3).to(BF)
    elif case == "late peak":
        e = int(pool.table[0, (t - 5) // 32])
        pool.k[e, :, (t - 5) % 32] = (3 * q[0, ::G, 0]).to(BF)
    elif case == "tiny q":
        q *= 2.0 ** -20
        pool.k = (pool.k.float() * 2.0 ** 20).to(BF)
    q = q.to(BF)
    o, lse = run_verify(pool, q, t, n)
    check_verify(pool, q, [t], n, o, lse, case)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n", [(1, 6), (4, 6), (8, 4), (8, 8), (4, 21), (8, 21), (8, 33)])
@pytest.mark.parametrize("t", [0, 62, 127, 300])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_a_block_row_that_is_no_number_is_hidden_from_the_queries_before_it(d, G, n, t, bad):
    pool = ref.Pool([t + n] * 2, 1, 16, d, seed=n)
    q = queries(2, G, n, d, n)
    spots = {0: (3, 5), 1: (1, d - 1)}                             # sequence: the block's row, its column
    clean = pool.v.clone()
    for i, (row, col) in spots.items():
        e = int(pool.table[i, (t + row) // 16])
        pool.v[e, 0, (t + row) % 16, col] = bad
        clean[e, 0, (t + row) % 16, col] = 0
    o, lse = run_verify(pool, q, t, n)
    for i, (row, col) in spots.items():
        assert not torch.isfinite(o[i, :, row:, col]).any()
        o[i, :, row:, col] = 0
    pool.v = clean
    for i, (row, col) in spots.items():
        k, v, _ = pool.unit(i, 0, torch.arange(t + n))
        visible = torch.arange(t + n)[None, :] <= (t + torch.arange(n).repeat(G))[:, None]
        wo, wl, spread = ref.attend(q[i].reshape(G * n, d), k, v, visible)
        wo = wo.view(G, n, d)
        wo[:, row:, col] = 0
        ref.check(o[i].reshape(G * n, d), lse[i].reshape(-1), wo.view(G * n, d), wl, spread, f"seq {i}")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n", [(4, 1), (4, 6), (8, 21)])
@pytest.mark.parametrize("t", [40, 3000])
def test_what_is_no_number_reaches_those_who_see_it(d, G, n, t):
    """A NaN query; a NaN key and a NaN value in the context."""
    pool = ref.Pool([t + n] * 4, 1, 16, d, seed=n)
    q = queries(4, G, n, d, n)
    q[0, 0, 0, 7] = math.nan
    pool.k[int(pool.table[1, 1]), 0, 3, 9] = math.nan
    pool.v[int(pool.table[2, 1]), 0, 3, 9] = math.nan
    o, lse = run_verify(pool, q, t, n)
    assert o[0, 0, 0].isnan().all() and lse[0, 0, 0].isnan()
    assert o[1].isnan().all() and lse[1].isnan().all()
    assert o[2, :, :, 9].isnan().all() and torch.isfinite(lse[2]).all()
    rest = [c for c in range(d) if c != 9]
    assert torch.isfinite(o[2][..., rest]).all() and torch.isfinite(o[3]).all()
    if G > 1:
        assert torch.isfinite(o[0, 1:]).all()
    # a block row's NaN key: the queries before it do not see it
    if n > 2:
        pool = ref.Pool([t + n], 1, 16, d, seed=n)
        pool.k[int(pool.table[0, (t + 2) // 16]), 0, (t + 2) % 16] = math.nan
        o, lse = run_verify(pool, queries(1, G, n, d, n), t, n)
        assert torch.isfinite(o[0, :, :2]).all() and o[0, :, 2:].isnan().all() and lse[0, :, 2:].isnan().all()


def test_lengths_out_of_range_are_recorded_and_clamped():
    n, d = 2, 64
    pool = ref.Pool([50 + n] * 3, 2, 16, d, seed=n)
    q = queries(3, 4, n, d, n)
    o, lse = run_verify(pool, q, 50, n, [-1, 51, 7], status=-1)
    check_verify(pool, q, [0, 50, 7], n, o, lse)


def test_sequences_share_pages():
    n, d, t = 1, 128, 96
    pool = ref.Pool([t + n] * 3, 2, 16, d, seed=n)
    pool.table[1, :6] = pool.table[0, :6]
    pool.table[2, :3] = pool.table[0, 3:6]
    q = queries(3, 8, n, d, n)
    o, lse = run_verify(pool, q, t, n)
    check_verify(pool, q, [t] * 3, n, o, lse)


# ------------------------------------------------------------------------------------ drafter passes


def run_draft(pool, q, t, idx, count, budget, j, seq=None, flags=0, status=0, ws_bytes=None):
    K, V, table = pool.cuda()
    cache = bd.PagedCache(K, V)
    b, h_q, d = q.shape
    lens = None if seq is None else torch.tensor(seq, dtype=torch.int32, device="cuda")
    shape = cache.shape(b, h_q, t, pool.cap, lens)
    ws = bd.Workspace(ws_bytes or bd.bd_workspace_size(shape, bd.BD_OP_PAGED_DRAFT, budget, j + 1))
    o = torch.full(q.shape, 7.0, dtype=BF, device="cuda")
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    dev = q.cuda(), idx.cuda(), count.cuda()
    torch.cuda.synchronize()
    for _ in range(2):
        bd.bd_paged_draft_attn(shape, dev[0], cache, table, dev[1], dev[2], budget, j, o, lse, ws, flags=flags)
    torch.cuda.synchronize()
    assert ws.status() == status
    return o.cpu(), lse.cpu()


def view(b, h_kv, budget, lens, seed):
    g = torch.Generator().manual_seed(seed)
    idx = torch.full((b, h_kv, budget), -1, dtype=torch.int32)
    count = torch.zeros(b, h_kv, dtype=torch.int32)
    for i in range(b):
        for h in range(h_kv):
            n = min(budget, lens[i])
            idx[i, h, :n] = torch.randperm(lens[i], generator=g)[:n].sort().values.int() if lens[i] else idx[i, h, :n]
            count[i, h] = n
    return idx, count


def check_draft(pool, q, lens, idx, count, j, o, lse):
    b, h_q, d = q.shape
    h_kv = pool.k.shape[1]
    G = h_q // h_kv
    for i in range(b):
        for h in range(h_kv):
            kept = idx[i, h, :int(count[i, h])].long()
            kept = kept[(kept >= 0) & (kept < lens[i])]
            k, v, there = pool.unit(i, h, torch.cat([kept, lens[i] + torch.arange(j + 1)]))
            hs = slice(h * G, (h + 1) * G)
            want = ref.attend(q[i, hs], k, v, there[None, :].expand(G, -1))
            ref.check(o[i, hs], lse[i, hs], *want, f"seq {i} head {h}")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 4, 8, 16, 5])
@pytest.mark.parametrize("budget,j", [(1, 0), (64, 3), (300, 0), (2000, 19)])
@pytest.mark.parametrize("page,layout", [(16, "heads"), (64, "rows")])
@pytest.mark.parametrize("lens", [[2100, 2100], [2100, 0, 17]])
@pytest.mark.parametrize("flags", [0, bd.BD_DRAFT_VIEW_READY])
def test_draft(d, G, budget, j, page, layout, lens, flags):
    b, h_kv = len(lens), 2
    pool = ref.Pool([t + j + 1 for t in lens], h_kv, page, d, seed=budget, layout=layout, cap=max(lens) + j + 1)
    q = queries(b, h_kv * G, 1, d, 3)[:, :, 0].contiguous()
    idx, count = view(b, h_kv, budget, lens, 5)
    o, lse = run_draft(pool, q, max(lens), idx, count, budget, j, lens if len(set(lens)) > 1 else None, flags)
    check_draft(pool, q, lens, idx, count, j, o, lse)


@pytest.mark.parametrize("b,h_kv,G,budget,t,d", [(1, 1, 8, 8192, 9000, 128), (2, 4, 4, 8000, 8200, 64), (24, 8, 4, 512, 600, 128),
                                                (1, 1, 16, 20000, 20500, 128)])
def test_draft_many_and_long(b, h_kv, G, budget, t, d):
    pool = ref.Pool([t + 2] * b, h_kv, 16, d, seed=budget)
    q = queries(b, h_kv * G, 1, d, 3)[:, :, 0].contiguous()
    idx, count = view(b, h_kv, budget, [t] * b, 5)
    o, lse = run_draft(pool, q, t, idx, count, budget, 1)
    check_draft(pool, q, [t] * b, idx, count, 1, o, lse)
    # a workspace of the header and the counters alone: one cluster a unit
    o, lse = run_draft(pool, q, t, idx, count, budget, 1, ws_bytes=256 + (4 * b * h_kv + 255) // 256 * 256)
    check_draft(pool, q, [t] * b, idx, count, 1, o, lse)


@pytest.mark.parametrize("d", [64, 128])
def test_draft_skips_what_is_not_there(d):
    """Absent pages of kept and drafted positions (no error), entries past the pool and indices past the context (errors)."""
    t, j, budget = 300, 5, 128
    pool = ref.Pool([t + j + 1] * 3, 2, 16, d, seed=1)
    pool.table[0, 2:9] = -1
    pool.table[1, :] = -1
    pool.table[2, -1] = -1
    q = queries(3, 8, 1, d, 3)[:, :, 0].contiguous()
    idx, count = view(3, 2, budget, [t] * 3, 5)
    o, lse = run_draft(pool, q, t, idx, count, budget, j)
    check_draft(pool, q, [t] * 3, idx, count, j, o, lse)
    assert (lse[1] == -math.inf).all() and (o[1] == 0).all()
    pool.table[0, 4] = len(pool.k)
    run_draft(pool, q, t, idx, count, budget, j, status=-1)
    pool.table[0, 4] = -1
    idx[0, 0, 5], idx[2, 1, 0] = t, -9
    o, lse = run_draft(pool, q, t, idx, count, budget, j, status=-1)
    check_draft(pool, q, [t] * 3, idx, count, j, o, lse)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("budget", [40, 3000])
def test_draft_keeps_nan(d, budget):
    t = 3200
    pool = ref.Pool([t + 1] * 4, 1, 16, d, seed=1)
    q = queries(4, 4, 1, d, 3)[:, :, 0].contiguous()
    idx, count = view(4, 1, budget, [t] * 4, 5)
    at = [int(idx[i, 0, 7]) for i in range(4)]
    q[0, 0, 3] = math.nan
    pool.k[int(pool.table[1, at[1] // 16]), 0, at[1] % 16, 3] = math.nan
    pool.v[int(pool.table[2, at[2] // 16]), 0, at[2] % 16, 3] = math.nan
    o, lse = run_draft(pool, q, t, idx, count, budget, 0)
    assert o[0, 0].isnan().all() and lse[0, 0].isnan() and torch.isfinite(o[0, 1:]).all()
    assert o[1].isnan().all() and lse[1].isnan().all()
    assert o[2, :, 3].isnan().all() and torch.isfinite(o[2][:, 4:]).all() and torch.isfinite(lse[2]).all()
    assert torch.isfinite(o[3]).all()
