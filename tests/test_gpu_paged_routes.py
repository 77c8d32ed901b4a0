"""Verify blocks over a paged cache on every route: clusters (few short units), the tile list cut over the GPU (many or long
units; up to 8 rows, at head_dim 64 up to 24) and the tensor-memory kernel; each with pages that are not there, unequal lengths,
rows that are no number."""

import math

import pytest
import torch

from tests import paged_reference as ref
from tests.test_gpu_paged_attn import queries, run_verify

pytestmark = pytest.mark.gpu


def check_some(pool, q, lens, n, o, lse, some, heads=None):
    b, h_q, _, d = q.shape
    h_kv = pool.k.shape[1]
    G = h_q // h_kv
    for i in some:
        rows = torch.arange(lens[i] + n)
        for h in heads if heads is not None else range(h_kv):
            k, v, there = pool.unit(i, h, rows)
            hs = slice(h * G, (h + 1) * G)
            visible = (rows[None, :] <= (lens[i] + torch.arange(n).repeat(G))[:, None]) & there[None, :]
            want = ref.attend(q[i, hs].reshape(G * n, d), k, v, visible)
            ref.check(o[i, hs].reshape(G * n, d), lse[i, hs].reshape(-1), *want, f"seq {i} head {h}")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n", [(4, 1), (8, 1), (4, 2), (4, 4), (4, 6), (4, 9), (8, 21)])
@pytest.mark.parametrize("page", [16, 64, 256])
def test_many_units_of_equal_lengths(d, G, n, page):
    b, h_kv, t = 42, 8, 150
    pool = ref.Pool([t + n] * b, h_kv, page, d, seed=n, cap=t + n + 9)
    q = queries(b, h_kv * G, n, d, n)
    o, lse = run_verify(pool, q, t, n)
    check_some(pool, q, [t] * b, n, o, lse, (0, 17, b - 1), (0, 3, 7))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n", [(4, 1), (4, 2), (4, 6), (8, 21)])
@pytest.mark.parametrize("page", [16, 32, 128])
def test_many_units_of_unequal_lengths_with_absent_pages(d, G, n, page):
    base = [777, 64, 5, 300, 0, 129, 1, 256]
    lens, h_kv = base * 40, 1
    pool = ref.Pool([t + n for t in lens], h_kv, page, d, seed=n, cap=max(lens) + n)
    for i in range(0, len(lens), 8):
        pool.table[i, 1:5] = -1
        pool.table[i + 1, :-(-(64 + n) // page)] = -1
        pool.table[i + 2, 0] = -5
        pool.table[i + 3, 300 // page] = -1
    q = queries(len(lens), h_kv * G, n, d, n)
    o, lse = run_verify(pool, q, max(lens), n, lens)
    check_some(pool, q, lens, n, o, lse, [*range(8), *range(152, 160), *range(312, 320)])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n,t", [(4, 1, 30000), (8, 1, 9000), (4, 4, 30000), (4, 6, 20000), (8, 21, 9000)])
@pytest.mark.parametrize("page", [16, 128])
def test_long_units(d, G, n, t, page):
    """Units that span many CTAs, with pages gone behind a window and inside it."""
    pool = ref.Pool([t + n, t // 2 + n], 1, page, d, seed=n, cap=t + n)
    gone = slice(t // page // 8, t // page // 2)
    pool.table[0, gone] = -1
    pool.table[1, 3:9] = -1
    q = queries(2, G, n, d, n)
    o, lse = run_verify(pool, q, t, n, [t, t // 2])
    check_some(pool, q, [t, t // 2], n, o, lse, (0, 1))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n", [(4, 2), (1, 6), (4, 6), (8, 21)])
@pytest.mark.parametrize("b", [2, 320])
def test_no_number_in_a_block_row_on_every_route(d, G, n, b):
    t, row, col = 62, 1, 5
    pool = ref.Pool([t + n] * b, 1, 16, d, seed=n)
    q = queries(b, G, n, d, n)
    clean = pool.v.clone()
    for i in (0, b - 1):
        e = int(pool.table[i, (t + row) // 16])
        pool.v[e, 0, (t + row) % 16, col] = math.nan
        clean[e, 0, (t + row) % 16, col] = 0
    # and a key that is no number, of the second sequence's block
    pool.k[int(pool.table[1 if b > 2 else 0, (t + n - 1) // 16]), 0, (t + n - 1) % 16, 0] = math.nan
    o, lse = run_verify(pool, q, t, n)
    for i in (0, b - 1):
        assert o[i, :, row:n - 1, col].isnan().all() and torch.isfinite(o[i, :, :row]).all()
    bad = 1 if b > 2 else 0
    assert o[bad, :, n - 1].isnan().all() and lse[bad, :, n - 1].isnan().all()
    assert torch.isfinite(lse[bad, :, :n - 1]).all()
    if b > 2:
        assert torch.isfinite(o[1:-1, :, :n - 1]).all() and torch.isfinite(o[2:-1]).all()
        check_some(pool, q, [t] * b, n, o, lse, (2, 100, b - 2))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n", [(4, 1), (8, 1), (4, 2), (4, 4), (4, 6)])
@pytest.mark.parametrize("b,t,page", [(2, 6000, 16), (24, 3000, 64), (40, 1500, 128)])
def test_what_is_left_behind_a_window(d, G, n, b, t, page):
    """Many tiles in a row that are not there: behind the first page, in the middle, at the end, all but one, all."""
    h_kv = 8
    pool = ref.Pool([t + n] * b, h_kv, page, d, seed=t + n)
    per = pool.table.shape[1]
    for i in range(b):
        kind = i % 6
        if kind == 0:
            pool.table[i, 1:per - 2] = -1
        elif kind == 1:
            pool.table[i, per // 3:per // 2] = -1
        elif kind == 2:
            pool.table[i, per // 2:] = -1
        elif kind == 3:
            pool.table[i, torch.arange(per) != per // 2] = -1
        elif kind == 4:
            pool.table[i, ::2] = -1
        else:
            pool.table[i] = -1
    q = queries(b, h_kv * G, n, d, 3)
    o, lse = run_verify(pool, q, t, n)
    check_some(pool, q, [t] * b, n, o, lse, range(min(6, b)), (0, 5))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n", [(4, 6), (8, 4), (8, 21)])
@pytest.mark.parametrize("page", [16, 32, 256])
def test_stale_tiles_behind_a_window(d, G, n, page):
    """Long units whose middle, end or block is not there, after units that are whole and hold NaN in rows that are hidden: what
    lay in shared memory before has no part in them.  A block's rows among what is there, and not."""
    b, h_kv, t = 6, 4, 9000
    pool = ref.Pool([t + n] * b, h_kv, page, d, seed=n)
    per = pool.table.shape[1]
    for i, (lo, hi) in enumerate([(0, 0), (1, per - 1), (0, 0), (3, per), (per // 4, per - per // 8), (0, per)]):
        pool.table[i, lo:hi] = -1
    for i in (0, 2):                       # the block's last V row: hidden from its first queries, seen by the last
        pool.v[int(pool.table[i, (t + n - 1) // page]), :, (t + n - 1) % page] = math.nan
    q = queries(b, h_kv * G, n, d, n)
    o, lse = run_verify(pool, q, t, n)
    assert not torch.isnan(o[[1, 3, 4, 5]].float()).any() and (o[5] == 0).all() and (lse[5] == -math.inf).all()
    for i in (0, 2):
        assert torch.isnan(o[i, :, -1].float()).all() and not torch.isnan(o[i, :, :-1].float()).any()
    check_some(pool, q, [t] * b, n, o, lse, (1, 3, 4), (0, 3))
