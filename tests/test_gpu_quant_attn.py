"""Attention over a 4-bit cache on the GPU against 64 bits: verify blocks (one query to the longest),
drafter passes, at the lengths, masks and scales where a kernel can go wrong."""

import math

import pytest
import torch

import paper_2606_00144_gb300 as bd
from tests import quant_reference as ref

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def make_cache(b, h_kv, cap, d, seed=0, k_size=1.0, v_size=1.0):
    g = torch.Generator().manual_seed(seed)
    out = []
    for size in (k_size, v_size):
        x = torch.randn(b, h_kv, cap, d, generator=g) * size
        out += ref.quantise(x.to(BF))
    return out


def spoil(tensors, lens, n):
    """NaN scales and arbitrary codes in every row past a sequence's own block."""
    for i, t in enumerate(lens):
        for codes in tensors[0::2]:
            codes[i, :, t + n:] = 0x0f
        for scales in tensors[1::2]:
            scales[i, :, t + n:] = math.nan


def run_verify(tensors, q, t, n, seq=None, ws_n=None, stream=None):
    b, h_kv, cap = tensors[0].shape[:3]
    cache = bd.QuantCache(*(x.cuda() for x in tensors))
    h_q = q.shape[1]
    shape = cache.shape(h_q, t, seq)
    ws = bd.Workspace(bd.bd_workspace_size(shape, bd.BD_OP_QUANT_VERIFY, 0, ws_n or n))
    o = torch.full(q.shape, 7.0, dtype=BF, device="cuda")
    lse = torch.full(q.shape[:3], 7.0, dtype=torch.float32, device="cuda")
    bd.bd_quant_verify_attn(shape, q.cuda(), n, cache, o, lse, ws, stream)
    first = o.clone()
    bd.bd_quant_verify_attn(shape, q.cuda(), n, cache, o, lse, ws, stream)      # the workspace is left as it was
    assert ws.status() == 0
    assert torch.equal(first, o)
    return o, lse


def check_verify(tensors, q, lens, n, o, lse, what=""):
    b, h_q, _, d = q.shape
    h_kv = tensors[0].shape[1]
    G = h_q // h_kv
    for i in range(b):
        t = lens[i]
        for h in range(h_kv):
            k = ref.values(tensors[0][i, h, :t + n], tensors[1][i, h, :t + n])
            v = ref.values(tensors[2][i, h, :t + n], tensors[3][i, h, :t + n])
            hs = slice(h * G, (h + 1) * G)
            lim = t + torch.arange(n).repeat(G)
            visible = torch.arange(t + n)[None, :] <= lim[:, None]
            wo, wl, spread = ref.attend(q[i, hs].reshape(G * n, d), k, v, visible)
            ref.check(o[i, hs].reshape(G * n, d), lse[i, hs].reshape(-1), wo, wl, spread, v.abs().max(), f"{what} seq {i} head {h}")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n", [(1, 1), (4, 1), (4, 2), (8, 2), (4, 6), (1, 17), (8, 4), (8, 5), (3, 21), (8, 21), (8, 25), (16, 3)])
@pytest.mark.parametrize("t", [0, 1, 15, 127, 128, 130, 1000])
def test_verify_lengths(d, G, n, t):
    b, h_kv = 2, 2
    tensors = make_cache(b, h_kv, t + n + 3, d, seed=t + 7 * n)
    spoil(tensors, [t] * b, n)
    q = torch.randn(b, h_kv * G, n, d, generator=torch.Generator().manual_seed(n)).to(BF)
    o, lse = run_verify(tensors, q, t, n)
    check_verify(tensors, q, [t] * b, n, o, lse)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n", [(4, 1), (4, 6), (8, 21), (1, 6)])
@pytest.mark.parametrize("lens", [[0, 1, 2, 700], [513, 0, 129, 128], [5000, 31, 4999, 64], [3, 3, 3, 3]])
def test_verify_unequal_lengths(d, G, n, lens):
    b, h_kv, t = len(lens), 2, max(lens)
    tensors = make_cache(b, h_kv, t + n + 1, d, seed=sum(lens))
    spoil(tensors, lens, n)
    q = torch.randn(b, h_kv * G, n, d, generator=torch.Generator().manual_seed(n)).to(BF)
    o, lse = run_verify(tensors, q, t, n, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    check_verify(tensors, q, lens, n, o, lse)


@pytest.mark.parametrize("b,h_kv,G,n,t,d", [
    (1, 1, 4, 6, 40000, 128), (1, 2, 8, 1, 33001, 64), (5, 4, 4, 6, 2049, 128), (40, 8, 4, 6, 260, 128),
    (40, 8, 1, 1, 517, 64), (2, 2, 8, 96, 300, 128), (1, 1, 8, 96, 5000, 64), (3, 4, 8, 21, 4100, 128),
])
def test_verify_many_and_long(b, h_kv, G, n, t, d):
    """Units that span many CTAs, more units than CTAs, 768 query rows a KV head."""
    tensors = make_cache(b, h_kv, t + n, d, seed=n)
    q = torch.randn(b, h_kv * G, n, d, generator=torch.Generator().manual_seed(n)).to(BF)
    o, lse = run_verify(tensors, q, t, n, ws_n=min(768 // G, n + 3) if n < 96 else n)
    check_verify(tensors, q, [t] * b, n, o, lse)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 6])
@pytest.mark.parametrize("case", ["tiny v", "large v", "mixed v", "sharp", "zero rows", "mixed k", "offset v", "late peak", "tiny q"])
def test_verify_sizes_of_values(d, n, case):
    """V and K of any size, scales that change by many octaves from row to row, near one-hot softmax,
    a peak that arrives late, V with an offset (the codes' own must cancel)."""
    b, h_kv, G, t = 1, 2, 4, 777
    g = torch.Generator().manual_seed(11)
    k, v = (torch.randn(b, h_kv, t + n, d, generator=g) for _ in range(2))
    q = torch.randn(b, h_kv * G, n, d, generator=g)
    step = torch.exp2(torch.randint(-12, 13, (b, h_kv, t + n, 1), generator=g).float())
    if case == "tiny v":
        v *= 2.0 ** -60
    elif case == "large v":
        v *= 2.0 ** 60
    elif case == "mixed v":
        v *= step
    elif case == "sharp":
        q *= 8
    elif case == "zero rows":
        k[:, :, ::3] = 0
        v[:, :, ::2] = 0
        v[:, :, :40] = 0
        q[:, 0] = 0
    elif case == "mixed k":
        k *= torch.exp2(torch.randint(-12, 2, (b, h_kv, t + n, 1), generator=g).float())
    elif case == "offset v":
        v = v * 0.05 + 3
    elif case == "late peak":
        k[:, :, -n - 5] = 3 * q[:, ::G, 0]
    elif case == "tiny q":
        q *= 2.0 ** -20
        k *= 2.0 ** 20
    tensors = [x for y in (k, v) for x in ref.quantise(y.to(BF))]
    q = q.to(BF)
    o, lse = run_verify(tensors, q, t, n)
    check_verify(tensors, q, [t] * b, n, o, lse, case)


def test_a_nan_in_a_row_or_a_query_stays_where_it_belongs():
    b, h_kv, G, n, t, d = 2, 2, 4, 6, 300, 128
    tensors = make_cache(b, h_kv, t + n, d)
    q = torch.randn(b, h_kv * G, n, d, generator=torch.Generator().manual_seed(1)).to(BF)
    tensors[1][0, 1, 17, 2] = math.nan                       # a K group: every query of that head sees it
    tensors[3][1, 0, t + 3, 1] = math.nan                    # a V group of the block's fourth row
    q[1, 6, 2, 5] = math.nan
    o, lse = (x.cpu() for x in run_verify_nan(tensors, q, t, n))
    assert o[0, G:].isnan().all() and lse[0, G:].isnan().all() and torch.isfinite(o[0, :G]).all()
    assert o[1, :G, 3:, 32:64].isnan().all() and torch.isfinite(o[1, :G, 3:, :32]).all()
    assert torch.isfinite(lse[1, :G]).all()
    assert o[1, 6, 2].isnan().all() and torch.isfinite(o[1, 6, 1]).all() and torch.isfinite(o[1, 7]).all()


def run_verify_nan(tensors, q, t, n):
    cache = bd.QuantCache(*(x.cuda() for x in tensors))
    shape = cache.shape(q.shape[1], t)
    ws = bd.Workspace(bd.bd_workspace_size(shape, bd.BD_OP_QUANT_VERIFY, 0, n))
    o, lse = torch.empty_like(q, device="cuda"), torch.empty(q.shape[:3], device="cuda")
    bd.bd_quant_verify_attn(shape, q.cuda(), n, cache, o, lse, ws)
    torch.cuda.synchronize()
    return o, lse


def test_a_length_outside_the_shape_is_recorded():
    b, h_kv, G, n, t, d = 3, 1, 4, 2, 50, 64
    tensors = make_cache(b, h_kv, t + n, d)
    q = torch.randn(b, h_kv * G, n, d).to(BF)
    cache = bd.QuantCache(*(x.cuda() for x in tensors))
    seq = torch.tensor([20, 51, -1], dtype=torch.int32, device="cuda")
    shape = cache.shape(h_kv * G, t, seq)
    ws = bd.Workspace(bd.bd_workspace_size(shape, bd.BD_OP_QUANT_VERIFY, 0, n))
    o, lse = torch.empty_like(q, device="cuda"), torch.empty(q.shape[:3], device="cuda")
    bd.bd_quant_verify_attn(shape, q.cuda(), n, cache, o, lse, ws)
    assert ws.status() == -1 and ws.status() == 0
    check_verify(tensors, q, [20, 50, 0], n, o, lse)


# ------------------------------------------------------------------------------------ drafter passes


def run_draft(tensors, q, t, idx, count, j, seq=None, flags=0):
    cache = bd.QuantCache(*(x.cuda() for x in tensors))
    shape = cache.shape(q.shape[1], t, seq)
    budget = idx.shape[-1]
    ws = bd.Workspace(bd.bd_workspace_size(shape, bd.BD_OP_QUANT_DRAFT, budget, j + 1))
    o = torch.full(q.shape, 7.0, dtype=BF, device="cuda")
    lse = torch.full(q.shape[:2], 7.0, dtype=torch.float32, device="cuda")
    args = (shape, q.cuda(), cache, idx.cuda(), count.cuda(), budget, j, o, lse, ws)
    bd.bd_quant_draft_attn(*args, flags=flags)
    first = o.clone()
    bd.bd_quant_draft_attn(*args, flags=flags)
    assert torch.equal(first, o)
    return o, lse, ws.status()


def check_draft(tensors, q, lens, idx, count, j, o, lse):
    b, h_q, d = q.shape
    h_kv = tensors[0].shape[1]
    G = h_q // h_kv
    for i in range(b):
        for h in range(h_kv):
            kept = idx[i, h, :count[i, h]].long()
            kept = kept[(kept >= 0) & (kept < lens[i])]
            rows = torch.cat([kept, lens[i] + torch.arange(j + 1)])
            k, v = (ref.values(tensors[2 * x][i, h, rows], tensors[2 * x + 1][i, h, rows]) for x in (0, 1))
            hs = slice(h * G, (h + 1) * G)
            wo, wl, spread = ref.attend(q[i, hs], k, v, torch.ones(G, len(rows), dtype=torch.bool))
            ref.check(o[i, hs], lse[i, hs], wo, wl, spread, v.abs().max(), f"seq {i} head {h}")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 4, 7, 8, 16])
@pytest.mark.parametrize("t,budget,j", [(1, 1, 0), (40, 33, 2), (300, 128, 0), (1000, 700, 19), (9000, 8192, 5)])
def test_draft_views(d, G, t, budget, j):
    b, h_kv = 2, 2
    tensors = make_cache(b, h_kv, t + j + 1 + 2, d, seed=budget)
    spoil(tensors, [t] * b, j + 1)
    g = torch.Generator().manual_seed(budget)
    idx = torch.full((b, h_kv, budget), -1, dtype=torch.int32)
    count = torch.empty(b, h_kv, dtype=torch.int32)
    for i in range(b):
        for h in range(h_kv):
            n = [budget, 0, budget // 2, max(0, budget - 1)][2 * i + h]
            idx[i, h, :n] = torch.randperm(t, generator=g)[:n].sort().values.int()
            count[i, h] = n
    q = torch.randn(b, h_kv * G, d, generator=g).to(BF)
    o, lse, status = run_draft(tensors, q, t, idx, count, j)
    assert status == 0
    check_draft(tensors, q, [t] * b, idx, count, j, o, lse)


@pytest.mark.parametrize("d", [64, 128])
def test_draft_unequal_lengths_and_bad_entries(d):
    """Unsorted and repeated positions are used as they are; those outside a sequence's context are skipped
    and recorded, like a count outside the budget."""
    lens, h_kv, G, j, budget = [90, 1, 0, 61], 2, 4, 3, 50
    b, t = len(lens), 90
    tensors = make_cache(b, h_kv, t + j + 1, d, seed=3)
    spoil(tensors, lens, j + 1)
    g = torch.Generator().manual_seed(2)
    idx = torch.stack([torch.randint(0, max(n, 1), (h_kv, budget), generator=g, dtype=torch.int32) for n in lens])
    count = torch.tensor([[50, 17], [1, 0], [0, 0], [33, 50]], dtype=torch.int32)
    q = torch.randn(b, h_kv * G, d, generator=g).to(BF)
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
    o, lse, status = run_draft(tensors, q, t, idx, count, j, seq)
    assert status == 0
    check_draft(tensors, q, lens, idx, count, j, o, lse)
    idx[0, 0, 5], idx[3, 1, 49], idx[3, 0, 0] = 90, -1, 2 ** 31 - 1
    o, lse, status = run_draft(tensors, q, t, idx, count, j, seq)
    assert status == -1
    check_draft(tensors, q, lens, idx, count, j, o, lse)
    count[0, 1] = 51
    o, lse, status = run_draft(tensors, q, t, idx, count, j, seq)
    count[0, 1] = 50
    assert status == -1
    check_draft(tensors, q, lens, idx, count, j, o, lse)


@pytest.mark.parametrize("b,h_kv,budget", [(8, 8, 512), (16, 32, 300), (1, 1, 30000)])
def test_draft_few_and_many_units(b, h_kv, budget):
    G, j, d, t = 4, 4, 128, budget + 77
    tensors = make_cache(b, h_kv, t + j + 1, d, seed=1)
    g = torch.Generator().manual_seed(9)
    idx = torch.rand(b, h_kv, t, generator=g).topk(budget, -1).indices.sort(-1).values.int()
    count = torch.full((b, h_kv), budget, dtype=torch.int32)
    q = torch.randn(b, h_kv * G, d, generator=g).to(BF)
    o, lse, status = run_draft(tensors, q, t, idx, count, j, flags=bd.BD_DRAFT_VIEW_READY)
    assert status == 0
    some = slice(0, 1)
    check_draft([x[some] for x in tensors], q[some], [t], idx[some], count[some], j, o[some], lse[some])
    check_draft([x[-1:] for x in tensors], q[-1:], [t], idx[-1:], count[-1:], j, o[-1:], lse[-1:])
