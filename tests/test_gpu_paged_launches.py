"""Verify blocks over a paged cache, each route by the kernels that it launches (clusters of one and several CTAs and with query
rows in chunks, the tile list with one and three n8 tiles, the tensor-memory kernel with one and two M tiles, with boxes of 16 whole
rows and of halves), in pages of 16 to 4096 rows, some of them gone; against 64 bits."""

import re

import pytest
import torch

import paper_2606_00144_gb300 as bd
from tests import paged_reference as ref
from tests.launched import kernels
from tests.test_gpu_paged_attn import queries, run_verify
from tests.test_gpu_paged_routes import check_some

pytestmark = pytest.mark.gpu
BF = torch.bfloat16

CLUSTER, STREAM, TENSOR = "cluster", "stream", "tensor memory"


def route(name, grid):
    m = re.match(r"_ZN2bd19paged_verify_kernelILi(\d+)ELi(\d)ELb(\d)E", name)
    if m:
        return (int(m[1]), CLUSTER if m[3] == "1" else STREAM, int(m[2]), grid[:2] if m[3] == "1" else None)
    m = re.match(r"_ZN2bd16verify_tc_kernelILi(\d+)ELi(\d)ELb0ELi(\d)E", name)
    return (int(m[1]), TENSOR, int(m[2]), int(m[3]))


# batch, KV heads, group, context, block; then, for head_dim 64 and 128, what runs: the kernel, its tiles of query rows, and a
# cluster's grid (CTAs of a unit, units)
CASES = [
    (42, 8, 4, 150, 1, (CLUSTER, 1, (1, 336)), (CLUSTER, 1, (1, 336))),
    (42, 8, 4, 150, 6, (STREAM, 3, None), (CLUSTER, 1, (1, 1008))),
    (1, 2, 4, 1000, 1, (CLUSTER, 1, (8, 2)), (CLUSTER, 1, (8, 2))),
    (1, 2, 4, 30000, 1, (STREAM, 1, None), (STREAM, 1, None)),
    (1, 2, 4, 30000, 6, (STREAM, 3, None), (TENSOR, 1, None)),
    (42, 8, 4, 150, 9, (TENSOR, 1, None), (TENSOR, 1, None)),
    (2, 1, 8, 9000, 21, (TENSOR, 2, None), (TENSOR, 2, None)),
    (1, 2, 4, 2500, 150, (TENSOR, 2, None), (TENSOR, 2, None)),           # 600 rows: three chunks
]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 64, 512, 4096])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c[:5])))
def test_the_route_and_its_results(case, page, d):
    b, h_kv, G, t, n = case[:5]
    kernel, tiles, grid = case[5 if d == 64 else 6]
    pool = ref.Pool([t + n] * b, h_kv, page, d, seed=n, cap=t + n)
    pages = pool.table.shape[1]
    pool.table[0, 1:max(1, pages * 2 // 3)] = -1             # behind a window
    if b > 1:
        pool.table[b - 1, 0] = -1
    q = queries(b, h_kv * G, n, d, n)
    K, V, table = pool.cuda()
    cache, o = bd.PagedCache(K, V), torch.empty(b, h_kv * G, n, d, dtype=BF, device="cuda")
    shape = cache.shape(b, h_kv * G, t, pool.cap)
    ws, dev = bd.Workspace(bd.bd_workspace_size(shape, bd.BD_OP_PAGED_VERIFY, 0, n)), q.cuda()
    bd.bd_paged_verify_attn(shape, dev, n, cache, table, o, None, ws)
    launched = kernels(lambda: bd.bd_paged_verify_attn(shape, dev, n, cache, table, o, None, ws))
    boxes = (2 if page == 16 and d == 128 else 1) if kernel == TENSOR else grid
    assert route(*launched[0]) == (d, kernel, tiles, boxes), launched
    assert len(launched) == (1 if kernel == CLUSTER else 2)
    o, lse = run_verify(pool, q, t, n)
    check_some(pool, q, [t] * b, n, o, lse, {0, b - 1}, (0, h_kv - 1))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [512, 2048])
@pytest.mark.parametrize("n", [1, 6, 21])
def test_unequal_lengths_in_large_pages(d, page, n):
    lens = [5000, 511, 512, 1, 0, 4095, 2047]
    pool = ref.Pool([t + n for t in lens], 2, page, d, seed=n, cap=5000 + n)
    pool.table[0, 1] = -1
    q = queries(len(lens), 16, n, d, n)
    o, lse = run_verify(pool, q, 5000, n, lens)
    check_some(pool, q, lens, n, o, lse, range(len(lens)))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("page", [512, 2048])
def test_rows_join_and_come_back_in_large_pages(d, dtype, page):
    lens, n, h_q, h_kv = [3000, 510, 0], 5, 4, 2
    pool = ref.Pool([t + n for t in lens], h_kv, page, d, seed=7, cap=3000 + n)
    K, V, table = pool.cuda()
    cache, g = bd.PagedCache(K, V), torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(3, h, n, d, generator=g).to(dtype) for h in (h_q, h_kv, h_kv))
    q_out = torch.empty(3, h_q, n, d, dtype=BF, device="cuda")
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda")        # (a shape holds its address alone)
    shape = cache.shape(3, h_q, 3000, pool.cap, seq)
    freq = 10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)
    bd.bd_paged_append(shape, q.cuda(), k.cuda(), v.cuda(), bd.Rope(freq), cache, table, q_out)
    back_k, back_v = (torch.zeros(3, h_kv, n, d, dtype=BF, device="cuda") for _ in "kv")
    bd.bd_paged_read(shape, cache, table, back_k, back_v)
    context = torch.full((3, h_kv, 3000, d), 7.0, dtype=BF, device="cuda")
    bd.bd_paged_read(shape, cache, table, context, first_row=0)
    for i, t in enumerate(lens):
        for got, rows in ((q_out, q), (back_k, k)):
            want = ref.rotate(rows[i], t + torch.arange(n), freq, False)
            assert ((got[i].cpu().double() - want).abs() <= ref.rotate_tolerance(rows[i], want, freq, False)).all()
        assert torch.equal(back_v[i].cpu(), v[i].to(BF))
        for h in range(h_kv):
            assert torch.equal(context[i, h, :t].cpu().double(), pool.unit(i, h, torch.arange(t))[0])
        assert (context[i, :, t:] == 7).all()
