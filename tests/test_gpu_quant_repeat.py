"""The tensor-memory kernel's merges, over and over: CTAs whose warpgroups end a segment with different numbers of tiles,
units of one tile next to long ones, maxima that grow from tile to tile.  Every call gives the first one's bits, and the
first is right."""

import pytest
import torch

import paper_2606_00144_gb300 as bd
from tests import quant_reference as ref
from tests.test_gpu_quant_attn import BF, check_verify
from tests.test_gpu_quant_attn_long import room, run

pytestmark = pytest.mark.gpu
REPEATS = 60


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n", [(1, 1), (4, 6), (8, 4), (8, 8), (4, 21), (8, 21)])
@pytest.mark.parametrize("grow", [False, True])
def test_every_call_gives_the_same_bits(d, G, n, grow):
    lens = [0, 130, 700, 1500, 2999, 64]
    b, t = len(lens), max(lens)
    g = torch.Generator().manual_seed(n)
    k, v = (torch.randn(b, 1, t + n, d, generator=g) for _ in range(2))
    q = torch.randn(b, G, n, d, generator=g)
    if grow:
        k[..., :8] *= 1 + torch.arange(t + n).view(1, 1, -1, 1) / 128   # a tile's scores spread further than the one's before
    tensors = [x for y in (k, v) for x in ref.quantise(y.to(BF))]
    q = q.to(BF)
    cap = room(G * n, d) + n
    cache = bd.QuantCache.empty(b, 1, cap, d)
    for whole, x in zip((cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales), tensors):
        whole.zero_()
        whole[:, :, :t + n] = x.cuda()
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
    shape = cache.shape(G, cap - n, seq)
    ws = bd.Workspace(bd.bd_workspace_size(shape, bd.BD_OP_QUANT_VERIFY, 0, n))
    qd = q.cuda()
    o, lse = torch.empty_like(qd), torch.empty(q.shape[:3], device="cuda")
    bd.bd_quant_verify_attn(shape, qd, n, cache, o, lse, ws)
    first = o.clone(), lse.clone()
    same = torch.ones((), dtype=torch.bool, device="cuda")
    for _ in range(REPEATS):
        o.fill_(7.0)
        bd.bd_quant_verify_attn(shape, qd, n, cache, o, lse, ws)
        same &= (o == first[0]).all() & (lse == first[1]).all()
    assert ws.status() == 0
    assert same.item()
    check_verify(tensors, q, lens, n, first[0], first[1])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n", [(1, 8), (4, 6), (4, 8), (8, 8), (4, 21)])
def test_maxima_that_grow_with_every_tile(d, G, n):
    """Every tile raises some row's maximum by more than it may trail, in every instance: the path that single lanes
    write from."""
    t = 2600
    g = torch.Generator().manual_seed(G + n)
    k, v = torch.randn(2, 1, t + n, d, generator=g) * 0.1, torch.randn(2, 1, t + n, d, generator=g)
    q = torch.randn(2, G, n, d, generator=g)
    q[..., 0] = 8.0
    k[..., 0] = torch.arange(t + n) // 128 * 6.5 * d ** 0.5 / 8        # 6.5 nats a tile: 9.4 in log2 units
    k[..., 1:32] = 0                                         # (a scale's group of its own)
    tensors = [x for y in (k, v) for x in ref.quantise(y.to(BF))]
    q = q.to(BF)
    o, lse = run(tensors, q, [t, t - 700], n)
    check_verify(tensors, q, [t, t - 700], n, o, lse)
