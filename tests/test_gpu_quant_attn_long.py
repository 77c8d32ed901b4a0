"""Verify blocks of short sequences in a cache with room for long ones: the launch is planned for the room
(the tensor-memory kernel, a unit's tiles over many CTAs), the lengths are the sequences' own."""

import math

import pytest
import torch

import paper_2606_00144_gb300 as bd
from tests import quant_reference as ref
from tests.test_gpu_quant_attn import BF, check_verify, make_cache, run_verify, run_verify_nan

pytestmark = pytest.mark.gpu


def room(rows, d):
    """Rows a sequence may have, so many that two KV heads' blocks are the tensor-memory kernel's."""
    if d == 64:
        return 400_000 if rows <= 8 else 120_000
    return 60_000


def widened(tensors, cap):
    """The same rows in a cache of cap rows, what is past them codes and NaN scales that no query may see."""
    out = []
    for x in tensors:
        y = torch.full((*x.shape[:2], cap, x.shape[3]), 0x0f if x.dtype == torch.uint8 else math.nan, dtype=x.dtype)
        y[:, :, :x.shape[2]] = x
        out.append(y)
    return out


def run(tensors, q, lens, n):
    t = room(q.shape[1] // tensors[0].shape[1] * n, q.shape[3])
    wide = widened(tensors, t + n)
    for i, m in enumerate(lens):
        for x in wide:
            x[i, :, m + n:] = 0x0f if x.dtype == torch.uint8 else math.nan
    return run_verify(wide, q, t, n, torch.tensor(lens, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n", [(1, 1), (4, 1), (8, 1), (3, 3), (4, 6), (8, 4), (1, 33), (8, 8), (4, 21), (8, 13), (8, 25)])
@pytest.mark.parametrize("lens", [[0, 1], [15, 127], [128, 129], [260, 1000], [5, 3000]])
def test_short_sequences(d, G, n, lens):
    tensors = make_cache(2, 1, max(lens) + n, d, seed=sum(lens) + n)
    q = torch.randn(2, G, n, d, generator=torch.Generator().manual_seed(n)).to(BF)
    o, lse = run(tensors, q, lens, n)
    check_verify(tensors, q, lens, n, o, lse)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n", [(4, 1), (4, 6), (4, 12)])
@pytest.mark.parametrize("case", ["tiny v", "large v", "mixed v", "sharp", "zero rows", "mixed k", "offset v", "late peak", "tiny q"])
def test_sizes_of_values(d, G, n, case):
    t = 777
    g = torch.Generator().manual_seed(13)
    k, v = (torch.randn(2, 1, t + n, d, generator=g) for _ in range(2))
    q = torch.randn(2, G, n, d, generator=g)
    if case == "tiny v":
        v *= 2.0 ** -60
    elif case == "large v":
        v *= 2.0 ** 60
    elif case == "mixed v":
        v *= torch.exp2(torch.randint(-12, 13, (2, 1, t + n, 1), generator=g).float())
    elif case == "sharp":
        q *= 8
    elif case == "zero rows":
        k[:, :, ::3] = 0
        v[:, :, ::2] = 0
        v[:, :, :40] = 0
        q[:, 0] = 0
    elif case == "mixed k":
        k *= torch.exp2(torch.randint(-12, 2, (2, 1, t + n, 1), generator=g).float())
    elif case == "offset v":
        v = v * 0.05 + 3
    elif case == "late peak":
        k[:, :, -n - 5] = 3 * q[:, ::G, 0]
    elif case == "tiny q":
        q *= 2.0 ** -20
        k *= 2.0 ** 20
    tensors = [x for y in (k, v) for x in ref.quantise(y.to(BF))]
    q = q.to(BF)
    o, lse = run(tensors, q, [t, t], n)
    check_verify(tensors, q, [t, t], n, o, lse, case)


@pytest.mark.parametrize("n", [6, 12])
def test_a_nan_stays_where_it_belongs(n):
    G, t, d = 4, 20_000, 128
    tensors = make_cache(2, 2, t + n, d)
    q = torch.randn(2, 2 * G, n, d, generator=torch.Generator().manual_seed(1)).to(BF)
    tensors[1][0, 1, 17, 2] = math.nan                       # a K group: every query of that head sees it
    tensors[3][1, 0, t + 3, 1] = math.nan                    # a V group of the block's fourth row
    q[1, 6, 2, 5] = math.nan
    o, lse = (x.cpu() for x in run_verify_nan(tensors, q, t, n))
    assert o[0, G:].isnan().all() and lse[0, G:].isnan().all() and torch.isfinite(o[0, :G]).all()
    assert o[1, :G, 3:, 32:64].isnan().all() and torch.isfinite(o[1, :G, 3:, :32]).all()
    assert torch.isfinite(lse[1, :G]).all()
    assert o[1, 6, 2].isnan().all() and torch.isfinite(o[1, 6, 1]).all() and torch.isfinite(o[1, 7]).all()


def test_a_length_outside_the_shape_is_recorded():
    G, n, t, d = 4, 6, 60_000, 64
    tensors = make_cache(3, 1, t + n, d)
    q = torch.randn(3, G, n, d, generator=torch.Generator().manual_seed(2)).to(BF)
    cache = bd.QuantCache(*(x.cuda() for x in tensors))
    seq = torch.tensor([2000, t + 1, -1], dtype=torch.int32, device="cuda")    # (the shape holds its address only)
    shape = cache.shape(G, t, seq)
    ws = bd.Workspace(bd.bd_workspace_size(shape, bd.BD_OP_QUANT_VERIFY, 0, n))
    o, lse = torch.empty_like(q, device="cuda"), torch.empty(q.shape[:3], device="cuda")
    bd.bd_quant_verify_attn(shape, q.cuda(), n, cache, o, lse, ws)
    assert ws.status() == -1 and ws.status() == 0
    check_verify(tensors, q, [2000, t, 0], n, o, lse)
