"""Scores that are what is left of a cancellation: the products of a query and a key are summed in 32 bits, so a score is
off by a few 2^-22 of sum |q k| / sqrt(d), in every kernel that reads the 4-bit cache."""

import math

import pytest
import torch

import paper_2606_00144_gb300 as bd
from tests import quant_reference as ref
from tests.test_gpu_quant_attn import BF, run_draft, run_verify
from tests.test_gpu_quant_attn_long import run

pytestmark = pytest.mark.gpu


def make(b, rows, d, g):
    """Keys whose neighbouring elements are equal, so that queries of opposite neighbours cancel."""
    c = torch.randint(1, 16, (b, 1, rows, d // 2), generator=g, dtype=torch.uint8)
    scales = torch.full((b, 1, rows, d // 32), 0.25).to(BF)
    _, _, vc, vs = (x for y in (torch.zeros(b, 1, rows, d), torch.randn(b, 1, rows, d, generator=g))
                    for x in ref.quantise(y.to(BF)))
    return [c | c << 4, scales, vc, vs]


def queries(shape, g):
    """Elements of some 512, the second of a pair the first's opposite but for a unit in the last place."""
    x = (512 * (1 + torch.rand(*shape[:-1], shape[-1] // 2, generator=g))).to(BF)
    x *= torch.randint(0, 2, x.shape, generator=g) * 2 - 1
    y = (x.view(torch.int16) ^ 1).view(BF)
    return torch.stack([x, -y], -1).flatten(-2).contiguous()


def check(q, k, v, visible, o, lse):
    d = q.shape[-1]
    wo, wl, spread = ref.attend(q, k, v, visible)
    size = (q.double().abs() @ k.abs().T / math.sqrt(d)).max().item()
    # a score's error e moves a weight by e of it, and the normaliser too: 2 e; an output's rounding and the weights' 11 bits
    # as everywhere.  A sum of 128 exact products in 32 bits, four to eight at a time: some 2^-22 of the sum of their sizes
    err = size * 2.0 ** -22
    tol = 2.0 ** -8 * wo.abs() + (2.0 ** -10 + 2 * err) * spread + 2.0 ** -31 * v.abs().max()
    worst = ((o.double().cpu() - wo).abs() / tol).max().item()
    assert worst <= 1, f"{worst:.2f} times the tolerance"
    worst = ((lse.double().cpu() - wl).abs() / (5e-5 + 1e-5 * wl.abs() + err)).max().item()
    assert worst <= 1, f"lse {worst:.2f} times the tolerance"


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n", [(1, 1), (4, 6), (8, 8), (4, 21)])
@pytest.mark.parametrize("long", [False, True])
def test_verify(d, G, n, long):
    t = 600
    g = torch.Generator().manual_seed(d + n)
    tensors, q = make(2, t + n, d, g), queries((2, G, n, d), g)
    o, lse = run(tensors, q, [t, t], n) if long else run_verify(tensors, q, t, n)
    visible = torch.arange(t + n)[None, :] <= (t + torch.arange(n).repeat(G))[:, None]
    for i in range(2):
        k, v = (ref.values(tensors[2 * x][i, 0], tensors[2 * x + 1][i, 0]) for x in (0, 1))
        check(q[i].reshape(-1, d), k, v, visible, o[i].reshape(-1, d), lse[i].reshape(-1))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 8, 16])
def test_draft(d, G):
    t, j, budget = 700, 3, 400
    g = torch.Generator().manual_seed(d + G)
    tensors, q = make(1, t + j + 1, d, g), queries((1, G, d), g)
    idx = torch.randperm(t, generator=g)[:budget].sort().values.int().view(1, 1, budget)
    o, lse, status = run_draft(tensors, q, t, idx, torch.full((1, 1), budget, dtype=torch.int32), j)
    assert status == 0
    rows = torch.cat([idx[0, 0].long(), t + torch.arange(j + 1)])
    k, v = (ref.values(tensors[2 * x][0, 0, rows], tensors[2 * x + 1][0, 0, rows]) for x in (0, 1))
    check(q[0], k, v, torch.ones(G, len(rows), dtype=torch.bool), o[0], lse[0])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 4, 8, 16])
@pytest.mark.parametrize("n_seq", [200])
@pytest.mark.parametrize("long", [False, True])
def test_one_key(d, G, n_seq, long):
    """The log-sum-exp of one key is its score, to a few units of 32 bits of sum |q k| / sqrt(d)."""
    g = torch.Generator().manual_seed(d + G)
    cap = 12_000 if long else 4                              # (the kernel of long contexts, of short ones)
    codes = torch.randint(0, 256, (n_seq, 1, 1, d // 2), generator=g, dtype=torch.uint8)
    scale = torch.full((n_seq, 1, 1, d // 32), 0.25).to(BF)
    q = (torch.randn(n_seq, G, 1, d, generator=g) * 512).to(BF)
    cache = bd.QuantCache.empty(n_seq, 1, cap, d)
    for x in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales):
        x.zero_()
    cache.k_codes[:, :, :1], cache.k_scales[:, :, :1] = codes.cuda(), scale.cuda()
    seq = torch.zeros(n_seq, dtype=torch.int32, device="cuda")
    shape = cache.shape(G, cap - 1, seq)
    ws = bd.Workspace(bd.bd_workspace_size(shape, bd.BD_OP_QUANT_VERIFY, 0, 1))
    o, lse = torch.empty_like(q, device="cuda"), torch.empty(n_seq, G, 1, device="cuda")
    bd.bd_quant_verify_attn(shape, q.cuda(), 1, cache, o, lse, ws)
    assert ws.status() == 0
    k = ref.values(codes, scale)
    want = (q.double() * k).sum(-1) / math.sqrt(d)
    size = (q.double() * k).abs().sum(-1) / math.sqrt(d)
    worst = ((lse.double().cpu() - want).abs() / (2.0 ** -22 * size + 2.0 ** -22 * want.abs())).max().item()
    assert worst <= 1, f"{worst:.2f} times the tolerance"
