"""Rows whose groups differ in size by up to sixteen octaves.  The attentions take a group's values to within 2^-19 of the
largest scale in its row (exactly where its own is at least 2^-8 of that): the tolerances below are this, on top of what
every call's are."""

import math

import pytest
import torch

from tests import quant_reference as ref
from tests.test_gpu_quant_attn import BF, run_draft, run_verify
from tests.test_gpu_quant_attn_long import run

pytestmark = pytest.mark.gpu


def make(b, rows, d, side, octaves, g, same):
    """K and V with group 1 of every row (same) or of every second one 2^-octaves of the others."""
    k, v = (torch.randn(b, 1, rows, d, generator=g) for _ in range(2))
    x = k if side == "k" else v
    x[:, :, :: 1 if same else 2, 32:64] *= 2.0 ** -octaves
    return [x for y in (k, v) for x in ref.quantise(y.to(BF))]


def check(tensors, q, visible, o, lse, what=""):
    """tensors: one unit's rows; q [r, d]."""
    d = q.shape[-1]
    k, v = (ref.values(tensors[2 * i], tensors[2 * i + 1]) for i in (0, 1))
    ks, vs = (tensors[2 * i + 1].double() for i in (0, 1))
    wo, wl, spread = ref.attend(q, k, v, visible)
    uneven = ks < 2.0 ** -8 * ks.amax(1, keepdim=True)       # [rows, groups]
    size = (q.double().abs() @ k.abs().T).max(1).values
    rounded = q.double().abs().unflatten(1, (-1, 32)).sum(-1) @ (uneven * ks.amax(1, keepdim=True)).T * 2.0 ** -19
    err = (2.0 ** -22 * size + rounded.max(1).values) / math.sqrt(d)      # of a score, by query
    x = (q.double() @ k.T / math.sqrt(d)).masked_fill(~visible, -math.inf)
    p = torch.softmax(x, 1)
    v_err = ((vs < 2.0 ** -8 * vs.amax(1, keepdim=True)) * vs.amax(1, keepdim=True)).repeat_interleave(32, 1) * 2.0 ** -19
    tol = 2.0 ** -8 * wo.abs() + (2.0 ** -10 + 2 * err[:, None]) * spread + p @ v_err + 2.0 ** -31 * v.abs().max()
    worst = ((o.double().cpu() - wo).abs() / tol).max().item()
    assert worst <= 1, f"{what}: {worst:.2f} times the tolerance"
    worst = ((lse.double().cpu() - wl).abs() / (5e-5 + 1e-5 * wl.abs() + err)).max().item()
    assert worst <= 1, f"{what}: lse {worst:.2f} times the tolerance"


def block(t, G, n):
    return torch.arange(t + n)[None, :] <= (t + torch.arange(n).repeat(G))[:, None]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n", [(1, 1), (4, 6), (4, 21)])
@pytest.mark.parametrize("long", [False, True])
@pytest.mark.parametrize("side", ["k", "v"])
@pytest.mark.parametrize("octaves", [8, 12, 16])
@pytest.mark.parametrize("same", [True, False])
def test_verify(d, G, n, long, side, octaves, same):
    t = 500
    g = torch.Generator().manual_seed(octaves + n)
    tensors = make(2, t + n, d, side, octaves, g, same)
    q = torch.randn(2, G, n, d, generator=g)
    if side == "k" and same:
        q[..., 32:64] *= 2.0 ** (octaves // 2)               # queries that look at the small group
    q = q.to(BF)
    o, lse = run(tensors, q, [t, t], n) if long else run_verify(tensors, q, t, n)
    for i in range(2):
        check([x[i, 0] for x in tensors], q[i].reshape(-1, d), block(t, G, n), o[i].reshape(-1, d), lse[i].reshape(-1), f"seq {i}")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [4, 16])
@pytest.mark.parametrize("side", ["k", "v"])
@pytest.mark.parametrize("octaves", [8, 16])
def test_draft(d, G, side, octaves):
    t, j, budget = 400, 2, 200
    g = torch.Generator().manual_seed(octaves + G)
    tensors = make(1, t + j + 1, d, side, octaves, g, True)
    q = torch.randn(1, G, d, generator=g).to(BF)
    idx = torch.randperm(t, generator=g)[:budget].sort().values.int().view(1, 1, budget)
    o, lse, status = run_draft(tensors, q, t, idx, torch.full((1, 1), budget, dtype=torch.int32), j)
    assert status == 0
    rows = torch.cat([idx[0, 0].long(), t + torch.arange(j + 1)])
    check([x[0, 0, rows] for x in tensors], q[0], torch.ones(G, len(rows), dtype=torch.bool), o[0], lse[0])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n", [(1, 1), (4, 6), (8, 4), (8, 8), (4, 21)])
@pytest.mark.parametrize("long", [False, True])
@pytest.mark.parametrize("octaves", [12, 14])
def test_scores_of_a_small_group_alone(d, G, n, long, octaves):
    """The queries see nothing but the small group, whose values are plus or minus one code: rounded away, every key
    would weigh the same."""
    t = 300
    codes = torch.full((2, 1, t + n, d // 2), 0x88, dtype=torch.uint8)
    codes[:, :, ::2, 16:32] = 0x99
    codes[:, :, 1::2, 16:32] = 0x77
    scales = torch.ones(2, 1, t + n, d // 32).to(BF)
    codes[..., 0] = 0x8f                                     # (the largest scale has a value to it)
    scales[..., 1] = 1.375 * 2.0 ** -octaves
    g = torch.Generator().manual_seed(n)
    tensors = [codes, scales, *ref.quantise(torch.randn(2, 1, t + n, d, generator=g).to(BF))]
    q = torch.zeros(2, G, n, d)
    q[..., 32:64] = 2.0 ** octaves / 8
    q = q.to(BF)
    o, lse = run(tensors, q, [t, t], n) if long else run_verify(tensors, q, t, n)
    for i in range(2):
        check([x[i, 0] for x in tensors], q[i].reshape(-1, d), block(t, G, n), o[i].reshape(-1, d), lse[i].reshape(-1), f"seq {i}")
