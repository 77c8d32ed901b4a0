"""Query rows of one KV head whose sizes are octaves apart: each has its own digits."""

import pytest
import torch

from tests import quant_reference as ref
from tests.test_gpu_quant_attn import BF, run_verify
from tests.test_gpu_quant_attn_long import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n", [(4, 2), (4, 6), (4, 21)])
@pytest.mark.parametrize("long", [False, True])
@pytest.mark.parametrize("octaves", [24, 30, 100])
def test_one_head_is_larger(d, G, n, long, octaves):
    t = 500
    g = torch.Generator().manual_seed(octaves + n)
    tensors = [x for _ in range(2) for x in ref.quantise(torch.randn(2, 1, t + n, d, generator=g).to(BF))]
    q = torch.randn(2, G, n, d, generator=g)
    q[:, 1] *= 2.0 ** octaves
    q = q.to(BF)
    o, lse = run(tensors, q, [t, t], n) if long else run_verify(tensors, q, t, n)
    assert torch.isfinite(o.float()).all() and torch.isfinite(lse).all()
    visible = (torch.arange(t + n)[None, :] <= (t + torch.arange(n))[:, None])
    for i in range(2):
        k, v = (ref.values(tensors[2 * x][i, 0], tensors[2 * x + 1][i, 0]) for x in (0, 1))
        for h in range(G):
            wo, wl, spread = ref.attend(q[i, h], k, v, visible)
            if h == 1:
                # one key has it all, as long as its score is clear of the next one's by more than the scores' error
                two = (q[i, h].double() @ k.T * d ** -0.5).masked_fill(~visible, -float("inf")).topk(2, -1).values
                clear = (two[:, 0] - two[:, 1]) > 30 + 2.0 ** -18 * two.abs().max()
                best = (wl[clear], lse[i, h].double().cpu()[clear])
                assert ((best[0] - best[1]).abs() <= 2.0 ** -18 * best[0].abs()).all()
                wo, spread, got = wo[clear], spread[clear], o[i, h].cpu()[clear]
                ref.check(got, best[0], wo, best[0], spread, v.abs().max(), f"seq {i} head {h}")
            else:
                ref.check(o[i, h], lse[i, h], wo, wl, spread, v.abs().max(), f"seq {i} head {h}")


@pytest.mark.parametrize("long", [False, True])
def test_one_query_is_smaller(long):
    """A query row 2^-40 of the others over keys 2^40 as large: its scores are ordinary ones, theirs are not."""
    G, n, d, t = 4, 6, 128, 400
    g = torch.Generator().manual_seed(3)
    k, v = torch.randn(1, 1, t + n, d, generator=g) * 2.0 ** 40, torch.randn(1, 1, t + n, d, generator=g)
    tensors = [x for y in (k, v) for x in ref.quantise(y.to(BF))]
    q = torch.randn(1, G, n, d, generator=g)
    q[:, 2, 3] *= 2.0 ** -40
    q = q.to(BF)
    if long:
        o, lse = run([x.expand(2, -1, -1, -1).contiguous() for x in tensors], q.expand(2, -1, -1, -1).contiguous(), [t, t], n)
    else:
        o, lse = run_verify(tensors, q, t, n)
    k, v = (ref.values(tensors[2 * x][0, 0], tensors[2 * x + 1][0, 0]) for x in (0, 1))
    wo, wl, spread = ref.attend(q[0, 2, 3:4], k, v, torch.arange(t + n)[None, :] <= t + 3)
    ref.check(o[0, 2, 3:4], lse[0, 2, 3:4], wo, wl, spread, v.abs().max())
