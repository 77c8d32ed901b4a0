"""One workspace for a context that grows: its size at any length serves every length that the cache can hold."""

import ctypes

import pytest

import paper_2606_00144_gb300 as bd
from paper_2606_00144_gb300 import binding
from tests.test_quant_abi import lib, shape  # noqa: F401  (lib: a fixture)

LENGTHS = [0, 1, 100, 700, 900, 1100, 3000, 6000, 6200, 7040, 7168, 9000, 16384, 30000, 65536, 99000]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("batch,h_q,h_kv", [(1, 8, 2), (8, 32, 8), (1, 4, 4), (2, 32, 4), (40, 32, 8)])
@pytest.mark.parametrize("lens", [None, 4096])
@pytest.mark.parametrize("n", [1, 6, 21])
def test_a_size_serves_every_length(lib, d, batch, h_q, h_kv, lens, n):  # noqa: F811
    def size(t, n):
        s = shape(batch=batch, h_q=h_q, h_kv=h_kv, head_dim=d, t_ctx=t, t_cap=100_000)
        s.seq_lens = lens
        return lib.bd_workspace_size(ctypes.byref(s), binding.BD_OP_QUANT_VERIFY, 0, n)

    sizes = {t: size(t, n) for t in LENGTHS}
    assert min(sizes.values()) > 0
    # what a call at a length needs is no more than what any other length was told
    assert len(set(sizes.values())) == 1, sizes
    assert all(size(t, m) <= sizes[0] for t in LENGTHS for m in range(1, n))


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 6])
@pytest.mark.parametrize("lens", [False, True])
def test_a_loop_over_growing_and_shrinking_contexts(d, n, lens):
    import torch

    b, h_kv, G, cap = 8, 8, 4, 20_000
    cache = bd.QuantCache.empty(b, h_kv, cap, d)
    for x in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales):
        x.zero_()
    q = torch.zeros(b, h_kv * G, n, d, dtype=torch.bfloat16, device="cuda")
    o, lse = torch.empty_like(q), torch.empty(q.shape[:3], device="cuda")
    seq = torch.zeros(b, dtype=torch.int32, device="cuda") if lens else None
    ws = bd.Workspace(bd.bd_workspace_size(cache.shape(h_kv * G, 700, seq), bd.BD_OP_QUANT_VERIFY, 0, n))
    for t in [0, 700, 900, 5000, 6200, 7040, 7168, 12000, cap - n, 300]:
        if lens:
            seq.fill_(t)
        bd.bd_quant_verify_attn(cache.shape(h_kv * G, t, seq), q, n, cache, o, lse, ws)
        want = torch.log(t + 1 + torch.arange(n, dtype=torch.float64))
        assert (lse.double().cpu() - want).abs().max() < 1e-4
    assert ws.status() == 0


@pytest.mark.gpu
def test_a_step_is_made_for_the_whole_cache():
    import torch

    b, h_kv, G, d, gamma, W, budget, cap = 2, 2, 4, 128, 5, 16, 64, 12_000
    cache = bd.QuantCache.empty(b, h_kv, cap, d)
    g = torch.Generator("cuda").manual_seed(1)
    rows = torch.randn(b, h_kv, cap, d, generator=g, device="cuda").to(torch.bfloat16)
    bd.bd_quant_write(cache.shape(h_kv * G, 0), rows, rows, cache)
    q = torch.randn(b, h_kv * G, W, d, generator=g, device="cuda").to(torch.bfloat16)
    st = bd.QuantSpecStep(b, h_kv * G, h_kv, d, 100, cap, budget, 4, 16, window=W, gamma=gamma)
    for t in [100, 700, 3000, 6200, 7100, cap - gamma - 1]:
        st.shape = cache.shape(h_kv * G, t)
        st.run(cache, q, q[:, :, :gamma].permute(2, 0, 1, 3).contiguous(), q[:, :, :gamma + 1].contiguous())
        assert (st.count == budget).all() and st.ws.status() == 0
