"""QuantSpecStep: speculative steps over a 4-bit cache the way a decoding loop makes them (prefill written, window
normalisers, selection, drafter passes, the block's rows, the verify block, acceptance, the cache update), each
call against 64 bits over what the cache holds; and the rows read back for the selection being there in time."""

import pytest
import torch

import paper_2606_00144_gb300 as bd
from tests import quant_reference as ref

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def unit(cache, i, h, rows):
    k = ref.values(cache.k_codes[i, h, rows].cpu(), cache.k_scales[i, h, rows].cpu())
    return k, ref.values(cache.v_codes[i, h, rows].cpu(), cache.v_scales[i, h, rows].cpu())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 4])
def test_a_decoding_loop_over_a_4_bit_cache(d, G):
    b, h_kv, W, gamma, budget, steps = 2, 2, 8, 3, 64, 3
    h_q, t0 = h_kv * G, 300
    cap = t0 + steps * (gamma + 1) + 8
    g = torch.Generator("cuda").manual_seed(d + G)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda").to(BF)

    lens = torch.tensor([t0, t0 - 37], dtype=torch.int32, device="cuda")
    cache = bd.QuantCache.empty(b, h_kv, cap, d)
    k_pre, v_pre = randn(b, h_kv, t0, d), randn(b, h_kv, t0, d)
    bd.bd_quant_write(cache.shape(h_q, 0), k_pre, v_pre, cache)              # the prefill
    st = bd.QuantSpecStep(b, h_q, h_kv, d, t0, cap, budget, 4, 16, window=W, gamma=gamma, seq_lens=lens)
    q_win = randn(b, h_q, W, d)
    lse_win = st.window_lse(cache, q_win)
    for i in range(b):
        t = int(lens[i])
        for h in range(h_kv):
            k, v = unit(cache, i, h, slice(0, t))
            hs = slice(h * G, (h + 1) * G)
            visible = torch.arange(t)[None, :] <= (t - W + torch.arange(W).repeat(G))[:, None]
            _, want, _ = ref.attend(q_win[i, hs].cpu().reshape(-1, d), k.bfloat16().double(), v, visible)
            assert (lse_win[i, hs].reshape(-1).cpu().double() - want).abs().max() < 1e-4
    st.select(cache, q_win, lse_win)
    torch.cuda.synchronize()
    # the same selection from keys that are surely there
    keys = torch.empty(b, h_kv, cap, d, dtype=BF, device="cuda")
    bd.bd_quant_read(st.shape, cache, keys[:, :, :t0], first_row=0)
    torch.cuda.synchronize()
    idx, count = torch.empty_like(st.idx), torch.empty_like(st.count)
    bd.bd_select_budget(st.shape, keys, q_win, lse_win, W, budget, 4, 16, 1, idx, count, st.ws)
    assert torch.equal(idx, st.idx) and torch.equal(count, st.count) and (count == budget).all()

    for step in range(steps):
        # as many positions as the longest sequence has by now
        st.shape = cache.shape(h_q, int(lens.max()), lens)
        now = lens.tolist()
        k_block, v_block = randn(b, gamma + 1, h_kv, d), randn(b, gamma + 1, h_kv, d)   # as a projection leaves them
        st.write(k_block.transpose(1, 2), v_block.transpose(1, 2), cache)
        q_draft, q_verify = randn(gamma, b, h_q, d), randn(b, h_q, gamma + 1, d)
        for j in range(gamma):
            st.draft(j, q_draft[j], cache, view_ready=j > 0)
        st.verify(q_verify, cache)
        assert st.ws.status() == 0
        for i in range(b):
            t = now[i]
            for h in range(h_kv):
                hs = slice(h * G, (h + 1) * G)
                block = slice(t, t + gamma + 1)
                qc, qs = ref.quantise(k_block[i, :, h].cpu())
                assert torch.equal(cache.k_codes[i, h, block].cpu(), qc)
                assert torch.equal(cache.k_scales[i, h, block].cpu(), qs)
                for j in range(gamma):
                    rows = torch.cat([st.idx[i, h, :int(st.count[i, h])].long().cpu(), t + torch.arange(j + 1)])
                    k, v = unit(cache, i, h, rows)
                    o, l, spread = ref.attend(q_draft[j, i, hs].cpu(), k, v, torch.ones(G, len(rows), dtype=torch.bool))
                    ref.check(st.draft_o[j, i, hs], st.draft_lse[j, i, hs], o, l, spread, v.abs().max(), f"step {step} draft {j}")
                n = gamma + 1
                k, v = unit(cache, i, h, slice(0, t + n))
                visible = torch.arange(t + n)[None, :] <= (t + torch.arange(n).repeat(G))[:, None]
                o, l, spread = ref.attend(q_verify[i, hs].cpu().reshape(-1, d), k, v, visible)
                ref.check(st.verify_o[i, hs].reshape(-1, d), st.verify_lse[i, hs].reshape(-1), o, l, spread, v.abs().max(),
                          f"step {step} verify")
        # each sequence accepts its own number of drafts and moves on
        accepted = torch.tensor([step % (gamma + 1), 1], dtype=torch.int32, device="cuda")
        bd.bd_advance(st.shape, W, gamma + 1, accepted, q_verify, st.verify_lse, q_win, lse_win)
        assert lens.tolist() == [now[0] + step % (gamma + 1) + 1, now[1] + 2]


@pytest.mark.parametrize("stream", [False, True])
def test_the_keys_read_back_are_there_when_the_selection_streams_them(stream):
    """The selection and the window pass stream context rows before their dependency wait: the read just before them
    must have landed.  Caches in turn, so that a stale row is another cache's."""
    b, h_q, h_kv, d, t, W, budget = 4, 16, 4, 128, 8192, 32, 512
    caches = []
    for i in range(3):
        k = torch.randn(b, h_kv, t, d, device="cuda", generator=torch.Generator("cuda").manual_seed(i)).to(BF)
        cache = bd.QuantCache.empty(b, h_kv, t + 6, d)
        bd.bd_quant_write(cache.shape(h_q, 0), k, k, cache)
        caches.append(cache)
    q_win = torch.randn(b, h_q, W, d, device="cuda").to(BF)
    st = bd.QuantSpecStep(b, h_q, h_kv, d, t, t + 6, budget, 4, 128, window=W)
    want = []
    for cache in caches:
        keys = torch.zeros(b, h_kv, t + 6, d, dtype=BF, device="cuda")
        bd.bd_quant_read(st.shape, cache, keys[:, :, :t], first_row=0)
        torch.cuda.synchronize()
        plain = bd.SpecStep(b, h_q, h_kv, d, t, t + 6, budget, 4, 128, window=W)
        lse = plain.window_lse(keys, q_win)
        plain.select(keys, q_win, lse)
        torch.cuda.synchronize()
        want.append((lse.clone(), plain.idx.clone()))
    s = torch.cuda.Stream() if stream else None
    torch.cuda.synchronize()
    for turn in range(20):
        cache, (lse, idx) = caches[turn % 3], want[turn % 3]
        got = st.window_lse(cache, q_win, stream=s)
        st.select(cache, q_win, lse, stream=s)
        torch.cuda.synchronize()
        assert torch.equal(got, lse), turn
        assert torch.equal(st.idx, idx), turn


def test_a_step_replays_from_a_graph():
    b, h_q, h_kv, d, t, gamma, budget = 2, 8, 2, 128, 2000, 4, 256
    cache = bd.QuantCache.empty(b, h_kv, t + gamma + 1, d)
    rows = [torch.randn(b, h_kv, t, d, device="cuda").to(BF) for _ in range(2)]
    bd.bd_quant_write(cache.shape(h_q, 0), *rows, cache)
    st = bd.QuantSpecStep(b, h_q, h_kv, d, t, t + gamma + 1, budget, 4, 64, window=16, gamma=gamma)
    q_win, q_draft = torch.randn(b, h_q, 16, d, device="cuda").to(BF), torch.randn(gamma, b, h_q, d, device="cuda").to(BF)
    q_verify, block = torch.randn(b, h_q, gamma + 1, d, device="cuda").to(BF), torch.randn(2, b, h_kv, gamma + 1, d, device="cuda").to(BF)

    def step():
        st.write(block[0], block[1], cache)
        st.run(cache, q_win, q_draft, q_verify)

    step()
    torch.cuda.synchronize()
    want = [x.clone() for x in (st.idx, st.draft_o, st.verify_o, st.verify_lse)]
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=s):
        step()
    for x in (st.idx, st.draft_o, st.verify_o, st.verify_lse):
        x.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for x, y in zip((st.idx, st.draft_o, st.verify_o, st.verify_lse), want):
        assert torch.equal(x, y)


def test_a_step_that_cannot_be_planned_is_refused():
    with pytest.raises(bd.BudgetDraftError):
        bd.QuantSpecStep(1, 34, 2, 128, 100, 110, 32, 4, 8)       # a group of 17: no drafter pass
