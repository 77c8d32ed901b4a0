"""PagedSpecStep: speculative steps over a paged cache the way a decoding loop makes them (prompts appended with their rotation,
window normalisers, selection, drafter passes, the block's tokens appended, the verify block, acceptance, the cache update, pages
taken as the sequences grow), each call against 64 bits over what the pool holds; graphs and streams."""

import pytest
import torch

import paper_2606_00144_gb300 as bd
from tests import paged_reference as ref

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def unit(cache, table, i, h, rows):
    e = table[i][rows // cache.page_size].long()
    return cache.k.cpu()[e, h, rows % cache.page_size].double(), cache.v.cpu()[e, h, rows % cache.page_size].double()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 4])
@pytest.mark.parametrize("page", [16, 32])
def test_a_decoding_loop_over_a_paged_cache(d, G, page):
    b, h_kv, W, gamma, budget, steps = 2, 2, 8, 3, 64, 3
    h_q, prompts = h_kv * G, [300, 263]
    cap = 300 + steps * (gamma + 1) + 8
    g = torch.Generator("cuda").manual_seed(d + G)

    def randn(*shape, dtype=BF):
        return torch.randn(*shape, generator=g, device="cuda").to(dtype)

    per = -(-cap // page)
    cache = bd.PagedCache.empty(2 * per + 3, h_kv, page, d)
    cache.k.fill_(float("nan"))
    cache.v.fill_(float("nan"))
    free = torch.randperm(2 * per + 3, generator=torch.Generator().manual_seed(1)).tolist()
    table = torch.full((b, per), -1, dtype=torch.int32)

    def take(lens):                       # pages for the first lens[i] positions
        for i, n in enumerate(lens):
            for j in range(-(-n // page)):
                if table[i, j] < 0:
                    table[i, j] = free.pop()
        return table.cuda()

    freq = 10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)
    rope = bd.Rope(freq)
    dev = take(prompts)
    # the prompts, packed: fp32 projections [token, heads, d]
    total = sum(prompts)
    qkv = randn(total, h_q + 2 * h_kv, d, dtype=torch.float32).transpose(0, 1)
    q, k, v = qkv.split([h_q, h_kv, h_kv])
    q_rot = torch.empty(h_q, total, d, dtype=BF, device="cuda")
    starts = torch.tensor([0, prompts[0], total], dtype=torch.int32, device="cuda")
    bd.bd_paged_append(cache.shape(b, h_q, 0, cap), q, k, v, rope, cache, dev, q_rot, row_starts=starts)
    for i, t in enumerate(prompts):
        rows = k[:, starts[i]:starts[i + 1]].cpu()
        want = ref.rotate(rows, torch.arange(t), freq, False)
        tol = ref.rotate_tolerance(rows, want, freq, False)
        for h in range(h_kv):
            assert ((unit(cache, table, i, h, torch.arange(t))[0] - want[h]).abs() <= tol[h]).all()

    lens = torch.tensor(prompts, dtype=torch.int32, device="cuda")
    st = bd.PagedSpecStep(b, h_q, h_kv, d, max(prompts), cap, budget, 4, 16, window=W, gamma=gamma, seq_lens=lens)
    # the last W queries of each prompt, as the append left them
    q_win = torch.stack([q_rot[:, int(starts[i + 1]) - W:int(starts[i + 1])] for i in range(b)]).contiguous()
    lse_win = st.window_lse(cache, dev, q_win)
    for i, t in enumerate(prompts):
        for h in range(h_kv):
            kk, vv = unit(cache, table, i, h, torch.arange(t))
            hs = slice(h * G, (h + 1) * G)
            visible = torch.arange(t)[None, :] <= (t - W + torch.arange(W).repeat(G))[:, None]
            _, want, _ = ref.attend(q_win[i, hs].cpu().reshape(-1, d), kk, vv, visible)
            assert (lse_win[i, hs].reshape(-1).cpu().double() - want).abs().max() < 1e-4
    st.select(cache, dev, q_win, lse_win)
    # the same selection over a contiguous cache
    keys = torch.zeros(b, h_kv, cap, d, dtype=BF, device="cuda")
    bd.bd_paged_read(st.shape, cache, dev, keys[:, :, :max(prompts)], first_row=0)
    torch.cuda.synchronize()
    idx, count = torch.empty_like(st.idx), torch.empty_like(st.count)
    bd.bd_select_budget(st.shape, keys, q_win, lse_win, W, budget, 4, 16, 1, idx, count, st.ws)
    assert torch.equal(idx, st.idx) and torch.equal(count, st.count) and (count == budget).all()

    n = gamma + 1
    for step in range(steps):
        now = lens.tolist()
        st.shape = cache.shape(b, h_q, max(now), cap, lens)
        dev = take([t + n for t in now])
        qkv = randn(b, n, h_q + 2 * h_kv, d).transpose(1, 2)           # the block's projections
        q, k, v = qkv.split([h_q, h_kv, h_kv], dim=1)
        q_verify = torch.empty(b, h_q, n, d, dtype=BF, device="cuda")
        st.append(q, k, v, rope, cache, dev, q_verify)
        q_draft = randn(gamma, b, h_q, d)
        for j in range(gamma):
            st.draft(j, q_draft[j], cache, dev, view_ready=j > 0)
        st.verify(q_verify, cache, dev)
        assert st.ws.status() == 0
        for i in range(b):
            t = now[i]
            want = ref.rotate(q[i].cpu(), t + torch.arange(n), freq, False)
            assert ((q_verify[i].cpu().double() - want).abs() <= ref.rotate_tolerance(q[i].cpu(), want, freq, False)).all()
            for h in range(h_kv):
                hs = slice(h * G, (h + 1) * G)
                for j in range(gamma):
                    rows = torch.cat([st.idx[i, h, :int(st.count[i, h])].long().cpu(), t + torch.arange(j + 1)])
                    kk, vv = unit(cache, table, i, h, rows)
                    want = ref.attend(q_draft[j, i, hs].cpu(), kk, vv, torch.ones(G, len(rows), dtype=torch.bool))
                    ref.check(st.draft_o[j, i, hs], st.draft_lse[j, i, hs], *want, f"step {step} draft {j}")
                kk, vv = unit(cache, table, i, h, torch.arange(t + n))
                visible = torch.arange(t + n)[None, :] <= (t + torch.arange(n).repeat(G))[:, None]
                want = ref.attend(q_verify[i, hs].cpu().reshape(-1, d), kk, vv, visible)
                ref.check(st.verify_o[i, hs].reshape(-1, d), st.verify_lse[i, hs].reshape(-1), *want, f"step {step} verify")
        # acceptance of 0 .. gamma drafts, lengths and window moved on the device, positions joined to the view
        accept = torch.tensor([step % n, (step + 2) % n], dtype=torch.int32, device="cuda")
        idx = torch.full((b, h_kv, budget + 16), -1, dtype=torch.int32, device="cuda")
        idx[:, :, :st.idx.shape[2]] = st.idx
        bd.bd_advance(st.shape, W, n, accept, q_verify, st.verify_lse, q_win, lse_win, idx, st.count)
        st.idx = idx[:, :, :st.idx.shape[2] + 0].contiguous()
        st.count.clamp_(max=budget)
        assert lens.tolist() == [t + int(a) + 1 for t, a in zip(now, accept.tolist())]


def test_a_captured_pass_follows_the_table_and_the_lengths():
    """A decoding pass (append, attention) in a graph: replays read what the tables, lengths and rows hold then."""
    b, h_kv, G, d, page, cap = 3, 2, 4, 128, 16, 400
    pool = ref.Pool([cap] * b, h_kv, page, d, seed=4, cap=cap)
    K, V, table = pool.cuda()
    cache = bd.PagedCache(K, V)
    lens = torch.zeros(b, dtype=torch.int32, device="cuda")
    shape = cache.shape(b, h_kv * G, cap - 1, cap, lens)
    ws = bd.Workspace(bd.bd_workspace_size(shape, bd.BD_OP_PAGED_VERIFY, 0, 1))
    rope = bd.Rope.of_base(d)
    qkv = torch.zeros(b, 1, h_kv * (G + 2), d, dtype=BF, device="cuda").transpose(1, 2)
    q, k, v = qkv.split([h_kv * G, h_kv, h_kv], dim=1)
    q_out = torch.empty(b, h_kv * G, 1, d, dtype=BF, device="cuda")
    o, lse = torch.empty_like(q_out), torch.empty(b, h_kv * G, 1, device="cuda")

    def step():
        bd.bd_paged_append(shape, q, k, v, rope, cache, table, q_out)
        bd.bd_paged_verify_attn(shape, q_out, 1, cache, table, o, lse, ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    g = torch.Generator().manual_seed(9)
    for t in ([0, 17, 399], [100, 15, 16], [255, 256, 1]):
        lens.copy_(torch.tensor(t, dtype=torch.int32))
        perm = torch.randperm(b, generator=g)
        table.copy_(pool.table[perm])
        qkv.copy_(torch.randn(qkv.shape, generator=g).to(BF))
        graph.replay()
        torch.cuda.synchronize()
        assert ws.status() == 0
        got = ref.Pool([cap] * b, h_kv, page, d, seed=4, cap=cap)
        got.k, got.v, got.table = K.cpu(), V.cpu(), table.cpu()
        for i in range(b):
            want = ref.rotate(q[i].cpu(), torch.tensor([t[i]]), 10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d), False)
            assert (q_out[i].cpu().double() - want).abs().max() < 0.02
            for h in range(h_kv):
                kk, vv, _ = got.unit(i, h, torch.arange(t[i] + 1))
                hs = slice(h * G, (h + 1) * G)
                want = ref.attend(q_out[i, hs, 0].cpu(), kk, vv, torch.ones(G, t[i] + 1, dtype=torch.bool))
                ref.check(o[i, hs, 0], lse[i, hs, 0], *want)


def test_a_chain_of_calls_on_another_stream():
    """Each call reads what the one before wrote, with nothing in between: tables and lengths from kernels just before."""
    b, h_kv, G, d, page, t = 8, 8, 4, 128, 16, 2000
    pool = ref.Pool([t + 4] * b, h_kv, page, d, seed=4)
    K, V, table = pool.cuda()
    cache = bd.PagedCache(K, V)
    lens = torch.full((b,), t, dtype=torch.int32, device="cuda")
    shape = cache.shape(b, h_kv * G, t, t + 4, lens)
    ws = bd.Workspace(bd.bd_workspace_size(shape, bd.BD_OP_PAGED_VERIFY, 0, 4))
    q = torch.randn(b, h_kv * G, 4, d, device="cuda").to(BF)
    kv = torch.randn(b, h_kv, 4, d, device="cuda").to(BF)
    rope = bd.Rope.of_base(d)
    runs = []
    torch.cuda.synchronize()
    for stream in (torch.cuda.Stream(), torch.cuda.current_stream()):
        out = []
        with torch.cuda.stream(stream):
            for i in range(20):
                where = torch.where(torch.arange(table.shape[1], device="cuda") >= i, table, -1).int().contiguous()
                lens.copy_(lens - 1).add_(1)
                q_out, o, lse = torch.empty_like(q), torch.empty_like(q), torch.empty(q.shape[:3], device="cuda")
                bd.bd_paged_append(shape, q, kv, kv, rope, cache, where, q_out)
                bd.bd_paged_verify_attn(shape, q_out, 4, cache, where, o, lse, ws)
                rows = torch.zeros(b, h_kv, 4, d, dtype=BF, device="cuda")
                bd.bd_paged_read(shape, cache, where, rows)
                out += [q_out, o, lse, rows]
        stream.synchronize()
        runs.append(out)
    for x, y in zip(*runs):
        assert torch.equal(x, y) and torch.isfinite(x).all()
    assert ws.status() == 0
    # the last table hid the first 19 pages
    last = ref.Pool([t + 4] * b, h_kv, page, d, seed=4)
    last.k, last.v = K.cpu(), V.cpu()
    last.table[:, :19] = -1
    for i in (0, b - 1):
        kk, vv, there = last.unit(i, 3, torch.arange(t + 4))
        visible = (torch.arange(t + 4)[None, :] <= (t + torch.arange(4).repeat(G))[:, None]) & there
        want = ref.attend(out[-4][i, 12:16].cpu().reshape(-1, d), kk, vv, visible)
        ref.check(out[-3][i, 12:16].reshape(-1, d), out[-2][i, 12:16].reshape(-1), *want)


def test_two_graphs_that_share_a_workspace():
    """Graphs of blocks that take different routes (partials of different sizes), one workspace, replayed in turn; and both at
    once with workspaces of their own."""
    d, page = 128, 16
    g = torch.Generator("cuda").manual_seed(2)

    def make(b, h_kv, G, t, n):
        per = -(-(t + n) // page)
        k, v = (torch.randn(b * per, h_kv, page, d, generator=g, device="cuda").to(BF) for _ in "kv")
        table = torch.randperm(b * per, generator=g, device="cuda").view(b, per).int()
        q = torch.randn(b, h_kv * G, n, d, generator=g, device="cuda").to(BF)
        cache = bd.PagedCache(k, v)
        shape = cache.shape(b, h_kv * G, t, t + n)
        return shape, q, n, cache, table

    calls = [make(1, 2, 4, 30000, 1), make(4, 8, 8, 1500, 21), make(2, 8, 4, 500, 1)]
    sizes = [bd.bd_workspace_size(c[0], bd.BD_OP_PAGED_VERIFY, 0, c[2]) for c in calls]
    shared = bd.Workspace(max(sizes))
    want = []
    for c, size in zip(calls, sizes):
        o, lse = torch.empty_like(c[1]), torch.empty(c[1].shape[:3], device="cuda")
        bd.bd_paged_verify_attn(*c, o, lse, bd.Workspace(size))
        want.append((o, lse))
    graphs, outs = [], []
    for c in calls:
        o, lse = torch.empty_like(c[1]), torch.empty(c[1].shape[:3], device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            bd.bd_paged_verify_attn(*c, o, lse, shared)
        graphs.append(graph)
        outs.append((o, lse))
    for order in ([0, 1, 2], [2, 1, 0], [1, 1, 0, 2]):
        for o, lse in outs:
            o.fill_(7)
            lse.fill_(7)
        for i in order:
            graphs[i].replay()
        torch.cuda.synchronize()
        for (o, lse), (wo, wl) in zip(outs, want):
            assert torch.equal(o, wo) and torch.equal(lse, wl)
    assert shared.status() == 0
    # at once, on streams of their own
    streams = [torch.cuda.Stream() for _ in calls]
    spaces = [bd.Workspace(size) for size in sizes]
    torch.cuda.synchronize()
    for _ in range(10):
        for c, s, w, (o, lse) in zip(calls, streams, spaces, outs):
            bd.bd_paged_verify_attn(*c, o, lse, w, stream=s)
    torch.cuda.synchronize()
    for w, (o, lse), (wo, wl) in zip(spaces, outs, want):
        assert w.status() == 0 and torch.equal(o, wo) and torch.equal(lse, wl)
