"""Rows that join a paged cache with their position rotation, and rows read back, on the GPU against 64 bits."""

import math
from fractions import Fraction

import pytest
import torch

import paper_2606_00144_gb300 as bd
from tests import paged_reference as ref

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def frequencies(dim, base=500000.0):
    return base ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim)


def randn(g, *s):
    return torch.randn(*s, generator=g)


def run_append(pool, lens, counts, h_q, d, dtype, rope, packed=False, t=None, by_token=False, q=True, kv=True, uniform=False,
               in_place=False, seed=0, h_kv=2):
    """Appends counts[b] tokens behind lens[b]; returns (sources, q_out, K, V) on the CPU, unused rows marked with 7."""
    g = torch.Generator().manual_seed(seed)
    b = len(lens)
    n = sum(counts) if packed else counts[0]
    behind = 4 if packed else 0        # rows behind the last sequence
    src = {}
    for name, h in (("q", h_q), ("k", h_kv), ("v", h_kv)):
        x = randn(g, h, n + behind, d) if packed else randn(g, b, h, n, d)
        src[name] = x.to(dtype)
    K, V, table = pool.cuda()

    def put(x):
        if by_token:                   # [token, heads, d] in memory
            return x.transpose(-3, -2).contiguous().cuda().transpose(-3, -2)
        return x.cuda()
    dev = {k: put(x) for k, x in src.items()}
    q_out = dev["q"] if in_place else torch.full(src["q"].shape, 7.0, dtype=BF, device="cuda")
    starts = None
    if packed:
        starts = torch.tensor([0] + torch.tensor(counts).cumsum(0).tolist(), dtype=torch.int32, device="cuda")
    seq = None if uniform else torch.tensor(lens, dtype=torch.int32, device="cuda")
    cache = bd.PagedCache(K, V)
    shape = cache.shape(b, h_q, t if t is not None else max(lens), pool.cap, seq)
    bd.bd_paged_append(shape, dev["q"] if q else None, dev["k"] if kv else None, dev["v"] if kv else None, rope, cache, table,
                       q_out if q else None, row_starts=starts)
    torch.cuda.synchronize()
    return src, q_out.cpu(), K.cpu(), V.cpu()


def check_append(pool, before, got, lens, counts, freq, interleaved, scale=1.0, packed=False, q=True, kv=True):
    src, q_out, K, V = got
    wantK, wantV = before[0].double(), before[1].double()
    tolK, tolV = torch.zeros_like(wantK), torch.zeros_like(wantV)
    done = torch.zeros(q_out.shape[:-1], dtype=torch.bool)
    at = 0
    for i, (t, n) in enumerate(zip(lens, counts)):
        pos = torch.arange(t, t + n)
        rows = {k: (x[:, at:at + n] if packed else x[i]) for k, x in src.items()}
        o = q_out[:, at:at + n] if packed else q_out[i]
        if q:
            want = ref.rotate(rows["q"], pos, freq, interleaved, scale)
            assert ((o.double() - want).abs() <= ref.rotate_tolerance(rows["q"], want, freq, interleaved, scale)).all(), f"q of {i}"
        (done[:, at:at + n] if packed else done[i])[...] = True
        at += n
        for j in range(n):
            if not kv or pos[j] >= pool.cap:
                continue
            e = int(pool.table[i, int(pos[j]) // pool.page])
            if not 0 <= e < len(K):
                continue
            r = int(pos[j]) % pool.page
            want = ref.rotate(rows["k"][:, j:j + 1], pos[j:j + 1], freq, interleaved, scale)
            wantK[e, :, r] = want[:, 0]
            tolK[e, :, r] = ref.rotate_tolerance(rows["k"][:, j:j + 1], want, freq, interleaved, scale)[:, 0]
            wantV[e, :, r] = rows["v"][:, j].double()
            tolV[e, :, r] = 2.0 ** -8 * wantV[e, :, r].abs()
    # every row of the pool: those written, and the rest as it was (NaN equal to NaN)
    for got_x, want, tol in ((K.double(), wantK, tolK), (V.double(), wantV, tolV)):
        same = (got_x.isnan() & want.isnan()) | ((got_x - want).abs() <= tol)
        assert same.all()
    if q:
        assert (q_out[~done] == 7).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("page,layout", [(16, "heads"), (32, "rows"), (64, "both")])
@pytest.mark.parametrize("lens,n", [([0], 1), ([15, 16, 17], 1), ([0, 5, 40], 21), ([31, 0, 0, 100], 6)])
def test_append_blocks(d, interleaved, dtype, page, layout, lens, n):
    pool = ref.Pool([t + n for t in lens], 2, page, d, seed=n, layout=layout)
    before = pool.k.clone(), pool.v.clone()
    freq = frequencies(d)
    got = run_append(pool, lens, [n] * len(lens), 6, d, dtype, bd.Rope(freq, interleaved), by_token=n % 2 == 1)
    check_append(pool, before, got, lens, [n] * len(lens), freq, interleaved)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("lens,counts", [([0], [1]), ([0, 0, 0], [17, 1, 40]), ([3, 900, 0, 55], [0, 33, 0, 5]), ([0] * 70, [i % 4 for i in range(70)])])
def test_append_packed_prompts(d, dtype, lens, counts):
    """Prompts of unequal lengths, empty ones among them (more sequences than a warp has lanes); rows behind the last are not
    touched."""
    pool = ref.Pool([t + n for t, n in zip(lens, counts)], 2, 16, d, seed=3)
    before = pool.k.clone(), pool.v.clone()
    freq = frequencies(d)
    got = run_append(pool, lens, counts, 4, d, dtype, bd.Rope(freq), packed=True, by_token=True)
    check_append(pool, before, got, lens, counts, freq, False, packed=True)


@pytest.mark.parametrize("rot", [16, 32, 48, 64, 112, 128])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_rotates_a_part_of_a_row(rot, interleaved):
    lens, n, d = [9, 300], 5, 128
    pool = ref.Pool([t + n for t in lens], 2, 16, d, seed=1)
    before = pool.k.clone(), pool.v.clone()
    freq = frequencies(rot, 100.0)
    got = run_append(pool, lens, [n] * 2, 4, d, torch.float32, bd.Rope(freq, interleaved, scale=1.25))
    check_append(pool, before, got, lens, [n] * 2, freq, interleaved, 1.25)


def test_append_without_a_rotation():
    lens, n, d = [9, 30], 5, 64
    pool = ref.Pool([t + n for t in lens], 2, 16, d, seed=1)
    before = pool.k.clone(), pool.v.clone()
    got = run_append(pool, lens, [n] * 2, 4, d, BF, None)
    src, q_out, K, V = got
    assert torch.equal(q_out, src["q"])
    check_append(pool, before, got, lens, [n] * 2, torch.zeros(8, dtype=torch.float64), False)


@pytest.mark.parametrize("t", [131071, (1 << 30) - 40])
def test_angles_of_far_positions(t):
    """fp32 angles would be off by up to 2^-7 turns at 131071, altogether at 2^30."""
    n, d = 3, 128
    pool = ref.Pool([64], 2, 16, d, seed=1, cap=64)
    # the sequence's last pages only: a table of t's size, its entries those of the pool's first pages
    per = -(-(t + n) // 16)
    big = torch.full((1, per), -1, dtype=torch.int32)
    for j in range(t // 16, (t + n - 1) // 16 + 1):
        big[0, j] = j - t // 16
    g = torch.Generator().manual_seed(5)
    q, k = randn(g, 1, 4, n, d), randn(g, 1, 2, n, d)
    K, V, _ = pool.cuda()
    cache = bd.PagedCache(K, V)
    q_out = torch.empty(1, 4, n, d, dtype=BF, device="cuda")
    freq = frequencies(d)
    bd.bd_paged_append(cache.shape(1, 4, t, t + n), q.cuda(), k.cuda(), k.cuda(), bd.Rope(freq), cache, big.cuda(), q_out)
    pos = torch.arange(t, t + n)
    # 64-bit angles are off by 2^-23 at 2^30 themselves: the product's part of a turn from integers
    want = torch.empty(1, 4, n, d, dtype=torch.float64)
    for i, p in enumerate(pos.tolist()):
        for j, w in enumerate(freq.tolist()):
            a = Fraction(w) * p / Fraction(628318530717958647692528676655900577, 10 ** 35)
            a = float(a - a.__floor__()) * 2 * math.pi
            x, y = q[0, :, i, j].double(), q[0, :, i, j + d // 2].double()
            want[0, :, i, j] = x * math.cos(a) - y * math.sin(a)
            want[0, :, i, j + d // 2] = x * math.sin(a) + y * math.cos(a)
    assert ((q_out.cpu().double() - want).abs() <= ref.rotate_tolerance(q, want, freq, False)).all()


def test_append_parts_and_in_place():
    """Queries alone, keys and values alone, and queries over themselves."""
    lens, n, d = [20, 3], 4, 128
    freq = frequencies(d)
    for kw in (dict(kv=False), dict(q=False), dict(in_place=True), dict(in_place=True, by_token=True)):
        pool = ref.Pool([t + n for t in lens], 2, 16, d, seed=1)
        before = pool.k.clone(), pool.v.clone()
        got = run_append(pool, lens, [n] * 2, 4, d, BF, bd.Rope(freq), **kw)
        check_append(pool, before, got, lens, [n] * 2, freq, False, q=kw.get("q", True), kv=kw.get("kv", True))


def test_pages_that_are_not_there_are_not_written():
    lens, n, d = [14, 40], 6, 64
    freq = frequencies(d)
    pool = ref.Pool([t + n for t in lens], 2, 16, d, seed=1)
    pool.table[0, 1] = -1                       # sequence 0's rows 16 .. 19
    pool.table[1, 2] = len(pool.k) + 3          # past the pool: sequence 1's rows 40 .. 45
    before = pool.k.clone(), pool.v.clone()
    got = run_append(pool, lens, [n] * 2, 4, d, BF, bd.Rope(freq))
    check_append(pool, before, got, lens, [n] * 2, freq, False)


def test_lengths_out_of_range_are_clamped_and_rows_past_the_capacity_are_not_written():
    d = 64
    freq = frequencies(d)
    pool = ref.Pool([48, 48, 48], 2, 16, d, seed=1, cap=48)
    before = pool.k.clone(), pool.v.clone()
    got = run_append(pool, [-5, 99, 10], [3] * 3, 4, d, BF, bd.Rope(freq), t=45)
    check_append(pool, before, got, [0, 45, 10], [3] * 3, freq, False)
    # packed: 60 tokens from position 10 in a cache of 48; those past the end are left alone
    pool = ref.Pool([48, 48], 2, 16, d, seed=1, cap=48)
    before = pool.k.clone(), pool.v.clone()
    src, q_out, K, V = run_append(pool, [10, 0], [60, 5], 4, d, BF, bd.Rope(freq), packed=True)
    assert (q_out[:, 38:60] == 7).all() and (q_out[:, 65:] == 7).all() and (q_out[:, :38] != 7).any(-1).all()
    assert torch.equal(V[int(pool.table[0, 2]), :, 15], src["v"][:, 37])


def test_broken_row_starts_stay_in_bounds():
    """Starts that do not ascend or pass the rows: some rows are left alone, nothing outside is touched."""
    d, b, n = 64, 3, 10
    pool = ref.Pool([32] * b, 2, 16, d, seed=1, cap=32)
    K, V, table = pool.cuda()
    cache = bd.PagedCache(K, V)
    rows = torch.ones(2, n, d, dtype=BF, device="cuda")
    for starts in ([0, 8, 2, 10], [5, 5, 5, 5], [-3, 0, 4, 1000], [1000, 0, -7, 3], [9, 8, 7, 6],
                   [-2**31, -2**31, -2**31, 10], [-2**31, 2**31 - 1, 0, 10]):
        q_out = torch.full((2, n, d), 7.0, dtype=BF, device="cuda")
        bd.bd_paged_append(cache.shape(b, 2, 0, 32), rows, rows, rows, None, cache, table, q_out,
                           row_starts=torch.tensor(starts, dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
        assert ((q_out == 7) | (q_out == 1)).all()
    unused = sorted(set(range(len(pool.k))) - set(pool.table.flatten().tolist()))
    assert K[unused].isnan().all() and V[unused].isnan().all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page,layout", [(16, "heads"), (16, "rows"), (128, "both")])
@pytest.mark.parametrize("lens", [[1], [0, 5, 77], [300, 299, 16]])
def test_read(d, page, layout, lens):
    b, h_kv, t, n = len(lens), 3, max(lens), 6
    pool = ref.Pool([x + n for x in lens], h_kv, page, d, seed=t, layout=layout)
    K, V, table = pool.cuda()
    cache = bd.PagedCache(K, V)
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
    shape = cache.shape(b, h_kv, t, pool.cap, seq)

    def expect(out, x, first, count):
        for i in range(b):
            for h in range(h_kv):
                lo = lens[i] if first is None else first
                pos = torch.arange(lo, lo + count)
                pos = pos if first is None else pos[pos < lens[i]]
                if len(pos):
                    assert torch.equal(out[i, h, :len(pos)], x[pool.table[i][pos // page].long(), h, pos % page])
                assert (out[i, h, len(pos):] == 7).all()

    for first, count in ((0, t), (t // 2, t - t // 2), (None, n), (max(0, t - 1), 1)):
        k, v = (torch.full((b, h_kv, count, d), 7.0, dtype=BF, device="cuda") for _ in "kv")
        bd.bd_paged_read(shape, cache, table, k, v, first_row=first)
        expect(k.cpu(), pool.k, first, count)
        expect(v.cpu(), pool.v, first, count)
        wide = torch.full((b, count + 2, h_kv, d + 8), 7.0, dtype=BF, device="cuda")     # rows of 16-byte alignment
        part = wide[:, 1:-1, :, 8:].transpose(1, 2)
        bd.bd_paged_read(shape, cache, table, None, part, first_row=first)
        expect(part.cpu(), pool.v, first, count)
        assert (wide[..., :8] == 7).all() and (wide[:, 0] == 7).all() and (wide[:, -1] == 7).all()


def test_pages_that_are_not_there_read_as_zeros():
    pool = ref.Pool([100, 60], 2, 16, 64, seed=2)
    pool.table[0, 1] = -1
    pool.table[0, 4] = -7
    pool.table[1, 0] = len(pool.k)
    K, V, table = pool.cuda()
    cache = bd.PagedCache(K, V)
    k = torch.full((2, 2, 100, 64), 7.0, dtype=BF, device="cuda")
    seq = torch.tensor([100, 60], dtype=torch.int32, device="cuda")
    bd.bd_paged_read(cache.shape(2, 2, 100, 100, seq), cache, table, k, first_row=0)
    k = k.cpu()
    assert (k[0, :, 16:32] == 0).all() and (k[0, :, 64:80] == 0).all() and (k[1, :, :16] == 0).all() and (k[1, :, 60:] == 7).all()
    assert torch.equal(k[0, :, 32:48], pool.k[int(pool.table[0, 2])])


def test_rows_behind_two_gigabytes_of_elements():
    """Offsets in the pool past 32 bits."""
    d, h_kv, page, n = 128, 2, 16, 20
    stride = (1 << 31) + 64
    K, V = (torch.empty(2 * stride + h_kv * page * d, dtype=BF, device="cuda").as_strided(
        (3, h_kv, page, d), (stride, page * d, d, 1)) for _ in "kv")
    for x in (K, V):
        x.fill_(math.nan)
    table = torch.tensor([[2, 1]], dtype=torch.int32, device="cuda")
    g = torch.Generator().manual_seed(0)
    q, k, v = randn(g, 1, 4, n, d).to(BF), randn(g, 1, h_kv, n, d).to(BF), randn(g, 1, h_kv, n, d).to(BF)
    cache = bd.PagedCache(K, V)
    q_out = torch.empty(1, 4, n, d, dtype=BF, device="cuda")
    bd.bd_paged_append(cache.shape(1, 4, 0, n), q.cuda(), k.cuda(), v.cuda(), None, cache, table, q_out)
    assert torch.equal(K[2, :, :16].cpu(), k[0, :, :16]) and torch.equal(V[1, :, :4].cpu(), v[0, :, 16:])
    assert K[0].isnan().all() and K[1, :, 4:].isnan().all()
    out = torch.empty(1, h_kv, n, d, dtype=BF, device="cuda")
    bd.bd_paged_read(cache.shape(1, 4, n, n), cache, table, out, first_row=0)
    assert torch.equal(out.cpu(), k)
    o, lse = torch.empty(1, 4, 1, d, dtype=BF, device="cuda"), torch.empty(1, 4, 1, device="cuda")
    s = cache.shape(1, 4, n - 1, n)
    ws = bd.Workspace(bd.bd_workspace_size(s, bd.BD_OP_PAGED_VERIFY, 0, 1))
    bd.bd_paged_verify_attn(s, q_out[:, :, -1:].contiguous(), 1, cache, table, o, lse, ws)
    idx, cnt = torch.arange(n - 1, dtype=torch.int32, device="cuda").repeat(1, h_kv, 1), torch.full((1, h_kv), n - 1, dtype=torch.int32, device="cuda")
    o2, lse2 = torch.empty(1, 4, d, dtype=BF, device="cuda"), torch.empty(1, 4, device="cuda")
    ws2 = bd.Workspace(bd.bd_workspace_size(s, bd.BD_OP_PAGED_DRAFT, n - 1, 1))
    bd.bd_paged_draft_attn(s, q_out[:, :, -1].contiguous(), cache, table, idx, cnt, n - 1, 0, o2, lse2, ws2)
    for h in range(h_kv):
        qs = q[0, 2 * h:2 * h + 2, -1]
        want = ref.attend(qs, k[0, h].double(), v[0, h].double(), torch.ones(2, n, dtype=torch.bool))
        ref.check(o[0, 2 * h:2 * h + 2, 0], lse[0, 2 * h:2 * h + 2, 0], *want)
        ref.check(o2[0, 2 * h:2 * h + 2], lse2[0, 2 * h:2 * h + 2], *want)


def test_no_rows_is_nothing():
    cache = bd.PagedCache.empty(2, 2, 16, 64)
    table = torch.zeros(1, 2, dtype=torch.int32, device="cuda")
    shape = cache.shape(1, 4, 0, 32)
    none = [torch.empty(1, h, 0, 64, dtype=BF, device="cuda") for h in (4, 2, 2, 4)]
    bd.bd_paged_append(shape, *none[:3], None, cache, table, none[3])
    some = torch.zeros(1, 4, 3, 64, dtype=BF, device="cuda")
    bd.bd_paged_append(shape, some[:, :, :0], some[:, :2, :0], some[:, 2:, :0], None, cache, table, none[3])
    starts = torch.zeros(2, dtype=torch.int32, device="cuda")
    packed = [torch.empty(h, 0, 64, dtype=BF, device="cuda") for h in (4, 2, 2, 4)]
    bd.bd_paged_append(shape, *packed[:3], None, cache, table, packed[3], row_starts=starts)
    bd.bd_paged_read(shape, cache, table, none[1], none[2], first_row=0)
    bd.bd_paged_read(shape, cache, table, none[1], first_row=32)
    torch.cuda.synchronize()


@pytest.mark.parametrize("h_q,h_kv,d", [(1, 1, 64), (3, 1, 128), (71, 1, 64), (12, 12, 128), (5, 5, 64), (64, 8, 128)])
@pytest.mark.parametrize("total", [1, 7, 3000])
def test_append_head_counts(h_q, h_kv, d, total):
    """Rows of a token that divide a CTA's slots in many ways, few tokens and many."""
    pool = ref.Pool([total], h_kv, 64, d, seed=1)
    freq = frequencies(d, 10000.0)
    got = run_append(pool, [0], [total], h_q, d, BF, bd.Rope(freq), by_token=True, h_kv=h_kv, uniform=True, t=0)
    src, q_out, K, V = got
    want = ref.rotate(src["q"][0], torch.arange(total), freq, False)
    assert ((q_out[0].double() - want).abs() <= ref.rotate_tolerance(src["q"][0], want, freq, False)).all()
    pos = torch.arange(total)
    at = pool.table[0][pos // 64].long()
    want = ref.rotate(src["k"][0], pos, freq, False)
    for h in range(h_kv):
        assert ((K[at, h, pos % 64].double() - want[h]).abs() <= ref.rotate_tolerance(src["k"][0, h], want[h], freq, False)).all()
        assert torch.equal(V[at, h, pos % 64], src["v"][0, h])


@pytest.mark.parametrize("batch", [33, 1025, 1100])
def test_packed_prompts_of_many_sequences(batch):
    """More sequences than one round of probes, and two, tell apart; many of them empty."""
    d, h = 64, 1
    g = torch.Generator().manual_seed(batch)
    counts = [int(x) for x in torch.randint(0, 4, (batch,), generator=g)]
    counts[:3], counts[-2:] = [0, 0, 2], [3, 0]
    pool = ref.Pool([max(c, 1) for c in counts], h, 16, d, seed=3, cap=16)
    K, V, table = pool.cuda()
    cache = bd.PagedCache(K, V)
    n = sum(counts)
    rows = torch.randn(h, n, d, generator=g).to(BF)
    starts = torch.tensor([0] + torch.tensor(counts).cumsum(0).tolist(), dtype=torch.int32)
    bd.bd_paged_append(cache.shape(batch, h, 0, 16), None, rows.cuda(), rows.cuda(), None, cache, table, None, row_starts=starts.cuda())
    K, V = K.cpu(), V.cpu()
    for i in range(batch):
        e = int(pool.table[i, 0])
        assert torch.equal(K[e, 0, :counts[i]], rows[0, int(starts[i]):int(starts[i + 1])])
        assert torch.equal(V[e, 0, :counts[i]], rows[0, int(starts[i]):int(starts[i + 1])])
