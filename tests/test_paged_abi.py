"""Host-side checks of the paged cache's entry points (no GPU): bad arguments are refused before any launch, by the C ABI
with a status and by the binding with an exception."""

import ctypes
import types

import pytest
import torch

import paper_2606_00144_gb300 as bd
from paper_2606_00144_gb300 import binding

BD_OK, INVALID, UNSUPPORTED, MISALIGNED, WORKSPACE = 0, -1, -2, -3, -4
A = 0x10000          # a fake, 16-byte aligned address: validation never dereferences it
BF16, F32 = binding.BD_DTYPE_BF16, binding.BD_DTYPE_F32
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    bd.build()
    return bd.library()


def shape(**kw):
    base = dict(batch=2, h_q=8, h_kv=2, head_dim=128, t_ctx=100, t_cap=112)
    base.update(kw)
    return bd.make_shape(**base)


def strides(*s):
    return (ctypes.c_int64 * 3)(*s)


def cache(**kw):
    base = dict(k=A, v=A, k_strides=strides(4096, 2048, 128), v_strides=strides(4096, 2048, 128), n_pages=20, page_size=16)
    base.update(kw)
    return ctypes.byref(binding.BdPagedCache(**base))


def rope(**kw):
    base = dict(turns=A, dim=128, interleaved=0, scale=1.0)
    base.update(kw)
    return ctypes.byref(binding.BdRope(**base))


def append(lib, s, n=6, dtype=BF16, q=A, qs=None, k=A, ks=None, v=A, vs=None, starts=None, r=None, c=None, table=A, pages=7, o=A, os=None):
    return lib.bd_paged_append(ctypes.byref(s) if s is not None else None, n, dtype, q, qs, k, ks, v, vs, starts, r or rope(), c or cache(),
                               table, pages, o, os, None)


def read(lib, s, first=0, n=6, c=None, table=A, pages=7, k=A, ks=None, v=A, vs=None):
    return lib.bd_paged_read(ctypes.byref(s), first, n, c or cache(), table, pages, k, ks, v, vs, None)


def verify(lib, s, q=A, n=6, c=None, table=A, pages=7, o=A, lse=A, ws=A, nbytes=BIG):
    return lib.bd_paged_verify_attn(ctypes.byref(s), q, n, c or cache(), table, pages, o, lse, ws, nbytes, None)


def draft(lib, s, q=A, c=None, table=A, pages=7, idx=A, cnt=A, budget=32, j=0, flags=0, o=A, lse=A, ws=A, nbytes=BIG):
    return lib.bd_paged_draft_attn(ctypes.byref(s), q, c or cache(), table, pages, idx, cnt, budget, j, flags, o, lse, ws, nbytes, None)


def test_append_validation(lib):
    assert append(lib, None) == INVALID
    assert append(lib, shape(), n=-1) == INVALID
    assert append(lib, shape(), n=13) == INVALID                      # t_ctx + n_rows > t_cap
    assert append(lib, shape(), n=2**31 - 1) == INVALID               # the sum does not wrap
    assert append(lib, shape(), n=0) == BD_OK                         # empty: no-op
    assert append(lib, shape(t_ctx=0), n=0) == BD_OK
    assert append(lib, shape(), n=0, q=None, k=None, v=None, o=None) == BD_OK
    assert append(lib, shape(), n=0, starts=A) == BD_OK
    assert append(lib, shape(), starts=A + 2) == MISALIGNED
    assert append(lib, shape(t_ctx=-1)) == INVALID
    assert append(lib, shape(head_dim=96)) == UNSUPPORTED
    assert append(lib, shape(), dtype=3) == INVALID
    assert append(lib, shape(), q=None, k=None, v=None, o=None) == INVALID
    assert append(lib, shape(), q=None) == INVALID                    # q_out without q_rows
    assert append(lib, shape(), o=None) == INVALID
    assert append(lib, shape(), k=A + 8) == MISALIGNED
    assert append(lib, shape(), o=A + 8) == MISALIGNED
    assert append(lib, shape(), ks=strides(1024, 128, 132)) == MISALIGNED     # rows of bf16: 8 elements
    assert append(lib, shape(), n=0, dtype=F32, ks=strides(1024, 128, 132)) == BD_OK
    assert append(lib, shape(), ks=strides(-1024, 128, 128)) == INVALID
    assert append(lib, shape(), os=strides(6144, 768, 64)) == INVALID         # rows would overwrite one another
    assert append(lib, shape(), os=strides(6144, 0, 128)) == INVALID
    for bad in (dict(dim=8), dict(dim=24), dict(dim=144), dict(dim=0), dict(interleaved=2), dict(turns=None)):
        assert append(lib, shape(), r=rope(**bad)) == INVALID, bad
    assert append(lib, shape(), r=rope(turns=A + 4)) == MISALIGNED
    assert append(lib, shape(head_dim=64), r=rope(dim=128)) == INVALID
    assert append(lib, shape(batch=8, t_ctx=0, t_cap=1 << 30), n=1 << 28, pages=1 << 26) == UNSUPPORTED   # 2^31 tokens


def test_the_cache_and_its_table_are_checked_by_every_call(lib):
    calls = [append, read, verify, draft]
    for call in calls:
        assert call(lib, shape(), c=cache(n_pages=0)) == INVALID
        assert call(lib, shape(), c=cache(page_size=0)) == INVALID
        assert call(lib, shape(), c=cache(page_size=8)) == UNSUPPORTED
        assert call(lib, shape(), c=cache(page_size=48)) == UNSUPPORTED
        assert call(lib, shape(), c=cache(n_pages=1 << 27)) == UNSUPPORTED               # 2^31 rows
        assert call(lib, shape(), c=cache(k=None)) == INVALID
        assert call(lib, shape(), c=cache(v=A + 8)) == MISALIGNED
        assert call(lib, shape(), c=cache(k_strides=strides(4096, 2048, 64))) == INVALID
        assert call(lib, shape(), c=cache(k_strides=strides(0, 2048, 128))) == INVALID
        assert call(lib, shape(), c=cache(v_strides=strides(1 << 39, 2048, 128))) == INVALID
        assert call(lib, shape(), c=cache(v_strides=strides(4100, 2048, 128))) == MISALIGNED
        assert call(lib, shape(), table=None) == INVALID
        assert call(lib, shape(), table=A + 2) == MISALIGNED
        assert call(lib, shape(), pages=6) == INVALID                                    # 96 positions of 112
        assert call(lib, shape(), pages=0) == INVALID
        assert call(lib, shape(head_dim=32)) == UNSUPPORTED
        assert call(lib, shape(h_q=6, h_kv=4)) == INVALID
        assert call(lib, shape(t_cap=(1 << 30) + 1), pages=1 << 27) == UNSUPPORTED
        assert call(lib, shape(batch=1 << 19), pages=7) == UNSUPPORTED                   # 2^20 (sequence, KV head) units
    # what a size of one strides does not matter
    one = shape(batch=1, h_q=4, h_kv=1)
    assert append(lib, one, n=0, c=cache(n_pages=1, k_strides=strides(3, 5, 128))) == BD_OK
    s = shape()
    s.seq_lens = A + 2
    assert all(call(lib, s) == MISALIGNED for call in calls)


def test_read_validation(lib):
    assert read(lib, shape(), first=-2) == INVALID
    assert read(lib, shape(), first=107, n=6) == INVALID
    assert read(lib, shape(), first=-1, n=13) == INVALID              # the rows behind the context
    assert read(lib, shape(), first=2**31 - 1, n=2**31 - 1) == INVALID
    assert read(lib, shape(), first=112, n=0) == BD_OK
    assert read(lib, shape(), k=None, v=None) == INVALID
    assert read(lib, shape(), n=0, k=None, v=None) == BD_OK
    assert read(lib, shape(), k=A + 8) == MISALIGNED
    assert read(lib, shape(), ks=strides(1536, 768, 0)) == INVALID    # rows would overwrite one another
    assert read(lib, shape(), ks=strides(1536, 768, 132)) == MISALIGNED
    assert read(lib, shape(), n=0, v=None, c=cache(v=None)) == BD_OK  # K alone


def test_verify_validation(lib):
    assert verify(lib, shape(), q=None) == INVALID
    assert verify(lib, shape(), o=None) == INVALID
    assert verify(lib, shape(), o=A + 2) == MISALIGNED
    assert verify(lib, shape(), lse=A + 2) == MISALIGNED
    assert verify(lib, shape(), n=0) == INVALID
    assert verify(lib, shape(), n=13) == INVALID
    assert verify(lib, shape(t_cap=400), n=193, pages=25) == UNSUPPORTED        # 4 * 193 rows > 768
    assert verify(lib, shape(), ws=None) == WORKSPACE
    assert verify(lib, shape(), ws=A + 16) == MISALIGNED
    assert verify(lib, shape(), nbytes=256) == WORKSPACE
    s = shape(batch=4096)
    s.seq_lens = A
    assert verify(lib, s) == UNSUPPORTED


def test_draft_validation(lib):
    assert draft(lib, shape(), idx=None) == INVALID
    assert draft(lib, shape(), cnt=A + 2) == MISALIGNED
    assert draft(lib, shape(), j=-1) == INVALID
    assert draft(lib, shape(), j=12) == INVALID
    assert draft(lib, shape(), j=2**31 - 1) == INVALID
    assert draft(lib, shape(), budget=0) == INVALID
    assert draft(lib, shape(), flags=2) == INVALID
    assert draft(lib, shape(h_q=34, h_kv=2)) == UNSUPPORTED           # group of 17
    assert draft(lib, shape(), budget=2**31 - 1) == UNSUPPORTED
    assert draft(lib, shape(), ws=None) == WORKSPACE
    assert draft(lib, shape(), ws=A + 16) == MISALIGNED
    assert draft(lib, shape(), nbytes=256) == WORKSPACE


def test_workspace_sizes(lib):
    def size(op, budget, n, lens=None, **kw):
        s = shape(**kw)
        s.seq_lens = lens
        return lib.bd_workspace_size(ctypes.byref(s), op, budget, n)

    V, D = bd.BD_OP_PAGED_VERIFY, bd.BD_OP_PAGED_DRAFT
    assert size(V, 0, 0) == 0 and size(D, 0, 1) == 0 and size(D, 64, 0) == 0
    assert size(V, 0, 193) == 0
    assert size(V, 0, 192) > 0
    assert size(V, 0, 6, head_dim=96) == 0
    # one size for every length up to t_cap, and for shorter blocks
    for lens in (None, A):
        for n in (1, 6, 21, 60):
            sizes = {t: size(V, 0, n, lens, t_ctx=t, t_cap=100_000, batch=8, h_q=32, h_kv=8) for t in (0, 1, 700, 9000, 65536)}
            assert len(set(sizes.values())) == 1 and min(sizes.values()) > 0, sizes
            assert all(size(V, 0, m, lens, t_cap=100_000, batch=8, h_q=32, h_kv=8) <= sizes[0] for m in range(1, n))


# ------------------------------------------------------------------------------------ the binding


class Placed:
    """A CPU tensor that claims to be on GPU `index`."""

    def __init__(self, t, index=0):
        self._t, self._index = t, index
        self.is_cuda, self.device = True, torch.device("cuda", index)

    def get_device(self):
        return self._index

    def data_ptr(self):
        return A

    def __getattr__(self, name):
        return getattr(self._t, name)


def bf(*s, index=0):
    return Placed(torch.zeros(*s, dtype=torch.bfloat16), index)


def i32(*s, index=0):
    return Placed(torch.zeros(*s, dtype=torch.int32), index)


def f32(*s, index=0):
    return Placed(torch.zeros(*s), index)


def test_pools_that_are_none():
    good = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    bd.PagedCache(good, good)
    bd.PagedCache(good.transpose(1, 2).contiguous().transpose(1, 2), good)
    for k, v, err in [(good[0], good[0], ValueError), (good, good[:3], ValueError), (good.float(), good.float(), TypeError),
                      (good[:, :, :8], good[:, :, :8], ValueError), (good[..., :32], good[..., :32], ValueError),
                      (good.transpose(2, 3), good.transpose(2, 3), ValueError),
                      (torch.zeros(4, 2, 48, 64, dtype=torch.bfloat16),) * 2 + (ValueError,),
                      (Placed(good, 0), Placed(good, 1), ValueError)]:
        with pytest.raises(err):
            bd.PagedCache(k, v)


def test_ropes():
    r = bd.Rope.of_base(128, 10000.0, device="cpu")
    # a turn is 2^64: pair 0 turns by a radian a position
    assert abs(int(r.turns[0]) % 2**64 / 2**64 - 0.15915494309189535) < 2.0 ** -52
    assert bd.Rope([-1.0] * 8, device="cpu").turns[0] == -r.turns[0]
    assert r.dim == 128 and not r.interleaved
    for bad in ([], [1.0] * 7, [1.0] * 72, [float("inf")] * 8, [[1.0] * 8]):
        with pytest.raises(ValueError):
            bd.Rope(bad, device="cpu")
    with pytest.raises(ValueError):
        bd.Rope([1.0] * 8, scale=float("nan"), device="cpu")


def setting():
    c = bd.PagedCache(bf(4, 2, 16, 64), bf(4, 2, 16, 64))
    return c, c.shape(2, 4, 10, 20), i32(2, 2)


def test_the_binding_refuses_rows(lib):
    c, s, table = setting()
    q, k, o = bf(2, 4, 3, 64), bf(2, 2, 3, 64), bf(2, 4, 3, 64)
    r = types.SimpleNamespace(_gpu=0, dim=64, _struct=None)

    def bad(err, match, **kw):
        a = dict(shape=s, q_rows=q, k_rows=k, v_rows=k, rope=r, cache=c, table=table, q_out=o)
        a.update(kw)
        with pytest.raises(err, match=match):
            bd.bd_paged_append(**a)

    bad(ValueError, "shape", shape=c.shape(2, 4, 10, 20).__class__(2, 4, 1, 64, 10, 20, None))
    bad(TypeError, "table", table=Placed(torch.zeros(2, 2, dtype=torch.int64)))
    bad(ValueError, "table", table=i32(3, 2))
    bad(ValueError, "table", table=i32(4))
    bad(ValueError, "GPU", table=i32(2, 2, index=1))
    bad(ValueError, "rows of", q_rows=None, k_rows=None, v_rows=None, q_out=None)
    bad(ValueError, "together", q_out=None)
    bad(TypeError, "bf16 or fp32", q_rows=Placed(torch.zeros(2, 4, 3, 64).half()))
    bad(TypeError, "bf16", k_rows=f32(2, 2, 3, 64))
    bad(TypeError, "bf16", q_out=f32(2, 4, 3, 64))
    bad(ValueError, "rows must be", k_rows=bf(2, 2, 4, 64))
    bad(ValueError, "rows must be", q_rows=bf(4, 3, 64))
    bad(ValueError, "adjacent", k_rows=Placed(torch.zeros(2, 2, 64, 3, dtype=torch.bfloat16).transpose(2, 3)))
    bad(ValueError, "GPU", v_rows=bf(2, 2, 3, 64, index=1))
    bad(ValueError, "GPU", rope=types.SimpleNamespace(_gpu=1, dim=64))
    bad(ValueError, "head_dim", rope=types.SimpleNamespace(_gpu=0, dim=128))
    bad(ValueError, "packed", row_starts=i32(3))
    packed = dict(q_rows=bf(4, 5, 64), k_rows=bf(2, 5, 64), v_rows=bf(2, 5, 64), q_out=bf(4, 5, 64))
    bad(ValueError, "row_starts", row_starts=i32(2), **packed)
    bad(TypeError, "row_starts", row_starts=Placed(torch.zeros(3, dtype=torch.int64)), **packed)
    bad(ValueError, "GPU", row_starts=i32(3, index=1), **packed)
    with pytest.raises(ValueError, match="rows must be"):
        bd.bd_paged_read(s, c, table, bf(2, 4, 3, 64), first_row=0)
    with pytest.raises(ValueError, match="negative"):
        bd.bd_paged_read(s, c, table, k, first_row=-1)
    with pytest.raises(ValueError, match="rows"):
        bd.bd_paged_read(s, c, table, None)
    with pytest.raises(TypeError):
        bd.bd_paged_read(s, c, table, f32(2, 2, 3, 64), first_row=0)


def test_the_binding_refuses_attention_tensors(lib):
    c, s, table = setting()
    ws = types.SimpleNamespace(ptr=A, nbytes=BIG, buf=bf(1))
    far = types.SimpleNamespace(ptr=A, nbytes=BIG, buf=bf(1, index=1))
    q, o, lse = bf(2, 4, 3, 64), bf(2, 4, 3, 64), f32(2, 4, 3)
    for a, err in [((bf(2, 4, 2, 64), o, lse, ws), ValueError), ((f32(2, 4, 3, 64), o, lse, ws), TypeError),
                   ((q, bf(2, 4, 3, 64, index=1), lse, ws), ValueError), ((q, o, f32(2, 4), ws), ValueError),
                   ((q, o, f32(2, 4, 3, index=1), ws), ValueError), ((q, o, lse, far), ValueError)]:
        with pytest.raises(err):
            bd.bd_paged_verify_attn(s, a[0], 3, c, table, *a[1:])
    q, o, lse, idx, cnt = bf(2, 4, 64), bf(2, 4, 64), f32(2, 4), i32(2, 2, 8), i32(2, 2)
    for a in [(bf(2, 4, 1, 64), idx, cnt), (q, i32(2, 2, 7), cnt), (q, idx, i32(4)), (q, i32(2, 2, 8, index=1), cnt)]:
        with pytest.raises(ValueError):
            bd.bd_paged_draft_attn(s, a[0], c, table, a[1], a[2], 8, 0, o, lse, ws)


def test_a_call_runs_with_the_caches_gpu_current(monkeypatch):
    """Tensors on GPU 1 while GPU 0 is current: every call reaches the library on GPU 1, with that GPU's stream, once."""
    current, calls = [0], []

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            self.before, current[0] = current[0], self.index

        def __exit__(self, *_):
            current[0] = self.before

    class Library:
        def __getattr__(self, name):
            return lambda *a: calls.append((name, current[0], a)) or 0

    monkeypatch.setattr(binding, "_lib", Library())
    monkeypatch.setattr(binding, "_device", lambda: current[0])
    monkeypatch.setattr(binding, "_raw_stream", lambda gpu: 100 + gpu)
    monkeypatch.setattr(torch.cuda, "device", Device)

    def at(make, *shape):
        return make(*shape, index=1)

    c = bd.PagedCache(at(bf, 4, 2, 16, 64), at(bf, 4, 2, 16, 64))
    s, table, ws = c.shape(2, 4, 10, 20), at(i32, 2, 2), types.SimpleNamespace(ptr=A, nbytes=BIG, buf=at(bf, 1))
    q, kv = at(bf, 2, 4, 3, 64), at(bf, 2, 2, 3, 64)
    bd.bd_paged_append(s, q, kv, kv, None, c, table, q)
    bd.bd_paged_read(s, c, table, kv)
    bd.bd_paged_read(s, c, table, kv, first_row=2)
    bd.bd_paged_verify_attn(s, q, 3, c, table, q, None, ws)
    bd.bd_paged_draft_attn(s, at(bf, 2, 4, 64), c, table, at(i32, 2, 2, 8), at(i32, 2, 2), 8, 1, at(bf, 2, 4, 64), None, ws)
    assert [(name, gpu, a[-1]) for name, gpu, a in calls] == [(x, 1, 101) for x in (
        "bd_paged_append", "bd_paged_read", "bd_paged_read", "bd_paged_verify_attn", "bd_paged_draft_attn")]
    assert [a[1] for _, _, a in calls[1:3]] == [binding.BD_PAGED_BLOCK_ROWS, 2] and current[0] == 0
