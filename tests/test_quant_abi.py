"""Host-side checks of the 4-bit cache's entry points (no GPU): bad arguments are refused before any launch,
by the C ABI with a status and by the binding with an exception."""

import ctypes

import pytest
import torch

import paper_2606_00144_gb300 as bd
from paper_2606_00144_gb300 import binding

BD_OK, INVALID, UNSUPPORTED, MISALIGNED, WORKSPACE = 0, -1, -2, -3, -4
A = 0x10000          # a fake, 16-byte aligned address: validation never dereferences it
BF16, F32 = binding.BD_DTYPE_BF16, binding.BD_DTYPE_F32


@pytest.fixture(scope="module")
def lib():
    bd.build()
    return bd.library()


def shape(**kw):
    base = dict(batch=2, h_q=8, h_kv=2, head_dim=128, t_ctx=100, t_cap=110)
    base.update(kw)
    return bd.make_shape(**base)


def cache(**kw):
    base = dict(k_codes=A, k_scales=A, v_codes=A, v_scales=A)
    base.update(kw)
    return ctypes.byref(binding.BdQuantCache(**base))


def strides(*s):
    return (ctypes.c_int64 * 3)(*s)


def write(lib, s, n=6, dtype=BF16, k=A, ks=None, v=A, vs=None, c=None):
    return lib.bd_quant_write(ctypes.byref(s) if s is not None else None, n, dtype, k, ks, v, vs, c or cache(), None)


def read(lib, s, first=0, n=6, dtype=BF16, k=A, ks=None, v=A, vs=None, c=None):
    return lib.bd_quant_read(ctypes.byref(s), first, n, dtype, c or cache(), k, ks, v, vs, None)


def verify(lib, s, q=A, n=6, c=None, o=A, lse=A, ws=A, nbytes=1 << 30):
    return lib.bd_quant_verify_attn(ctypes.byref(s), q, n, c or cache(), o, lse, ws, nbytes, None)


def draft(lib, s, q=A, c=None, idx=A, cnt=A, budget=32, j=0, flags=0, o=A, lse=A, ws=A, nbytes=1 << 30):
    return lib.bd_quant_draft_attn(ctypes.byref(s), q, c or cache(), idx, cnt, budget, j, flags, o, lse, ws, nbytes, None)


def test_write_validation(lib):
    assert write(lib, None) == INVALID
    assert write(lib, shape(), n=-1) == INVALID
    assert write(lib, shape(), n=11) == INVALID                       # t_ctx + n_rows > t_cap
    assert write(lib, shape(), n=2**31 - 1) == INVALID                # the sum does not wrap
    assert write(lib, shape(), n=0) == BD_OK                          # empty: no-op
    assert write(lib, shape(t_ctx=0), n=0) == BD_OK
    assert write(lib, shape(t_ctx=-1)) == INVALID
    assert write(lib, shape(head_dim=96)) == UNSUPPORTED
    assert write(lib, shape(), dtype=3) == INVALID
    assert write(lib, shape(), k=None, v=None) == INVALID
    assert write(lib, shape(), k=A + 8) == MISALIGNED
    assert write(lib, shape(), c=cache(k_codes=None)) == INVALID
    assert write(lib, shape(), c=cache(v_scales=A + 2)) == MISALIGNED
    assert write(lib, shape(), n=0, k=None, c=cache(k_codes=None, k_scales=None)) == BD_OK   # V alone
    assert lib.bd_quant_write(ctypes.byref(shape()), 1, BF16, A, None, A, None, None, None) == INVALID
    assert write(lib, shape(), ks=strides(1024, 128, 132)) == MISALIGNED      # rows of bf16: 8 elements
    assert write(lib, shape(), n=0, dtype=F32, ks=strides(1024, 128, 132)) == BD_OK
    assert write(lib, shape(), ks=strides(-1024, 128, 128)) == INVALID
    assert write(lib, shape(batch=65536, h_kv=2, h_q=2, t_ctx=0, t_cap=20000)) == UNSUPPORTED   # 2^31 rows and more


def test_read_validation(lib):
    assert read(lib, shape(), first=-2) == INVALID
    assert read(lib, shape(), first=105, n=6) == INVALID
    assert read(lib, shape(), first=-1, n=11) == INVALID              # the rows behind the context
    assert read(lib, shape(), first=2**31 - 1, n=2**31 - 1) == INVALID
    assert read(lib, shape(), first=110, n=0) == BD_OK
    assert read(lib, shape(), dtype=0) == INVALID
    assert read(lib, shape(), k=None, v=None) == INVALID
    assert read(lib, shape(), ks=strides(1536, 768, 0)) == INVALID    # rows would overwrite one another
    assert read(lib, shape(), ks=strides(1536, 768, 64)) == INVALID
    assert read(lib, shape(batch=1), n=0, ks=strides(0, 768, 128)) == BD_OK
    assert read(lib, shape(), c=cache(k_scales=None)) == INVALID


def test_verify_validation(lib):
    assert verify(lib, shape(head_dim=32)) == UNSUPPORTED
    assert verify(lib, shape(h_q=6, h_kv=4)) == INVALID
    assert verify(lib, shape(), q=None) == INVALID
    assert verify(lib, shape(), o=None) == INVALID
    assert verify(lib, shape(), o=A + 2) == MISALIGNED
    assert verify(lib, shape(), lse=A + 2) == MISALIGNED
    assert verify(lib, shape(), n=0) == INVALID
    assert verify(lib, shape(), n=11) == INVALID
    assert verify(lib, shape(t_cap=400), n=193) == UNSUPPORTED        # 4 * 193 rows > 768
    assert verify(lib, shape(), c=cache(v_codes=None)) == INVALID
    assert verify(lib, shape(), ws=None) == WORKSPACE
    assert verify(lib, shape(), ws=A + 16) == MISALIGNED
    assert verify(lib, shape(), nbytes=256) == WORKSPACE


def test_draft_validation(lib):
    assert draft(lib, shape(), idx=None) == INVALID
    assert draft(lib, shape(), cnt=A + 2) == MISALIGNED
    assert draft(lib, shape(), j=-1) == INVALID
    assert draft(lib, shape(), j=10) == INVALID
    assert draft(lib, shape(), j=2**31 - 1) == INVALID
    assert draft(lib, shape(), budget=0) == INVALID
    assert draft(lib, shape(), flags=2) == INVALID
    assert draft(lib, shape(h_q=34, h_kv=2)) == UNSUPPORTED           # group of 17
    assert draft(lib, shape(), budget=2**30) == UNSUPPORTED
    assert draft(lib, shape(), ws=None) == WORKSPACE
    assert draft(lib, shape(), nbytes=256) == WORKSPACE


def test_workspace_sizes(lib):
    def size(s, op, budget, n):
        return lib.bd_workspace_size(ctypes.byref(s), op, budget, n)

    for s in (shape(), shape(t_ctx=0), shape(batch=64, h_kv=8, t_ctx=16384, t_cap=16400), shape(h_q=2, t_cap=2000)):
        assert size(s, binding.BD_OP_QUANT_DRAFT, 512, 6) > 0
        most = size(s, binding.BD_OP_QUANT_VERIFY, 0, 21)
        # one buffer for the longest block serves every shorter one
        assert all(0 < size(s, binding.BD_OP_QUANT_VERIFY, 0, n) <= most for n in range(1, 22))
    assert size(shape(), binding.BD_OP_QUANT_VERIFY, 0, 0) == 0
    assert size(shape(), binding.BD_OP_QUANT_VERIFY, 0, 193) == 0
    assert size(shape(), binding.BD_OP_QUANT_DRAFT, 0, 1) == 0
    assert size(shape(t_ctx=0), binding.BD_OP_VERIFY, 0, 1) == 0      # the bf16 calls want a context


def cpu_cache(b=2, h=2, cap=20, d=64):
    return bd.QuantCache.empty(b, h, cap, d, device="cpu")


def test_the_cache_refuses_tensors_that_are_not_one():
    c = cpu_cache()
    assert (c.batch, c.h_kv, c.t_cap, c.head_dim) == (2, 2, 20, 64)
    assert c.nbytes == 2 * 2 * 2 * 20 * 36
    four = [c.k_codes, c.k_scales, c.v_codes, c.v_scales]

    def with_(i, t):
        return bd.QuantCache(*[t if k == i else x for k, x in enumerate(four)])

    with pytest.raises(TypeError):
        with_(0, four[0].to(torch.int8))
    with pytest.raises(TypeError):
        with_(3, four[3].float())
    with pytest.raises(ValueError):
        with_(2, four[2][:, :, :-1])
    with pytest.raises(ValueError):
        with_(1, four[1][..., :1])
    with pytest.raises(ValueError):
        with_(2, four[2].transpose(0, 1).contiguous().transpose(0, 1))
    with pytest.raises(ValueError):
        bd.QuantCache(*[t[..., :1] for t in four])


def test_the_binding_refuses_tensors_that_do_not_fit(lib):
    c = cpu_cache()
    s = c.shape(4, 10)
    rows = torch.zeros(2, 2, 3, 64, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        bd.bd_quant_write(s, rows.half(), rows.half(), c)
    with pytest.raises(TypeError):
        bd.bd_quant_write(s, rows, rows.float(), c)
    with pytest.raises(ValueError):
        bd.bd_quant_write(s, rows, rows[:, :, :2], c)
    with pytest.raises(ValueError):
        bd.bd_quant_write(s, None, None, c)
    with pytest.raises(ValueError):
        bd.bd_quant_write(s, rows.transpose(2, 3).contiguous().transpose(2, 3), None, c)
    with pytest.raises(ValueError):
        bd.bd_quant_write(cpu_cache(cap=21).shape(4, 10), rows, rows, c)   # a shape of another cache
    with pytest.raises(ValueError):
        bd.bd_quant_read(s, c, rows, first_row=-1)
    ws = type("W", (), dict(ptr=A, nbytes=1 << 20))()
    q = torch.zeros(2, 4, 3, 64, dtype=torch.bfloat16)
    lse = torch.zeros(2, 4, 3)
    with pytest.raises(TypeError):
        bd.bd_quant_verify_attn(s, q.float(), 3, c, q, lse, ws)
    with pytest.raises(ValueError):
        bd.bd_quant_verify_attn(s, q, 2, c, q, lse, ws)
    with pytest.raises(ValueError):
        bd.bd_quant_verify_attn(s, q, 3, c, q.transpose(1, 2).contiguous().transpose(1, 2), lse, ws)
    with pytest.raises(TypeError):
        bd.bd_quant_verify_attn(s, q, 3, c, q, lse.double(), ws)
    idx, count = torch.zeros(2, 2, 8, dtype=torch.int32), torch.zeros(2, 2, dtype=torch.int32)
    with pytest.raises(ValueError):
        bd.bd_quant_draft_attn(s, q[:, :, 0].contiguous(), c, idx, count, 9, 0, q[:, :, 0].contiguous(), None, ws)
    with pytest.raises(TypeError):
        bd.bd_quant_draft_attn(s, q[:, :, 0].contiguous(), c, idx.long(), count, 8, 0, q[:, :, 0].contiguous(), None, ws)


def test_the_binding_refuses_tensors_that_are_not_on_the_gpu(lib):
    """All of them fit but for where they are: no call reaches the library with a host pointer."""
    c = cpu_cache()
    s = c.shape(4, 10)
    rows = torch.zeros(2, 2, 3, 64, dtype=torch.bfloat16)
    ws = type("W", (), dict(ptr=A, nbytes=1 << 30))()
    q, lse = torch.zeros(2, 4, 3, 64, dtype=torch.bfloat16), torch.zeros(2, 4, 3)
    q1 = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    idx, count = torch.zeros(2, 2, 8, dtype=torch.int32), torch.zeros(2, 2, dtype=torch.int32)
    for call in (lambda: bd.bd_quant_write(s, rows, rows, c), lambda: bd.bd_quant_read(s, c, rows, None, first_row=0),
                 lambda: bd.bd_quant_verify_attn(s, q, 3, c, q, lse, ws),
                 lambda: bd.bd_quant_draft_attn(s, q1, c, idx, count, 8, 0, q1, None, ws)):
        with pytest.raises(ValueError, match="on the GPU"):
            call()
