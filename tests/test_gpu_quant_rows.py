"""bd_quant_write and bd_quant_read on the GPU: codes and scales are those of the definition, bit for
bit, and rows read back are the values they stand for; nothing else in the cache is touched."""

import math

import pytest
import torch

import paper_2606_00144_gb300 as bd
from tests import quant_reference as ref

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def rows(shape, dtype, seed=0):
    """Rows of every kind a group can be: sizes over many octaves, zeros, ties, one large element."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g) * torch.exp2(torch.randint(-30, 30, (*shape[:-1], 1), generator=g).float())
    kind = torch.randint(0, 8, (*shape[:-1], 1), generator=g)
    x = torch.where(kind == 0, torch.zeros_like(x), x)
    # quotients that lie half way between two codes: multiples of half the scale (7 / 7 = 1)
    half = torch.randint(-14, 15, shape, generator=g) / 2.0
    half[..., 0::32] = 7.0
    x = torch.where(kind == 1, half, x)
    x = torch.where((kind == 2) & (torch.rand(shape, generator=g) < 0.03), 100 * x, x)
    return x.to(dtype)


def filled(b, h, cap, d, seed=5):
    g = torch.Generator().manual_seed(seed)
    codes = [torch.randint(0, 256, (b, h, cap, d // 2), generator=g, dtype=torch.uint8) for _ in range(2)]
    scales = [torch.rand(b, h, cap, d // 32, generator=g).to(BF) for _ in range(2)]
    return codes, scales


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("b,h,d,t,n,lens", [
    (1, 1, 64, 0, 1, None), (1, 2, 128, 5, 6, None), (3, 2, 64, 33, 7, [33, 0, 9]), (2, 3, 128, 1, 1, [0, 1]),
    (2, 8, 128, 0, 333, None), (4, 1, 64, 700, 129, [1, 700, 350, 0]), (1, 32, 128, 40, 21, None),
])
def test_written_rows_are_the_definition(b, h, d, t, n, lens, dtype):
    cap = t + n + 2
    k, v = rows((b, h, n, d), dtype, 1), rows((b, h, n, d), dtype, 2)
    codes, scales = filled(b, h, cap, d)
    cache = bd.QuantCache(*(x.cuda() for pair in zip(codes, scales) for x in pair))
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda") if lens else None
    shape = cache.shape(2 * h, t, seq)
    bd.bd_quant_write(shape, k.cuda(), v.cuda(), cache)
    for which, x in enumerate((k, v)):
        want_c, want_s = codes[which].clone(), scales[which].clone()
        qc, qs = ref.quantise(x)
        for i in range(b):
            at = lens[i] if lens else t
            want_c[i, :, at:at + n], want_s[i, :, at:at + n] = qc[i], qs[i]
        got_c, got_s = (cache.k_codes, cache.k_scales) if which == 0 else (cache.v_codes, cache.v_scales)
        assert torch.equal(got_s.cpu().view(torch.int16), want_s.view(torch.int16))
        assert torch.equal(got_c.cpu(), want_c)
    # read back: the block's rows, then a range of context rows, in both types
    for out_dtype in (BF, F32):
        ko, vo = (torch.full((b, h, n, d), 3.0, dtype=out_dtype, device="cuda") for _ in range(2))
        bd.bd_quant_read(shape, cache, ko, vo)
        for got, x in ((ko, k), (vo, v)):
            want = ref.values(*ref.quantise(x)).float().to(out_dtype)
            assert torch.equal(got.cpu(), want)
    first, m = cap // 3, cap - cap // 3
    ko = torch.empty(b, h, m, d, dtype=F32, device="cuda")
    bd.bd_quant_read(shape, cache, ko, None, first_row=first)
    want = ref.values(cache.k_codes.cpu(), cache.k_scales.cpu())[:, :, first:]
    assert torch.equal(ko.cpu(), want.float())


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rows_of_any_strides(dtype):
    """Rows as a projection leaves them, [batch, row, head, d] inside a wider buffer, and a read into rows of a
    longer cache; the tensor that is not given keeps its rows."""
    b, h, n, d, t = 2, 4, 19, 128, 11
    qkv = rows((b, n, 3 * h, d), dtype, 3).cuda()
    k, v = qkv[:, :, h:2 * h].transpose(1, 2), qkv[:, :, 2 * h:].transpose(1, 2)
    cache = bd.QuantCache.empty(b, h, t + n, d)
    shape = cache.shape(h, t)
    bd.bd_quant_write(shape, k, v, cache)
    for codes, scales, x in ((cache.k_codes, cache.k_scales, k), (cache.v_codes, cache.v_scales, v)):
        qc, qs = ref.quantise(x.cpu().contiguous())
        assert torch.equal(codes[:, :, t:].cpu(), qc)
        assert torch.equal(scales[:, :, t:].cpu().view(torch.int16), qs.view(torch.int16))
    before = cache.k_codes.clone()
    bd.bd_quant_write(shape, None, k, cache)
    assert torch.equal(cache.k_codes, before)
    assert torch.equal(cache.v_codes[:, :, t:].cpu(), ref.quantise(k.cpu().contiguous())[0])
    wide = torch.full((b, h, 2 * n, d), 9.0, dtype=dtype, device="cuda")
    bd.bd_quant_read(shape, cache, wide[:, :, 3:3 + n], None, first_row=t)
    assert torch.equal(wide[:, :, 3:3 + n].cpu(), ref.values(*ref.quantise(k.cpu().contiguous())).float().to(dtype))
    assert (wide[:, :, :3] == 9).all() and (wide[:, :, 3 + n:] == 9).all()
    # one row for every sequence and head: strides of 0 are fine in a source
    one = rows((1, 1, 1, d), dtype, 4).cuda().expand(b, h, n, d)
    bd.bd_quant_write(shape, one, one, cache)
    assert (cache.k_codes[:, :, t:] == cache.k_codes[0, 0, t]).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_groups_that_are_not_numbers(dtype):
    """A NaN or an infinity makes its group NaN and no other; the smallest and largest numbers survive."""
    b, h, n, d = 1, 1, 8, 64
    x = torch.ones(b, h, n, d)
    x[0, 0, 0, 3] = math.nan
    x[0, 0, 1, 40] = math.inf
    x[0, 0, 2, 5] = -math.inf
    x[0, 0, 3, :] = 0
    x[0, 0, 4, :] = torch.linspace(-1, 1, d) * torch.finfo(BF).max
    x[0, 0, 5, :] = torch.linspace(-1, 1, d) * 2.0 ** -120
    x[0, 0, 6, :] = 2.0 ** -133          # a scale of 2^-133 / 7 rounds to 0 in bf16
    x[0, 0, 7, :] = -0.0
    x = x.to(dtype)
    cache = bd.QuantCache.empty(b, h, n, d)
    shape = cache.shape(1, 0)
    bd.bd_quant_write(shape, x.cuda(), x.cuda(), cache)
    qc, qs = ref.quantise(x)
    assert torch.equal(cache.k_codes.cpu(), qc)
    assert torch.equal(torch.nan_to_num(cache.k_scales.cpu().float(), nan=-5), torch.nan_to_num(qs.float(), nan=-5))
    out = torch.empty(b, h, n, d, dtype=F32, device="cuda")
    bd.bd_quant_read(shape, cache, out)
    nan = out.isnan().cpu()[0, 0]
    assert nan[0, :32].all() and not nan[0, 32:].any()
    assert nan[1, 32:].all() and not nan[1, :32].any() and nan[2, :32].all()
    assert not nan[3:].any()
    assert (out.cpu()[0, 0, 4] - x[0, 0, 4].float()).abs().max() <= torch.finfo(BF).max / 13


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rows_that_are_sixteen_bytes_aligned(dtype):
    """Rows that start on 16 but not on 32 bytes, in and out."""
    b, h, n, d = 2, 2, 37, 64
    off = 8 if dtype == BF else 4
    wide = rows((b, h, n, d + 2 * off), F32, 8).to(dtype).cuda()
    x = wide[..., off:off + d]
    assert x.data_ptr() % 32 == 16
    cache = bd.QuantCache.empty(b, h, n, d)
    shape = cache.shape(h, 0)
    bd.bd_quant_write(shape, x, x, cache)
    qc, qs = ref.quantise(x.cpu().contiguous())
    assert torch.equal(cache.v_codes.cpu(), qc) and torch.equal(cache.k_scales.cpu().view(torch.int16), qs.view(torch.int16))
    out = torch.full_like(wide, 5.0)
    bd.bd_quant_read(shape, cache, out[..., off:off + d], None, first_row=0)
    assert torch.equal(out[..., off:off + d].cpu(), ref.values(qc, qs).float().to(dtype))
    assert (out[..., :off] == 5).all() and (out[..., off + d:] == 5).all()


def test_groups_of_every_scale():
    """Scales over the whole range of bf16, subnormal ones among them, at quotients on and beside the ties."""
    e = torch.arange(-126, 121)
    x = torch.zeros(1, 1, len(e), 64)
    step = torch.arange(-16, 16) / 2.0
    step[0] = 7.0
    for i, k in enumerate(e.tolist()):
        x[0, 0, i, :32] = step * 2.0 ** k                       # ties: the scale is 2^k
        x[0, 0, i, 32:] = step * (1 + 2.0 ** -7) * 2.0 ** k
    x = x.clamp(-torch.finfo(BF).max, torch.finfo(BF).max)
    for dtype in (BF, F32):
        y = x.to(dtype)
        cache = bd.QuantCache.empty(1, 1, len(e), 64)
        shape = cache.shape(1, 0)
        bd.bd_quant_write(shape, y.cuda(), y.cuda(), cache)
        qc, qs = ref.quantise(y)
        assert torch.equal(cache.k_scales.cpu().view(torch.int16), qs.view(torch.int16))
        assert torch.equal(cache.k_codes.cpu(), qc)
        out = torch.empty(1, 1, len(e), 64, dtype=dtype, device="cuda")
        bd.bd_quant_read(shape, cache, out, None, first_row=0)
        assert torch.equal(out.cpu(), ref.values(qc, qs).float().to(dtype))


def test_an_empty_write_and_read():
    cache = bd.QuantCache.empty(2, 2, 9, 64)
    cache.k_codes.fill_(0x35)
    shape = cache.shape(2, 4)
    none = torch.empty(2, 2, 0, 64, dtype=BF, device="cuda")
    pad = torch.empty(16, dtype=BF, device="cuda")
    assert bd.library().bd_quant_write(bd.binding.ctypes.byref(shape), 0, bd.BD_DTYPE_BF16, pad.data_ptr(), None, None, None,
                                       bd.binding.ctypes.byref(cache._struct), None) == 0
    assert none.numel() == 0 and (cache.k_codes == 0x35).all()


def test_write_and_read_on_a_stream_of_their_own():
    """Rows made on one stream, written on another that waits for it, read back on a third."""
    b, h, n, d = 2, 4, 257, 128
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    cache = bd.QuantCache.empty(b, h, n, d)
    shape = cache.shape(h, 0)
    x = rows((b, h, n, d), BF, 6).cuda()
    torch.cuda.synchronize()
    s1.wait_stream(torch.cuda.current_stream())
    bd.bd_quant_write(shape, x, x, cache, stream=s1)
    s2.wait_stream(s1)
    out = torch.empty(b, h, n, d, dtype=F32, device="cuda")
    bd.bd_quant_read(shape, cache, out, stream=s2)
    torch.cuda.synchronize()
    assert torch.equal(out.cpu(), ref.values(*ref.quantise(x.cpu())).float())
