"""Writes and reads of no rows, as a loop makes them with an empty tensor, whose pointer is null: they do nothing."""

import pytest
import torch

import paper_2606_00144_gb300 as bd
from tests.test_quant_abi import BD_OK, BF16, F32, INVALID, MISALIGNED, cache, lib, read, shape, write  # noqa: F401


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_null_rows_are_a_no_op_where_there_are_none(lib, dtype):  # noqa: F811
    for call in (write, read):
        assert call(lib, shape(), n=0, dtype=dtype, k=None, v=None) == BD_OK
        assert call(lib, shape(), n=0, dtype=dtype, k=None) == BD_OK
        assert call(lib, shape(t_ctx=110), n=0, dtype=dtype, k=None, v=None) == BD_OK
        # anything else is refused as before
        assert call(lib, shape(), n=1, dtype=dtype, k=None, v=None) == INVALID
        assert call(lib, shape(), n=-1, dtype=dtype, k=None, v=None) == INVALID
        assert call(lib, shape(), n=0, dtype=7, k=None, v=None) == INVALID
        assert call(lib, shape(t_ctx=111), n=0, dtype=dtype, k=None, v=None) == INVALID
        assert call(lib, shape(), n=0, dtype=dtype, c=cache(k_codes=0x10008)) == MISALIGNED


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_empty_tensors(dtype):
    cache = bd.QuantCache.empty(2, 2, 20, 64)
    for x in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales):
        x.fill_(3)
    s = cache.shape(4, 10)
    rows = torch.zeros(2, 2, 5, 64, dtype=dtype, device="cuda")
    for none in (rows[:, :, :0], torch.empty(2, 2, 0, 64, dtype=dtype, device="cuda")):
        bd.bd_quant_write(s, none, none, cache)
        bd.bd_quant_write(s, none, None, cache)
        bd.bd_quant_read(s, cache, none, none)
        bd.bd_quant_read(s, cache, none, none, first_row=20)
        bd.bd_quant_read(s, cache, none, None, first_row=0)
    torch.cuda.synchronize()
    assert all((x == 3).all() for x in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales))
    with pytest.raises(bd.BudgetDraftError):
        bd.bd_quant_read(s, cache, rows[:, :, :0], None, first_row=21)
