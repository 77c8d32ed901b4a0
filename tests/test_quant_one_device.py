"""The 4-bit calls' tensors are on the cache's GPU: one on another is refused before any launch.  (Tensors that only say
where they are: no GPU is asked.)"""

import types

import pytest
import torch

import paper_2606_00144_gb300 as bd
from tests.test_quant_abi import A, lib  # noqa: F401


class Placed:
    """A CPU tensor that claims to be on GPU `index`."""

    def __init__(self, t, index):
        self._t, self._index = t, index
        self.is_cuda, self.device = True, torch.device("cuda", index)

    def get_device(self):
        return self._index

    def data_ptr(self):
        return A

    def __getattr__(self, name):
        return getattr(self._t, name)


def cache(index):
    c = bd.QuantCache.empty(2, 2, 20, 64, device="cpu")
    return bd.QuantCache(*(Placed(t, index) for t in (c.k_codes, c.k_scales, c.v_codes, c.v_scales)))


def test_a_tensor_on_another_gpu_is_refused(lib):  # noqa: F811
    c = cache(1)
    s = c.shape(4, 10)
    ws = types.SimpleNamespace(ptr=A, nbytes=1 << 30)
    at = {i: {name: Placed(t, i) for name, t in dict(
        rows=torch.zeros(2, 2, 3, 64, dtype=torch.bfloat16), q=torch.zeros(2, 4, 3, 64, dtype=torch.bfloat16),
        lse=torch.zeros(2, 4, 3), q1=torch.zeros(2, 4, 64, dtype=torch.bfloat16), lse1=torch.zeros(2, 4),
        idx=torch.zeros(2, 2, 8, dtype=torch.int32), count=torch.zeros(2, 2, dtype=torch.int32)).items()} for i in (0, 1)}

    def pick(odd, *names):
        return [at[0 if name == odd else 1][name] for name in names]

    for odd in (0, 1):
        rows = [at[0 if i == odd else 1]["rows"] for i in (0, 1)]
        with pytest.raises(ValueError, match="GPU"):
            bd.bd_quant_write(s, *rows, c)
        with pytest.raises(ValueError, match="GPU"):
            bd.bd_quant_read(s, c, *rows, first_row=0)
    for odd in ("q", "lse"):
        q, lse = pick(odd, "q", "lse")
        with pytest.raises(ValueError, match="GPU"):
            bd.bd_quant_verify_attn(s, q, 3, c, at[1]["q"], lse, ws)
    with pytest.raises(ValueError, match="GPU"):
        bd.bd_quant_verify_attn(s, at[1]["q"], 3, c, at[0]["q"], None, ws)
    for odd in ("q1", "lse1", "idx", "count"):
        q, lse, idx, count = pick(odd, "q1", "lse1", "idx", "count")
        with pytest.raises(ValueError, match="GPU"):
            bd.bd_quant_draft_attn(s, q, c, idx, count, 8, 0, at[1]["q1"], lse, ws)


def test_a_cache_on_two_gpus_is_refused():
    c = cache(0)
    with pytest.raises(ValueError):
        bd.QuantCache(c.k_codes, c.k_scales, Placed(c.v_codes._t, 1), c.v_scales)


@pytest.mark.gpu
def test_tensors_of_the_cache_s_gpu_are_taken():
    c = bd.QuantCache.empty(1, 1, 8, 64)
    rows = torch.zeros(1, 1, 8, 64, dtype=torch.bfloat16, device="cuda:0")
    bd.bd_quant_write(c.shape(1, 0), rows, rows, c)
    bd.bd_quant_read(c.shape(1, 8), c, rows, rows, first_row=0)
    torch.cuda.synchronize()
