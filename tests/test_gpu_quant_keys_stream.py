"""QuantSpecStep's buffer of keys on a stream of the caller's: made of memory that other streams' queued work is done with,
and given back only when every stream that used it is."""

import pytest
import torch

import paper_2606_00144_gb300 as bd

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
B, H_KV, D, T = 2, 4, 128, 4096


def make(seed):
    g = torch.Generator("cuda").manual_seed(seed)
    k = torch.randn(B, H_KV, T, D, generator=g, device="cuda").to(BF)
    cache = bd.QuantCache.empty(B, H_KV, T + 6, D)
    bd.bd_quant_write(cache.shape(H_KV, 0), k, k, cache)
    want = torch.empty_like(k)
    bd.bd_quant_read(cache.shape(H_KV, T), cache, want, first_row=0)
    st = bd.QuantSpecStep(B, H_KV, H_KV, D, T, T + 6, 256, 4, 64, window=16)
    torch.cuda.synchronize()
    return cache, want, st


@pytest.mark.parametrize("handle", [False, True])
def test_the_buffer_is_not_one_that_queued_work_still_writes(handle):
    cache, want, st = make(1)
    side = torch.cuda.Stream()
    # a buffer of the same size, given back while what writes it has yet to run
    other = torch.empty(B, H_KV, T + 6, D, dtype=BF, device="cuda")
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)
    other.fill_(3.0)
    del other
    keys = st.keys(cache, side.cuda_stream if handle else side)
    side.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(keys[:, :, :T], want)


def test_the_buffer_is_not_given_away_while_another_stream_uses_it():
    cache, want, st = make(2)
    shape = (B, H_KV, T + 6, D)
    st.keys(cache)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)
        keys = st.keys(cache, side)
        got = keys[:, :, :T].clone()
    del keys, st
    torch.empty(shape, dtype=BF, device="cuda").fill_(5.0)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
