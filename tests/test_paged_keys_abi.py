"""bd_paged_keys refuses bad arguments before any launch (no GPU)."""

import ctypes

import pytest

import paper_2606_00144_gb300 as bd
from paper_2606_00144_gb300 import binding
from tests.test_paged_abi import A, BD_OK, INVALID, MISALIGNED, UNSUPPORTED, bf, cache, f32, i32, lib, setting, shape, strides  # noqa: F401


def keys(lib, s, n=6, c=None, table=A, pages=7, k=A, ks=None):  # noqa: F811
    return lib.bd_paged_keys(ctypes.byref(s) if s is not None else None, n, c or cache(), table, pages, k, ks, None)


def test_validation(lib):  # noqa: F811
    assert keys(lib, None) == INVALID
    assert keys(lib, shape(), n=-1) == INVALID
    assert keys(lib, shape(), n=113) == INVALID                       # past t_cap
    assert keys(lib, shape(), n=2**31 - 1) == INVALID
    assert keys(lib, shape(), n=0, k=None) == BD_OK
    assert keys(lib, shape(), k=None) == INVALID
    assert keys(lib, shape(), k=A + 8) == MISALIGNED
    assert keys(lib, shape(), ks=strides(1536, 768, 0)) == INVALID
    assert keys(lib, shape(), ks=strides(1536, 768, 132)) == MISALIGNED
    assert keys(lib, shape(head_dim=96)) == UNSUPPORTED
    assert keys(lib, shape(), c=cache(k=None)) == INVALID
    assert keys(lib, shape(), c=cache(k_strides=strides(4100, 2048, 128))) == MISALIGNED
    assert keys(lib, shape(), c=cache(page_size=8)) == UNSUPPORTED
    assert keys(lib, shape(), table=None) == INVALID
    assert keys(lib, shape(), pages=6) == INVALID
    # V is not looked at (the keys' address keeps the call from launching)
    assert keys(lib, shape(), c=cache(v=None, v_strides=strides(1, 1, 1)), k=A + 8) == MISALIGNED


def test_the_selections_flag(lib):  # noqa: F811
    def select(flags):           # (the workspace's address keeps a call with good flags from launching)
        return lib.bd_select_budget(ctypes.byref(shape()), A, A, None, 8, 64, 4, 16, 1, flags, A, A, A + 16, 1 << 30, None)

    ready, hidden = bd.BD_SELECT_WINDOW_READY, bd.BD_SELECT_NAN_HIDDEN
    assert [select(f) for f in (0, ready, hidden, ready | hidden)] == [MISALIGNED] * 4
    assert [select(f) for f in (2, 8, 2 | hidden)] == [INVALID] * 3


def test_the_binding(lib, monkeypatch):  # noqa: F811
    c, s, table = setting()
    for rows, err in [(bf(2, 4, 3, 64), ValueError), (bf(2, 3, 64), ValueError), (f32(2, 2, 3, 64), TypeError),
                      (bf(2, 2, 3, 64, index=1), ValueError)]:
        with pytest.raises(err):
            bd.bd_paged_keys(s, c, table, rows)
    with pytest.raises(ValueError):
        bd.bd_paged_keys(s, c, i32(3, 2), bf(2, 2, 3, 64))
    calls = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: calls.append((name, a)) or 0

    monkeypatch.setattr(binding, "_lib", Library())
    monkeypatch.setattr(binding, "_device", lambda: 0)
    monkeypatch.setattr(binding, "_raw_stream", lambda gpu: 100 + gpu)
    bd.bd_paged_keys(s, c, table, bf(2, 2, 3, 64))
    assert calls[0][0] == "bd_paged_keys" and calls[0][1][1] == 3 and calls[0][1][-1] == 100
