"""bd_paged_append over its own source: a bf16 source may be its output, element for element; what would lie over rows that other
threads have still to read is refused before any launch (no GPU)."""

import pytest

from tests import test_paged_abi as abi
from tests.test_paged_abi import A, F32, INVALID, MISALIGNED, lib, strides  # noqa: F401

DENSE = (6144, 768, 128)          # 8 heads of 6 rows of 128
TOKENS = (6144, 128, 1024)        # the same memory, tokens outermost


@pytest.mark.parametrize("qs,os", [(None, None), (strides(*DENSE), None), (None, strides(*DENSE)), (strides(*TOKENS), strides(*TOKENS)),
                                   (strides(*TOKENS), strides(*DENSE))])
@pytest.mark.parametrize("packed", [False, True])
def test_fp32_queries_are_never_rotated_in_place(lib, qs, os, packed):  # noqa: F811
    """A bf16 row is half as many bytes: row r would lie over the source of row r / 2."""
    assert abi.append(lib, abi.shape(), dtype=F32, qs=qs, os=os, starts=A if packed else None) == INVALID


def test_bf16_queries_in_place_keep_their_strides(lib):  # noqa: F811
    for qs, os in [(None, TOKENS), (TOKENS, None), (DENSE, TOKENS), ((6144, 768, 256), DENSE), ((12288, 768, 128), DENSE)]:
        qs, os = (x and strides(*x) for x in (qs, os))
        assert abi.append(lib, abi.shape(), qs=qs, os=os) == INVALID
    # packed rows have no sequence stride; sizes of one have none either
    assert abi.append(lib, abi.shape(), qs=strides(0, 768, 256), os=strides(0, 768, 128), starts=A) == INVALID


def test_what_may_be_in_place_is_not_refused(lib):  # noqa: F811
    """(Keys at an address that is not aligned, which are looked at after the queries, keep the calls from launching.)"""
    for kw in [dict(), dict(qs=strides(*DENSE)), dict(os=strides(*DENSE)), dict(qs=strides(*TOKENS), os=strides(*TOKENS)),
               dict(starts=A, qs=strides(7, 768, 128)), dict(n=1, qs=strides(1024, 128, 3), os=strides(1024, 128, 128)),
               dict(dtype=F32, o=A + 0x100000), dict(o=A + 0x100000, os=strides(*TOKENS)), dict(q=None, o=None, dtype=F32)]:
        assert abi.append(lib, abi.shape(), k=A + 8, **kw) == MISALIGNED, kw
