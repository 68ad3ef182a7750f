"""Calls of e2s_serve.h that are refused on the host because an output would overwrite what
the call still reads, or another output, and calls that are not refused (the fake device
addresses are never dereferenced)."""
import pytest

from paper_2608_23253_amd import _lib as L
from test_serve_abi import A, append, attend, rotate


@pytest.mark.parametrize("kw", [dict(), dict(weights=1, wout=4 * A), dict(num_queries=40),
                                dict(num_queries=40, weights=1, wout=4 * A)])
def test_attend_not_in_place(kw):
    assert attend(q=2 * A, out=2 * A, **kw) == L.ERR_BAD_PARAM


@pytest.mark.parametrize("kw", [dict(qo=6 * A, ko=6 * A), dict(qo=4 * A, ko=6 * A),
                                dict(qo=6 * A, ko=2 * A), dict(q=A, k=A, qo=A, ko=6 * A)])
def test_rotate_keeps_queries_and_keys_apart(kw):
    assert rotate(**dict(dict(q=2 * A, k=4 * A), **kw)) == L.ERR_BAD_PARAM


def test_a_stride_that_nothing_takes_may_be_anything():
    """One sequence, or one token: its stride (of any value, as torch makes them) moves nothing.
    The calls stop at the missing page table."""
    for kw in (dict(batch=1, q_stride=(1, 128, 64)), dict(batch=1, out_stride=(3, 128, 64)),
               dict(num_queries=1, q_stride=(512, 128, 1), out_stride=(512, 128, 5))):
        assert attend(pages=None, **kw) == L.ERR_NULL_POINTER, kw
    for kw in (dict(batch=1, k_stride=(1, 320, 64)), dict(batch=1, v_stride=(7, 320, 64)),
               dict(num_tokens=1, src_tokens=1, k_stride=(640, 320, 1))):
        assert append(pages=None, **kw) == L.ERR_NULL_POINTER, kw
    assert attend(pages=None, q_stride=(512, 128, 1)) == L.ERR_MISALIGNED
    assert append(pages=None, v_stride=(7, 320, 64)) == L.ERR_MISALIGNED
