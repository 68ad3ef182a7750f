"""Calls of e2s_serve.h that are refused on the host because an output would overwrite what
the call still reads, or another output (the fake device addresses are never dereferenced)."""
import pytest

from paper_2608_23253_amd import _lib as L
from test_serve_abi import A, attend, rotate


@pytest.mark.parametrize("kw", [dict(), dict(weights=1, wout=4 * A), dict(num_queries=40),
                                dict(num_queries=40, weights=1, wout=4 * A)])
def test_attend_not_in_place(kw):
    assert attend(q=2 * A, out=2 * A, **kw) == L.ERR_BAD_PARAM


@pytest.mark.parametrize("kw", [dict(qo=6 * A, ko=6 * A), dict(qo=4 * A, ko=6 * A),
                                dict(qo=6 * A, ko=2 * A), dict(q=A, k=A, qo=A, ko=6 * A)])
def test_rotate_keeps_queries_and_keys_apart(kw):
    assert rotate(**dict(dict(q=2 * A, k=4 * A), **kw)) == L.ERR_BAD_PARAM
