"""Coefficients are refused where singular values may grow beyond 1024, as stated, and for nothing else: on the host, by the workspace's question."""
import ctypes as C

import pytest

from paper_2605_29346_amd import zg


def _status(triples):
    k = (C.c_float * (3 * len(triples)))(*(v for t in triples for v in t))
    a = zg.OrthogonalizeArgs(rows=4, cols=8, dtype=zg.F32, out_dtype=zg.F32, steps=len(triples), eps=1e-7, coefficients=C.addressof(k), d_G=1 << 24, ld_G=8, d_O=2 << 24, ld_O=8)
    return zg.lib().zg_orthogonalize_workspace(C.byref(a), C.byref(C.c_size_t()))


@pytest.mark.parametrize("triples", [[(1000.0, 0.0, 0.0)], [(1e-7, 0.0, 0.0), (1e7, -5e20, 0.0)], [(1e-20, 0.0, 0.0), (1e20, 0.0, 0.0)], [(0.0, 0.0, 0.0), (3e38, 3e38, 3e38)], [(1e-4, 0.0, 0.0), (1e6, 1e14, -2e22)]], ids=str)
def test_what_stays_below_is_taken(triples):
    assert _status(triples) == zg.OK, zg.lib().zg_last_error()


@pytest.mark.parametrize("triples", [[(1025.0, 0.0, 0.0)], [(1e-7, 0.0, 0.0), (1.1e10, 0.0, 0.0)], [(1.0, -1200.0, 2400.0)], [(32.0, 0.0, 0.0), (0.0, 0.1, 0.0)], [(1e-4, 0.0, 0.0), (1e6, 1e17, 0.0)]], ids=str)
def test_what_may_not_is_refused(triples):
    assert _status(triples) == zg.EINVAL
    assert b"1024" in zg.lib().zg_last_error()
