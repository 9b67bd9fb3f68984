"""beam_select's outputs may lie over its inputs only where every batch entry writes what it alone has read (no GPU needed: the
calls are refused before any device work)."""
import ctypes

import pytest

A = 1 << 20   # an address that is never read


@pytest.fixture(scope="module")
def iso():
    from paper_2607_03011_gb300 import isoloco
    isoloco.lib()
    return isoloco


def call(iso, b=2, w=4, keep=4, s=A, f=A + 4096, o=A + 8192, ob=A + 16384, ot=A + 32768, of=A + 65536, z=1 << 30):
    p = [None if v is None else ctypes.c_void_p(v) for v in (z, s, f, o, ob, ot, of)]
    return iso.lib().isoloco_beam_select(p[0], 8, 0, b, w, 8, p[1], p[2], 3, 1.0, keep, p[3], p[4], p[5], p[6], None)


@pytest.mark.parametrize("kw", [
    dict(o=A, keep=5), dict(o=A, keep=3), dict(o=A + 4), dict(o=A - 4), dict(o=A + 28), dict(of=A + 4096, keep=3), dict(of=A + 4095),
    dict(of=A + 4096 + 7), dict(ob=A), dict(ot=A + 24), dict(ob=A - 56), dict(o=A + 4096), dict(of=A), dict(of=A + 31), dict(ob=A + 4096 - 56),
    dict(ot=A + 16384), dict(ot=A + 16384 + 56), dict(o=A + 16384 + 60), dict(of=A + 8192), dict(of=A + 32768 + 63), dict(o=A + 32768)])
def test_refused(iso, kw):
    assert call(iso, **kw) == iso.ERR_INVALID
    assert "share" in iso.last_error()


def test_no_batch_entry_shares_nothing(iso):
    """(Not refused; without a GPU such a call fails later, for want of a device.)"""
    assert call(iso, b=0, o=A, of=A) != iso.ERR_INVALID
