"""Misaligned per-row arrays are refused before any device work (no GPU needed): a kernel that read or wrote
them would fault."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def iso():
    from paper_2607_03011_gb300 import isoloco
    isoloco.lib()
    return isoloco


@pytest.fixture(scope="module")
def p():
    buf = (ctypes.c_double * 64)()
    q = ctypes.c_void_p((ctypes.addressof(buf) + 15) // 16 * 16)
    q.keep = buf
    return q


@pytest.mark.parametrize("by", [1, 2, 3])
@pytest.mark.parametrize("name", ["logp", "entropy", "lse", "gl", "ge"])
def test_token_logprobs(iso, p, name, by):
    a = dict.fromkeys(["logp", "entropy", "lse", "gl", "ge"])
    a[name] = ctypes.c_void_p(p.value + by)
    rc = iso.lib().isoloco_token_logprobs(p, 8, 0, 2, 8, p, 8, 1.0, a["logp"], a["entropy"], a["lse"], 0, None, None, a["gl"],
                                          a["ge"], p, 8, None)
    assert rc == iso.ERR_INVALID and iso.last_error()


@pytest.mark.parametrize("by", [1, 2, 3])
@pytest.mark.parametrize("name", ["lse", "entropy", "gl", "ge"])
def test_token_logprobs_grad(iso, p, name, by):
    a = dict.fromkeys(["lse", "entropy", "gl", "ge"], p)
    a[name] = ctypes.c_void_p(p.value + by)
    rc = iso.lib().isoloco_token_logprobs_grad(p, 8, 0, 2, 8, p, 8, 1.0, a["lse"], a["entropy"], a["gl"], a["ge"], p, 8, None)
    assert rc == iso.ERR_INVALID and iso.last_error()
