"""The inner step's C entry points refuse bad arguments before any device work (no GPU needed)."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def iso():
    from paper_2607_03011_gb300 import isoloco
    isoloco.lib()
    return isoloco


@pytest.fixture(scope="module")
def ptr():
    buf = (ctypes.c_double * 64)()
    base = ctypes.addressof(buf)
    p = ctypes.c_void_p((base + 15) // 16 * 16)
    p.keep = buf
    return p


def odd(p, by=1):
    return ctypes.c_void_p(p.value + by)


BIG = 1 << 50


def test_embed(iso, ptr):
    L, bad, p = iso.lib(), iso.ERR_INVALID, ptr

    def call(w=p, ldw=8, dt=0, vocab=4, width=8, ids=p, ib=8, n=2, y=p, ldy=8):
        return L.isoloco_embed(w, ldw, dt, vocab, width, ids, ib, n, 1.0, y, ldy, None)

    for kw in (dict(w=None), dict(ldw=7), dict(dt=3), dict(dt=-1), dict(vocab=0), dict(width=0), dict(vocab=1 << 31), dict(width=(1 << 20) + 1, ldw=1 << 21, ldy=1 << 21), dict(ids=None),
               dict(ids=odd(p, 4)), dict(ib=2), dict(n=-1), dict(n=1 << 31), dict(y=None), dict(ldy=7), dict(w=odd(p, 2)), dict(y=odd(p))):
        assert call(**kw) == bad, kw
        assert iso.last_error()


def test_embed_grad(iso, ptr):
    L, bad, p = iso.lib(), iso.ERR_INVALID, ptr

    def call(dy=p, ldy=8, dt=1, vocab=4, width=8, ids=p, ib=8, n=2, dw=p, ldw=8, dwt=1, ws=p, wsb=BIG):
        return L.isoloco_embed_grad(dy, ldy, dt, vocab, width, ids, ib, n, 1.0, dw, ldw, dwt, ws, wsb, None)

    for kw in (dict(dy=None), dict(ldy=7), dict(dwt=2), dict(dt=5), dict(dw=None), dict(ldw=7), dict(ws=None), dict(wsb=0),
               dict(wsb=L.isoloco_embed_grad_workspace(4, 8, 2) - 1)):
        assert call(**kw) == bad, kw
    assert call(ws=odd(p, 8)) == iso.ERR_ALIGN
    assert L.isoloco_embed_grad_workspace(0, 1, 1) == bad and L.isoloco_embed_grad_workspace(1, 1, -1) == bad
    assert L.isoloco_embed_grad_workspace(10, 8, 0) > 0


def test_gated_ffn(iso, ptr):
    L, bad, p = iso.lib(), iso.ERR_INVALID, ptr

    def call(x=p, ldx=8, wg=p, wu=p, ldw=16, dt=1, n=2, d=8, f=16, act=0, h=p, ldh=16, saved=None, ws=p, wsb=BIG):
        return L.isoloco_gated_ffn(x, ldx, wg, wu, ldw, dt, n, d, f, act, h, ldh, saved, ws, wsb, None)

    for kw in (dict(x=None), dict(ldx=7), dict(wg=None), dict(wu=None), dict(ldw=15), dict(dt=0), dict(dt=3), dict(act=2), dict(act=-1),
               dict(n=-1), dict(d=0), dict(f=0), dict(f=(1 << 20) + 1), dict(h=None), dict(ldh=15),
               dict(ldw=17, ws=None), dict(ldh=17, wsb=0), dict(x=odd(p)), dict(wu=odd(p))):
        assert call(**kw) == bad, kw
    assert call(saved=odd(p, 8)) == iso.ERR_ALIGN and call(ldx=9, ws=odd(p, 8)) == iso.ERR_ALIGN


def test_gated_ffn_grad(iso, ptr):
    L, bad, p = iso.lib(), iso.ERR_INVALID, ptr

    def call(dh=p, ldh=16, x=p, ldx=8, wg=p, wu=p, ldw=16, dt=1, n=2, d=8, f=16, act=0, saved=p, dx=p, lddx=8, dwg=p, dwu=p, lddw=16,
             ws=p, wsb=BIG):
        return L.isoloco_gated_ffn_grad(dh, ldh, x, ldx, wg, wu, ldw, dt, n, d, f, act, saved, dx, lddx, dwg, dwu, lddw, ws, wsb, None)

    for kw in (dict(dh=None), dict(ldh=15), dict(saved=None), dict(lddx=7), dict(dwg=None), dict(dwu=None), dict(lddw=15), dict(wsb=16),
               dict(x=None), dict(dt=0)):
        assert call(**kw) == bad, kw
    assert call(saved=odd(p, 8)) == iso.ERR_ALIGN


def test_token_logprobs(iso, ptr):
    L, bad, p = iso.lib(), iso.ERR_INVALID, ptr

    def call(z=p, ld=8, dt=0, n=2, v=8, t=p, tb=8, scale=1.0, top=0, tl=None, ti=None, gz=None, ldg=8):
        return L.isoloco_token_logprobs(z, ld, dt, n, v, t, tb, scale, None, None, None, top, tl, ti, None, None, gz, ldg, None)

    for kw in (dict(z=None), dict(ld=7), dict(dt=9), dict(n=-1), dict(v=0), dict(t=None), dict(tb=1), dict(scale=0.0), dict(scale=-1.0),
               dict(scale=float("nan")), dict(scale=float("inf")), dict(top=9, tl=p, ti=p), dict(top=33, v=64, ld=64, tl=p, ti=p),
               dict(top=-1), dict(top=2, tl=p), dict(top=2, ti=p), dict(gz=p, ldg=7), dict(z=odd(p))):
        assert call(**kw) == bad, kw

    def grad(lse=p, ent=p, ge=p, gz=p, ldg=8):
        return L.isoloco_token_logprobs_grad(p, 8, 0, 2, 8, p, 8, 1.0, lse, ent, None, ge, gz, ldg, None)

    for kw in (dict(lse=None), dict(ent=None), dict(gz=None), dict(ldg=7)):
        assert grad(**kw) == bad, kw


def test_clip_grads(iso, ptr):
    L, bad, p = iso.lib(), iso.ERR_INVALID, ptr

    def arr(*entries):
        a = (iso.Tensor * len(entries))()
        for e, (d, n, t) in zip(a, entries):
            e.data, e.n, e.dtype = d, n, t
        return a

    good = arr((p.value, 4, 0))
    for a in (arr((None, 4, 0)), arr((p.value, -1, 0)), arr((p.value, 4, 3)), arr((p.value + 1, 4, 0)), arr((p.value, (1 << 33) + 1, 0))):
        assert L.isoloco_grad_norm(a, 1, p, p, BIG, None) == bad
        assert L.isoloco_clip_grads(a, None, 1, 1.0, p, p, BIG, None) == bad
        assert L.isoloco_clip_grads(good, a, 1, 1.0, p, p, BIG, None) == bad
    assert L.isoloco_grad_norm(None, 1, p, p, BIG, None) == bad and L.isoloco_grad_norm(good, -1, p, p, BIG, None) == bad
    assert L.isoloco_grad_norm(good, 1, None, p, BIG, None) == bad
    large = arr((p.value, 1 << 24, 0))  # (a small gradient needs no workspace)
    assert L.isoloco_grad_norm_workspace(good, 1) == 0 and L.isoloco_grad_norm_workspace(large, 1) > 8
    assert L.isoloco_grad_norm(large, 1, p, p, 8, None) == bad and L.isoloco_grad_norm(large, 1, p, None, BIG, None) == bad
    assert L.isoloco_grad_norm(large, 1, p, odd(p, 8), BIG, None) == iso.ERR_ALIGN
    for outs in (arr((p.value, 5, 0)), arr((p.value, 4, 1))):
        assert L.isoloco_clip_grads(good, outs, 1, 1.0, p, p, BIG, None) == bad
    for m in (0.0, -1.0, float("nan")):
        assert L.isoloco_clip_grads(good, None, 1, m, p, p, BIG, None) == bad


def test_tensor_layout_matches_the_header(tmp_path, iso):
    import os
    import shutil
    import subprocess
    from conftest import ROOT
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    src = tmp_path / "t.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "isoloco.h"\nint main(void) { printf("%zu %zu %zu %zu %d\\n", '
                   'sizeof(isoloco_tensor_t), offsetof(isoloco_tensor_t, data), offsetof(isoloco_tensor_t, n), '
                   'offsetof(isoloco_tensor_t, dtype), ISOLOCO_MAX_TOP); return 0; }\n')
    subprocess.run([gcc, "-std=c11", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "t")], check=True)
    out = [int(v) for v in subprocess.run([str(tmp_path / "t")], capture_output=True, text=True, check=True).stdout.split()]
    from paper_2607_03011_gb300 import inner
    assert out == [ctypes.sizeof(iso.Tensor), iso.Tensor.data.offset, iso.Tensor.n.offset, iso.Tensor.dtype.offset, inner.MAX_TOP]
