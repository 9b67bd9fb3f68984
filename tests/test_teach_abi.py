"""Distillation's and the beams' C entry points refuse bad arguments before any device work (no GPU needed)."""
import ctypes
import itertools

import pytest


@pytest.fixture(scope="module")
def iso():
    from paper_2607_03011_gb300 import isoloco
    isoloco.lib()
    return isoloco


@pytest.fixture(scope="module")
def ptr():
    buf = (ctypes.c_double * 64)()
    p = ctypes.c_void_p((ctypes.addressof(buf) + 15) // 16 * 16)
    p.keep = buf
    return p


def odd(p, by=1):
    return ctypes.c_void_p(p.value + by)


NAN, INF = float("nan"), float("inf")


def test_distill(iso, ptr):
    L, bad, p = iso.lib(), iso.ERR_INVALID, ptr

    def call(z=p, ld=8, dt=0, n=2, vocab=8, v=p, ldv=4, vt=0, i=p, ldi=4, ib=8, k=4, scale=1.0, tail=0, loss=p, saved=None, g=None, gz=None, ldg=8):
        return L.isoloco_distill(z, ld, dt, n, vocab, v, ldv, vt, i, ldi, ib, k, scale, tail, loss, saved, g, gz, ldg, None)

    def grad(g=p, z=p, ld=8, dt=0, n=2, vocab=8, v=p, ldv=4, vt=0, i=p, ldi=4, ib=8, k=4, scale=1.0, tail=0, saved=p, gz=p, ldg=8):
        return L.isoloco_distill_grad(g, z, ld, dt, n, vocab, v, ldv, vt, i, ldi, ib, k, scale, tail, saved, gz, ldg, None)

    shared = [dict(z=None), dict(z=odd(p, 2)), dict(ld=7), dict(dt=3), dict(dt=-1), dict(n=-1), dict(n=1 << 31), dict(vocab=0),
              dict(vocab=1 << 31, ld=1 << 32), dict(v=None), dict(v=odd(p)), dict(ldv=3), dict(vt=3), dict(i=None), dict(i=odd(p, 4)), dict(ldi=3), dict(ib=2),
              dict(k=0), dict(k=-1), dict(k=257, ldv=300, ldi=300), dict(scale=0.0), dict(scale=-1.0), dict(scale=NAN), dict(scale=INF),
              dict(tail=2), dict(tail=-1), dict(saved=odd(p, 2)), dict(gz=p, g=p, ldg=7), dict(z=p, gz=p, g=p, ldg=9), dict(gz=odd(p, 2), g=p), dict(gz=p, g=None), dict(gz=p, g=odd(p))]
    for kw in shared + [dict(loss=None), dict(loss=odd(p))]:
        assert call(**kw) == bad, kw
        assert iso.last_error()
    for kw in shared + [dict(gz=None), dict(saved=None)]:
        assert grad(**kw) == bad, kw


def test_beam_select(iso, ptr):
    L, bad, p = iso.lib(), iso.ERR_INVALID, ptr

    def call(z=p, ld=8, dt=0, b=2, w=3, vocab=8, s=p, f=None, end=-1, scale=1.0, keep=3, o=p, ob=p, ot=p, of=None):
        return L.isoloco_beam_select(z, ld, dt, b, w, vocab, s, f, end, scale, keep, o, ob, ot, of, None)

    for kw in (dict(z=None), dict(z=odd(p)), dict(ld=7), dict(dt=3), dict(b=-1), dict(b=1 << 31), dict(b=1 << 62), dict(w=0), dict(w=33), dict(vocab=0), dict(s=None),
               dict(s=odd(p, 2)), dict(f=p), dict(end=8), dict(scale=0.0), dict(scale=NAN), dict(keep=0), dict(keep=33, vocab=64, ld=64), dict(keep=25), dict(o=None),
               dict(o=odd(p)), dict(ob=None), dict(ob=odd(p, 4)), dict(ot=None), dict(ot=odd(p, 4))):
        assert call(**kw) == bad, kw
        assert iso.last_error()


def states(iso, *entries):
    a = (iso.State * max(1, len(entries)))()
    for e, (src, dst, sb, sw, so, db, dw, do, n, run) in zip(a, entries):
        e.src, e.dst, e.src_batch, e.src_beam, e.src_outer, e.dst_batch, e.dst_beam, e.dst_outer, e.outer, e.run = src, dst, sb, sw, so, db, dw, do, n, run
    return a


A, B = 1 << 20, 1 << 24   # addresses that are never read: every call here is refused, or has nothing to do


def test_beam_reorder(iso, ptr):
    L, bad, p = iso.lib(), iso.ERR_INVALID, ptr

    def call(*e, batch=2, width=3, ids=p, ib=8, count=None):
        return L.isoloco_beam_reorder(states(iso, *e), len(e) if count is None else count, batch, width, ids, ib, None)

    good = (A, B, 300, 100, 25, 300, 100, 25, 4, 25)
    for kw in (dict(width=0), dict(width=33), dict(batch=-1), dict(batch=1 << 31), dict(batch=1 << 61), dict(ids=None), dict(ids=odd(p, 4)), dict(ib=4, ids=odd(p, 2)),
               dict(ib=1), dict(count=-1)):
        assert call(good, **kw) == bad, kw
        assert iso.last_error()
    assert L.isoloco_beam_reorder(None, 1, 2, 3, p, 8, None) == bad
    for i in range(10):
        e = list(good)
        e[i] = None if i < 2 else -1
        assert call(tuple(e)) == bad, i
    assert call((A, B, 300, 1 << 47, 25, 300, 100, 25, 4, 25)) == bad
    assert call((A, B, 1 << 46, 100, 25, 300, 100, 25, 4, 25)) == bad
    # nothing to do
    assert call((None, None, 0, 0, 0, 0, 0, 0, 0, 25)) == 0 and call((None, None, 0, 0, 0, 0, 0, 0, 4, 0)) == 0 and call() == 0


def shared(iso, *e, batch=2, width=3):
    """Whether the call is refused for shared memory; without `beams`, so that it is refused in any case."""
    assert iso.lib().isoloco_beam_reorder(states(iso, *e), len(e), batch, width, None, 8, None) == iso.ERR_INVALID
    if "beams is NULL" in iso.last_error():
        return False
    assert "shares" in iso.last_error() or "overlaps" in iso.last_error()
    return True


def place(at, batch=300, beam=100, outer=25, n=4, run=25):
    return (at, at, batch, beam, outer, batch, beam, outer, n, run)


def move(src, dst, batch=300, beam=100, outer=25, n=4, run=25):
    return (src, dst, batch, beam, outer, batch, beam, outer, n, run)


def test_shared_memory_is_refused(iso):
    for e in ([place(A), place(A)], [place(A), place(A + 599)], [place(A), place(A + 24)], [move(A, A + 1)], [move(A, A + 300)], [move(A, A - 599)],
              [move(A, B), move(A + 5000, B)], [move(A, B), move(A + 5000, B + 599)], [move(A, B), move(B + 10, A + 10000)], [move(A, B), place(A)],
              [place(A, beam=0)], [place(A, batch=299)], [place(A, outer=24)], [place(A, batch=0)],
              [place(A, batch=600, beam=200), place(A + 124, batch=600, beam=200)],   # interleaved, one byte too near
              [place(A, batch=600, beam=200), place(A - 101 + 2, batch=600, beam=200)],
              [place(A, batch=1200, beam=400, outer=100, run=50), place(A + 49, batch=1200, beam=400, outer=100, run=50)],
              [place(A, batch=1200, beam=400, outer=100, run=50), place(A + 350 + 1 - 2, batch=1200, beam=400, outer=100, run=50)],
              [place(A, batch=600, beam=200), place(A + 150, batch=620, beam=200)]):   # strides that cannot be told apart
        assert shared(iso, *e), e


def oracle(a, b, batch, width):
    """Whether two states written in place share a byte, byte by byte."""
    def bytes_of(e):
        return {e[0] + i * e[2] + w * e[3] + o * e[4] + r for i in range(batch) for w in range(width) for o in range(e[8]) for r in range(e[9])}
    return bool(bytes_of(a) & bytes_of(b))


def test_no_overlap_is_missed(iso):
    """Over small layouts at all distances: whatever shares a byte is refused, and nested layouts that share none are not."""
    for (batch_s, beam_s, outer_s, n, run), at in itertools.product(
            [(96, 32, 8, 2, 4), (96, 32, 4, 2, 4), (16, 32, 8, 2, 4), (8, 32, 0, 1, 8), (2, 4, 12, 3, 2)], range(-100, 101)):
        a, b = place(A, batch_s, beam_s, outer_s, n, run), place(A + at, batch_s, beam_s, outer_s, n, run)
        if oracle(a, b, 2, 3):
            assert shared(iso, a, b), (a, b)
        elif (batch_s, beam_s) == (96, 32):
            assert not shared(iso, a, b), (a, b)


def test_beams_among_the_states(iso):
    L = iso.lib()
    for at in (A, A + 592, A - 40):
        assert L.isoloco_beam_reorder(states(iso, place(A)), 1, 2, 3, ctypes.c_void_p(at), 8, None) == iso.ERR_INVALID
        assert "beams" in iso.last_error() and "shares" in iso.last_error()


@pytest.mark.parametrize("e", [
    [place(A), place(A + 600)], [move(A, B)], [move(A, B), move(A, B + 600)], [move(A, A + 600)], [move(A, B, beam=100), place(A + 700)],
    [place(A, batch=600, beam=200), place(A + 100, batch=600, beam=200)],
    [place(A, batch=600, beam=200), place(A + 100, batch=600, beam=200, outer=50, n=2, run=50)],
    [(A, B, 0, 0, 25, 300, 100, 25, 4, 25)],                       # a source that repeats itself
    [place(A, batch=1200, beam=400, outer=100, run=50), place(A + 50, batch=1200, beam=400, outer=100, run=50)]])
def test_memory_apart_is_taken(iso, e):
    assert not shared(iso, *e)


def test_layout_matches_the_header(tmp_path, iso):
    import os
    import shutil
    import subprocess
    from conftest import ROOT
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    src = tmp_path / "t.c"
    names = [n for n, _ in iso.State._fields_]
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "isoloco.h"\nint main(void) { printf("%zu '
                   + "%zu " * len(names) + '%d %d %d\\n", sizeof(isoloco_state_t), '
                   + ", ".join(f"offsetof(isoloco_state_t, {n})" for n in names)
                   + ", ISOLOCO_MAX_LIST, ISOLOCO_MAX_BEAMS, ISOLOCO_TAIL_REST); return 0; }\n")
    subprocess.run([gcc, "-std=c11", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "t")], check=True)
    out = [int(v) for v in subprocess.run([str(tmp_path / "t")], capture_output=True, text=True, check=True).stdout.split()]
    from paper_2607_03011_gb300 import inner
    assert out == [ctypes.sizeof(iso.State)] + [getattr(iso.State, n).offset for n in names] + [inner.MAX_LIST, inner.MAX_BEAMS, inner._TAIL["rest"]]
