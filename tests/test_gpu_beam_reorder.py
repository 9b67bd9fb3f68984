"""What is kept for beams, moved along: the same values as indexing gives, in place and not."""
import pytest
import torch

import teach_ref as ref

pytestmark = pytest.mark.gpu


def parents(b, w, seed=0, idt=torch.int64):
    g = torch.Generator().manual_seed(seed + 10 * b + w)
    return torch.randint(0, w, (b, w), generator=g).to(idt)


def state(shape, dtype, seed=0):
    g = torch.Generator().manual_seed(seed + sum(shape))
    if dtype.is_floating_point:
        return torch.randn(shape, generator=g).to(dtype)
    return torch.randint(0, 2 if dtype == torch.bool else 100, shape, generator=g).to(dtype)


def both(states, beams, cut=lambda t: t):
    """In place and into other tensors; what lies outside the part that is moved stays as it is."""
    from paper_2607_03011_gb300 import inner
    b, w = beams.shape
    want = [ref.reorder(cut(s).reshape(b, w, *cut(s).shape[2 if s.dim() > 1 and s.shape[:2] == (b, w) else 1:]), beams) for s in states]
    src = [s.cuda() for s in states]
    out = [torch.full_like(s, 3) for s in src]
    res = inner.beam_reorder([cut(s) for s in src], beams.cuda(), out=[cut(o) for o in out])
    for s, o, r, v, t in zip(src, out, res, want, states):
        assert torch.equal(s.cpu(), t) and r.data_ptr() == cut(o).data_ptr()
        full = torch.full_like(t, 3)
        cut(full).copy_(v.reshape(cut(full).shape))
        assert torch.equal(o.cpu(), full)
    res = inner.beam_reorder([cut(s) for s in src], beams.cuda())
    for s, r, v, t in zip(src, res, want, states):
        full = t.clone()
        cut(full).copy_(v.reshape(cut(full).shape))
        assert torch.equal(s.cpu(), full)


@pytest.mark.parametrize("b,w", [(1, 1), (1, 4), (3, 5), (2, 8), (2, 16), (1, 17), (2, 32), (150, 3)])
@pytest.mark.parametrize("idt", [torch.int32, torch.int64])
def test_widths(b, w, idt):
    both([state((b * w, 3, 10, 16), torch.bfloat16), state((b, w, 37), torch.int64), state((b * w,), torch.float32)], parents(b, w, idt=idt))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16, torch.int64, torch.int32, torch.int16, torch.uint8, torch.bool,
                                   torch.float64, torch.float8_e4m3fn])
def test_types(dtype):
    if dtype == torch.float8_e4m3fn:
        s = [state((12, 5, 7), torch.uint8), state((12, 16, 16), torch.uint8)]
        b = parents(3, 4)
        from paper_2607_03011_gb300 import inner
        t = [v.cuda().view(dtype) for v in s]
        inner.beam_reorder(t, b.cuda())
        assert all(torch.equal(x.view(torch.uint8).cpu(), ref.reorder(v.view(3, 4, *v.shape[1:]), b).view(v.shape)) for x, v in zip(t, s))
    else:
        both([state((12, 5, 7), dtype), state((12, 1), dtype), state((12, 16, 16), dtype)], parents(3, 4))


@pytest.mark.parametrize("length", [0, 1, 3, 8, 20])
@pytest.mark.parametrize("d", [1, 3, 8, 64])
def test_used_part_of_a_cache(length, d):
    both([state((6, 4, 20, d), torch.bfloat16), state((6, 2, 20, d), torch.float32)], parents(2, 3, 1), lambda t: t[:, :, :length])
    both([state((6, 20, 2, d), torch.float16)], parents(2, 3, 2), lambda t: t[:, :length])
    both([state((6, 2, d, 20), torch.float16)], parents(2, 3, 3), lambda t: t[..., 20 - length:])
    both([state((2, 3, 20), torch.int64)], parents(2, 3, 4), lambda t: t[:, :, :length])


def test_large_pieces_many_states():
    both([state((8, 2, 300, 64), torch.bfloat16, i) for i in range(70)], parents(2, 4, 5))
    both([state((4, 1000003), torch.uint8)], parents(1, 4, 6))


def test_special_parents():
    for p in ([[0, 1, 2, 3]], [[0, 0, 0, 0]], [[3, 2, 1, 0]], [[1, 2, 3, 0]], [[-1, 4, 2 ** 40, 0]], [[3, 3, -2 ** 50, 1]]):
        both([state((4, 129), torch.float32), state((4, 33), torch.uint8)], torch.tensor(p))


def test_layers_of_one_tensor():
    """States that lie in between one another: layers inside each beam's memory."""
    from paper_2607_03011_gb300 import inner
    whole = state((6, 4, 2, 5, 8), torch.bfloat16)
    b = parents(2, 3, 7)
    t = whole.cuda()
    inner.beam_reorder([t[:, i, j] for i in range(4) for j in range(2)], b.cuda())
    assert torch.equal(t.cpu(), ref.reorder(whole.view(2, 3, 4, 2, 5, 8), b).view(whole.shape))
    t = whole.cuda()
    inner.beam_reorder([t[:, :, 0, :3], t[:, :, 1, 2:]], b.cuda())
    want = whole.clone()
    moved = ref.reorder(whole.view(2, 3, 4, 2, 5, 8), b).view(whole.shape)
    want[:, :, 0, :3], want[:, :, 1, 2:] = moved[:, :, 0, :3], moved[:, :, 1, 2:]
    assert torch.equal(t.cpu(), want)


def test_layouts():
    from paper_2607_03011_gb300 import inner
    b = parents(2, 3, 8)
    s = state((6, 4, 5, 8), torch.float32)
    t = s.cuda().transpose(2, 3).contiguous().transpose(2, 3)   # dense in another order: in place in any
    inner.beam_reorder([t], b.cuda())
    assert torch.equal(t.cpu(), ref.reorder(s.view(2, 3, 4, 5, 8), b).view(s.shape))
    one = state((1, 4, 6), torch.float32).expand(3, 4, 6)       # a source that repeats itself
    out = torch.zeros(3, 4, 6).cuda()
    inner.beam_reorder([one.cuda()[:1].expand(3, 4, 6)], torch.tensor([2, 0, 1]).cuda(), out=[out])
    assert torch.equal(out.cpu(), one)
    assert inner.beam_reorder([], b.cuda()) == []
    assert inner.beam_reorder([torch.zeros(0, 3, 4).cuda()], torch.zeros(0, 3, dtype=torch.int64).cuda())[0].shape == (0, 3, 4)


def test_refusals():
    from paper_2607_03011_gb300 import inner
    b = parents(2, 3).cuda()
    s = torch.zeros(6, 4, 5).cuda()
    for states, beams, out in [([s], b.float(), None), ([s], b.cpu(), None), ([s.cpu()], b, None), ([s], b, [s[:5]]), ([s], b, [s.half()]),
                               ([s], b, []), ([s[:5]], b, None), ([torch.zeros((), device="cuda")], b, None),
                               ([s], torch.zeros(2, 33, dtype=torch.int64).cuda(), None), ([s], b.t(), None),
                               ([s], b.view(1, 2, 3), None), ([torch.zeros(6, 4, 5, 6).cuda()[:, ::2, ::2, ::2]], b, None)]:
        with pytest.raises(ValueError):
            inner.beam_reorder(states, beams, out=out)
    for states, out in [([s, s], None), ([s[:, :3], s[:, 2:]], None), ([s], [torch.zeros(1, 4, 5).cuda().expand(6, 4, 5)]),
                        ([s[:, :2]], [s[:, 1:3]]), ([s, torch.ones_like(s)], [s, s]), ([torch.zeros(1, 4).cuda().expand(6, 4)], None)]:
        before = s.clone()
        with pytest.raises(inner.IsolocoError):
            inner.beam_reorder(states, b, out=out)
        assert torch.equal(s, before)
