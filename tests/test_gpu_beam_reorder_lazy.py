"""States that are conjugated or negated lazily: torch keeps a bit, and the memory holds other values than the tensor has."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def made(seed, *shape):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.complex(torch.randn(shape, generator=g, device="cuda"), torch.randn(shape, generator=g, device="cuda"))


BEAMS = torch.tensor([[1, 1, 0], [2, 0, 2]])


def want(s):
    return torch.stack([s.resolve_conj().resolve_neg()[i, BEAMS[i].cuda()] for i in range(2)])


def test_into_another_tensor():
    from paper_2607_03011_gb300 import inner
    c = made(1, 2, 3, 40)
    beams = BEAMS.cuda()
    # a lazy state and a plain result, and the other way round: refused, nothing is written
    lazy = [(c.conj(), torch.zeros_like(c)), (c, torch.zeros_like(c).conj()),
            (c.conj().imag, torch.zeros_like(c).imag), (c.imag, torch.zeros_like(c).conj().imag)]
    for s, o in lazy:
        with pytest.raises(ValueError):
            inner.beam_reorder([made(2, 2, 3, 8), s], beams, out=[made(3, 2, 3, 8), o])
        assert (o == 0).all()
    # both alike: the bytes are the values
    for s, o in ((c, torch.zeros_like(c)), (c.conj(), torch.zeros_like(c).conj()), (c.conj().imag, torch.zeros_like(c).conj().imag)):
        assert inner.beam_reorder([s], beams, out=[o])[0] is o
        assert torch.equal(o.resolve_conj().resolve_neg(), want(s))


def test_in_place():
    from paper_2607_03011_gb300 import inner
    for view in (lambda t: t, lambda t: t.conj(), lambda t: t.conj().imag, lambda t: t.real):
        c = made(4, 2, 3, 40)
        expected = want(view(c))
        assert torch.equal(inner.beam_reorder([view(c)], BEAMS.cuda())[0].resolve_conj().resolve_neg(), expected)
