"""Where clusters of 16 CTAs do not fit (faked on the host), smaller ones find the same continuations."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("b,w,vocab,keep", [(1, 16, 128000, 16), (2, 13, 5003, 26), (3, 4, 70001, 8), (40, 32, 1000, 32), (16, 8, 50021, 16)])
def test_smaller_clusters(b, w, vocab, keep):
    from paper_2607_03011_gb300 import inner, isoloco
    g = torch.Generator(device="cuda").manual_seed(vocab)
    z = torch.randn(b, w, vocab, generator=g, device="cuda").half()
    scores = torch.randn(b, w, generator=g, device="cuda")
    want = inner.beam_select(z, scores, keep=keep, end=3)
    L = isoloco.lib()
    assert L.isoloco_debug_refuse_clusters(1) == isoloco.OK
    try:
        got = inner.beam_select(z, scores, keep=keep, end=3)
        torch.cuda.synchronize()
    finally:
        assert L.isoloco_debug_refuse_clusters(0) == isoloco.OK
    assert all(torch.equal(a, c) for a, c in zip(want, got))
