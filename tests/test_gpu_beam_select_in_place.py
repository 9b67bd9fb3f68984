"""A selection whose scores and finished marks take their inputs' places, through the C entry point: the same answers as elsewhere."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("b,w,vocab", [(1, 4, 32000), (300, 5, 1003), (64, 16, 5000), (3, 32, 70001), (700, 32, 64), (2000, 1, 77)])
def test_in_place(b, w, vocab):
    from paper_2607_03011_gb300 import inner, isoloco
    g = torch.Generator(device="cuda").manual_seed(b + w)
    z = torch.randn(b, w, vocab, generator=g, device="cuda").bfloat16()
    scores = torch.randn(b, w, generator=g, device="cuda")
    finished = torch.rand(b, w, generator=g, device="cuda") < 0.3
    want = inner.beam_select(z, scores, finished=finished, end=7)
    beams, tokens = torch.empty(b, w, dtype=torch.int64, device="cuda"), torch.empty(b, w, dtype=torch.int64, device="cuda")
    rc = isoloco.lib().isoloco_beam_select(z.data_ptr(), vocab, 1, b, w, vocab, scores.data_ptr(), finished.data_ptr(), 7, 1.0, w, scores.data_ptr(),
                                           beams.data_ptr(), tokens.data_ptr(), finished.data_ptr(), torch.cuda.current_stream().cuda_stream)
    assert rc == 0, isoloco.last_error()
    assert all(torch.equal(x, y) for x, y in zip(want, (scores, beams, tokens, finished)))
