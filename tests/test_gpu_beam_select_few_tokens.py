"""Constrained steps: all tokens but a few masked, so that the places behind them are filled by equal entries, with many continuations asked for."""
import math

import pytest
import torch

import teach_ref as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("b,w,vocab", [(1, 4, 50021), (1, 16, 128000), (8, 8, 50021), (40, 8, 9001)])
@pytest.mark.parametrize("value", [-math.inf, "lowest", -3.0])
def test_equal_entries_behind_a_few(b, w, vocab, dtype, value):
    from paper_2607_03011_gb300 import inner
    g = torch.Generator().manual_seed(b * w + vocab)
    z = torch.full((b, w, vocab), ref.LOWEST[dtype] if value == "lowest" else value, dtype=dtype)
    allowed = torch.randint(0, vocab, (b, w, 5), generator=g)
    z.scatter_(2, allowed, torch.randn(b, w, 5, generator=g).to(dtype))
    scores = torch.randn(b, w, generator=g)
    want = ref.select(z[:2], scores[:2], 32)
    got = inner.beam_select(z.cuda(), scores.cuda(), keep=32)
    assert torch.equal(got.beams.cpu()[:2], want[1]) and torch.equal(got.tokens.cpu()[:2], want[2])
    fine = torch.isfinite(want[0])
    # the score, a difference of logits below 32 and a logarithm of a sum: a dozen roundings of numbers below 64
    assert ((got.scores.cpu()[:2].double() - want[0])[fine].abs() < 12 * 64 * 2.0 ** -24).all()
    assert torch.equal(torch.isfinite(got.scores.cpu()[:2]), fine)
