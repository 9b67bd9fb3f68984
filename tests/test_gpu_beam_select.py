"""A beam search's selection against a full ranking in 64 bits."""
import math

import pytest
import torch

import teach_ref as ref

pytestmark = pytest.mark.gpu

INF = math.inf
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def make(b, w, vocab, dtype, seed=0):
    g = torch.Generator().manual_seed(seed * 1000 + b + w + vocab)
    z = torch.randn(b, w, vocab, generator=g) * 3
    return z.to(dtype), -torch.rand(b, w, generator=g) * 5


def check(z, scores, keep, finished=None, end=None, scale=1.0, apart=True):
    from paper_2607_03011_gb300 import inner
    total, beams, tokens = ref.select(z, scores, min(keep + 1, z.shape[1] * z.shape[2], 10 ** 6), finished, end, scale)
    sure = torch.ones(z.shape[0], dtype=torch.bool)
    if apart and total.shape[1] > 1:
        # totals of different beams that are nearer to each other than sums of powers are good to may come in either order
        gap, other = (total[:, :-1] - total[:, 1:]), beams[:, :-1] != beams[:, 1:]
        sure = ~(other & torch.isfinite(total[:, 1:]) & (gap < 8 * ref.sum_of_powers(z.shape[2]))).any(1)
        assert sure.double().mean() > 0.9
    total, beams, tokens = total[:, :keep], beams[:, :keep], tokens[:, :keep]
    r = inner.beam_select(z.cuda(), scores.cuda(), keep=keep, finished=None if finished is None else finished.cuda(), end=end, scale=scale)
    assert torch.equal(r.beams.cpu()[sure], beams[sure]), (r.beams.cpu() - beams)[sure].nonzero()[:5]
    assert torch.equal(r.tokens.cpu()[sure], tokens[sure]), (r.tokens.cpu() - tokens)[sure].nonzero()[:5]
    for i in torch.nonzero(~sure).flatten().tolist():
        chosen = z[i].double().log_softmax(1)[r.beams[i].cpu(), r.tokens[i].cpu()] if scale == 1.0 and finished is None else None
        assert chosen is not None and len(set(zip(r.beams[i].tolist(), r.tokens[i].tolist()))) == keep
        assert ((scores[i].double()[r.beams[i].cpu()] + chosen - total[i]).abs() < 8 * ref.sum_of_powers(z.shape[2])).all()
        beams[i], tokens[i] = r.beams[i].cpu(), r.tokens[i].cpu()
    got = r.scores.cpu().double()
    assert torch.equal(torch.isnan(got), torch.isnan(total)) and torch.equal(got == -INF, total == -INF)
    fine = torch.isfinite(total)
    # the sum's share, and the fp32 roundings of the total (and of scale in the exponents: inside the share)
    assert ((got - total).abs()[fine] <= 2 * ref.sum_of_powers(z.shape[2]) + 2.0 ** -24 * total.abs()[fine]).all()
    if end is None:
        assert r.finished is None
    else:
        was = torch.zeros_like(beams, dtype=torch.bool) if finished is None else finished.gather(1, beams)
        assert torch.equal(r.finished.cpu(), was | (tokens == end))
    return r


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("b,w,vocab,keep", [(1, 1, 1, 1), (1, 1, 9, 4), (2, 3, 5, 15), (1, 4, 1000, 4), (3, 5, 1001, 10), (2, 8, 4099, 16),
                                            (7, 2, 8192, 1), (1, 32, 2053, 32), (1, 4, 32000, 8), (2, 16, 12345, 16)])
def test_sizes(b, w, vocab, keep, dtype):
    check(*make(b, w, vocab, dtype), keep)


@pytest.mark.parametrize("dtype,b,w,vocab", [(F32, 1, 2, 128001), (BF16, 2, 3, 262144), (F16, 1, 1, 300007)])
def test_long_rows(dtype, b, w, vocab):
    check(*make(b, w, vocab, dtype), 7, scale=0.75)


@pytest.mark.parametrize("b", [1, 20, 160, 400])
def test_many_batch_entries(b):
    check(*make(b, 4, 700, BF16, seed=1), 8)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_ties_within_a_beam(dtype):
    g = torch.Generator().manual_seed(1)
    z = torch.randint(-1, 2, (2, 3, 3001), generator=g).float()
    z[0, 1] = 0.0           # all equal
    z[1, 2, 1::2] = -0.0    # both zeros
    check(z.to(dtype), torch.tensor([[0.0, -1.125, -2.25], [-0.5, -0.25, -3.0]]), 32)


@pytest.mark.parametrize("vocab", [1000, 1001, 40003])
@pytest.mark.parametrize("dtype", [F32, F16])
def test_equal_beams_rank_by_number(vocab, dtype):
    """Beams with equal logits and scores have equal totals, wherever their rows lie."""
    z, _ = make(2, 1, vocab, dtype, seed=2)
    r = check(z.repeat(1, 7, 1), torch.zeros(2, 7), 20, apart=False)
    assert r.beams[0].tolist() == [i % 7 for i in range(20)] or len(set(r.tokens[0].tolist())) < 3


def test_first_step_and_few_answers():
    z, _ = make(2, 4, 500, BF16, seed=3)
    scores = torch.tensor([[0.0, -INF, -INF, -INF]]).repeat(2, 1)
    check(z, scores, 8)
    z, _ = make(2, 4, 3, F32, seed=3)          # fewer finite ones than are asked for
    check(z, scores, 12)
    check(z, torch.full((2, 4), -INF), 12)     # none


def test_finished_beams():
    z, scores = make(3, 5, 400, F32, seed=4)
    fin = torch.tensor([[True, False, True, False, False], [True] * 5, [False] * 5])
    for end in (0, 3, 399):
        check(z, scores, 10, fin, end)
    z[:, 0] = math.nan                          # a finished beam's logits are not read
    z[2, 0] = 0.0
    check(z, scores, 10, fin, 7)
    check(*make(2, 3, 400, BF16, seed=5), 6, None, 2)   # an end without finished beams
    scores[0, 0] = -INF
    check(z, scores, 20, fin, 7)
    check(z[:, :1], scores[:, :1], 3, fin[:, :1], 0)
    check(z[:2, :1, :1], scores[:2, :1], 1, torch.tensor([[True], [True]]), 0)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_masks(dtype):
    z, scores = make(6, 3, 300, dtype, seed=6)
    low = ref.LOWEST[dtype]
    z[0, 1] = -INF
    z[1, 0] = low
    z[2, :, 2:] = -INF
    z[3, :, 1:] = low
    z[4] = -INF
    z[5, 0, ::2], z[5, 1, 1::2] = -INF, low
    check(z, scores, 12)


def test_nan_and_infinities():
    z, scores = make(8, 3, 300, F32, seed=7)
    z[0, 1, 17] = math.nan
    z[1, 0, 5] = INF
    z[2] = math.nan
    scores[3, 1] = math.nan
    scores[4, 2] = INF
    z[5, 0], z[5, 0, 9] = -INF, math.nan
    scores[6] = -INF
    z[6, 1, 3] = math.nan                       # (not read)
    z[7, 2, 299] = math.nan
    check(z, scores, 9)
    check(z[5:6, :1, :20], scores[5:6, :1], 20)


def test_special_rows_in_many_batch_entries():
    """Finished, dead and masked beams, NaN and ties, among so many rows that the merging is a launch of its own."""
    z, scores = make(8, 5, 120, F32, seed=9)
    fin = torch.zeros(8, 5, dtype=torch.bool)
    fin[0], fin[1, ::2], fin[7, 1] = True, True, True
    z[2, 1], z[3, 0, 5], z[4, 3, 7] = -INF, math.nan, INF
    z[5, :, 2:] = ref.LOWEST[F32]
    scores[6, 2:], scores[7, 0], scores[7, 4] = -INF, math.nan, INF
    z[6, 0] = 0.25
    check(z.repeat(30, 1, 1), scores.repeat(30, 1), 10, fin.repeat(30, 1), 3)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_shares_of_rows_in_many_batch_entries(dtype):
    check(*make(40, 8, 90001, dtype, seed=10), 6)


@pytest.mark.parametrize("b,w", [(1, 2), (3, 16), (2, 13), (60, 16), (70, 12), (1, 32), (40, 32), (5, 9)])
def test_deals_of_rows_to_ctas(b, w):
    check(*make(b, w, 5003, F16, seed=11), min(2 * w, 32))


def test_pitch_and_leading_dimensions():
    from paper_2607_03011_gb300 import inner
    z, scores = make(6, 4, 133, F16, seed=8)
    wide = torch.zeros(6, 4, 150, dtype=F16).cuda()
    wide[..., 3:136] = z.cuda()
    want = check(z, scores, 4)
    for part, s in ((wide[..., 3:136], scores.cuda()), (wide[..., 3:136].view(2, 3, 4, 133), scores.cuda().view(2, 3, 4))):
        r = inner.beam_select(part, s)
        assert r.tokens.shape == s.shape
        assert all(torch.equal(a.reshape(-1), b.reshape(-1)) for a, b in zip(r[:3], want[:3]))
    one = inner.beam_select(z.cuda()[0], scores.cuda()[0])
    assert one.scores.shape == (4,) and torch.equal(one.tokens, want.tokens[0])
    none = inner.beam_select(z.cuda()[:0], scores.cuda()[:0], end=1)
    assert none.scores.shape == (0, 4) and none.finished.shape == (0, 4)


def test_refusals():
    from paper_2607_03011_gb300 import inner
    z, s = (t.cuda() for t in make(2, 3, 50, BF16))
    f = torch.zeros(2, 3, dtype=torch.bool, device="cuda")
    for args, kw in [((z.double(), s), {}), ((z.cpu(), s), {}), ((z, s.cpu()), {}), ((z, s.half()), {}), ((z, s[:, :2]), {}),
                     ((z, s.view(-1)), {}), ((z, s), dict(keep=0)), ((z, s), dict(keep=33)), ((z[..., :2], s), dict(keep=7)),
                     ((z, s), dict(finished=f)), ((z, s), dict(finished=f.int(), end=1)), ((z, s), dict(finished=f[:1], end=1)),
                     ((z, s), dict(end=50)), ((z, s), dict(end=-1)), ((z.repeat(1, 11, 1), s.repeat(1, 11)), {}), ((z[0, 0], s[0]), {}),
                     ((z.transpose(1, 2), s), {}), ((z[:, :0], s[:, :0]), {})]:
        with pytest.raises(ValueError):
            inner.beam_select(*args, **kw)
    for scale in (0.0, -1.0, math.nan, INF):
        with pytest.raises(inner.IsolocoError):
            inner.beam_select(z, s, scale=scale)
