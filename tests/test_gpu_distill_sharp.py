"""Teachers whose list holds nearly everything: what is left for the other tokens, r = 1 - sum q, is small beside the
roundings of q in fp32, and sets the gradient of every other token."""
import math

import pytest
import torch

import teach_ref as ref
from inner_ref import assert_within

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def lists(left, shape, k, g):
    """fp32 log probabilities of k entries that leave `left`: one sure entry, two heavy ones, or many alike."""
    q = torch.rand(k, generator=g, dtype=torch.float64) + 0.1
    if shape == "one":
        q[1:] *= left / q[1:].sum()
        q[0] = 1 - 2 * left
    elif shape == "two":
        q[2:] *= left / q[2:].sum()
        q[0], q[1] = 0.6, 0.4 - 2 * left
    else:
        q *= (1 - left) / q.sum()
    return q.log().float()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", ["one", "two", "many"])
@pytest.mark.parametrize("vocab", [300, 5003, 40000, 90001])
def test_small_rests(vocab, shape, dtype):
    from paper_2607_03011_gb300 import inner
    g = torch.Generator().manual_seed(vocab)
    lefts = [0.2, 0.03, 1e-3, 1e-4, 1e-5, 1e-6, 1e-7, 0.0, -1e-3]
    n, k = len(lefts), 48
    z = torch.randn(n, vocab, generator=g) * 2
    ids = torch.stack([torch.randperm(vocab, generator=g)[:k] for _ in range(n)])
    z = z.scatter_add(1, ids, torch.full((n, k), 20.0)).to(dtype)   # a student as sure as the teacher
    v = torch.stack([lists(max(a, 0.0), shape, k, g) for a in lefts])
    v[-1] += 1e-3                                   # more than everything: nothing is left
    w = torch.rand(n, generator=g) + 0.5
    loss, dz = ref.distill(z, v, ids, 1.0, "rest", w)
    rest = (1.0 - v.double().exp().sum(1)).clamp_min(0.0)
    assert (rest[:7] > 0).all() and rest[-1] == 0.0 and (rest[4:7] < 2e-5).all()

    zc, vc, ic, wc = z.cuda(), v.cuda(), ids.cuda(), w.cuda()
    r = inner.distill(zc, vc, ic, tail="rest", grad_loss=wc, save=True)
    alone = inner.distill(zc, vc, ic, tail="rest").loss
    back = inner.distill_grad(wc, zc, vc, ic, r.saved, tail="rest")
    for got in (r.loss.cpu(), alone.cpu()):
        assert_within(got, loss, ref.loss_bound(z, v, 1.0), "loss")
    # Outside the list an entry is w (p Q - r p / P).  p, P and their quotients are off by sums' and powers' shares of themselves (as
    # in ref.grad_bound), Q by (8 + k) 2^-24 of itself, and r by a rounding of its value and 2^-43 for each entry of the list.
    p = torch.softmax(z.double(), 1)
    outside = torch.ones(n, vocab, dtype=torch.float64).scatter_(1, ids, 0.0)
    share = p * outside / (p * outside).sum(1, keepdim=True)
    rel = 4 * ref.sum_of_powers(vocab) + (ref._size(z, v, 1.0)[:, None] + 16 + k) * 2.0 ** -23
    of_rest = (rest * 2.0 ** -23 + (k + 8) * 2.0 ** -43)[:, None]
    bound = w[:, None] * (rel * (2 * p * 1.01 + rest[:, None] * share) + of_rest * share) + 1.01 * w[:, None] * 2.0 ** -126
    for name, got in (("gradient", r.grad_logits), ("gradient by itself", back)):
        d = got.cpu()
        assert_within(d[outside > 0], dz[outside > 0], bound[outside > 0], name)
        assert_within(d, dz, ref.grad_bound(z, v, ids, 1.0, w, dz), name)


def test_the_outside_gradient_of_a_sure_pair():
    """Student and teacher both sure of two tokens, each leaving some 1e-6: the gradient outside is a difference of the student's
    share and the teacher's, of which fp32 sums of q would lose some hundredths."""
    from paper_2607_03011_gb300 import inner
    vocab = 64
    z = torch.full((1, vocab), 0.0)
    z[0, :2] = 17.0
    q = torch.tensor([[0.7, 0.3 - 2e-6]], dtype=torch.float64)
    v, ids = q.log().float(), torch.tensor([[0, 1]])
    _, dz = ref.distill(z, v, ids, 1.0, "rest", torch.ones(1))
    got = inner.distill(z.cuda(), v.cuda(), ids.cuda(), tail="rest", grad_loss=torch.ones(1, device="cuda")).grad_logits.cpu().double()
    rest, share = 1 - v.double().exp().sum().item(), 1 / (vocab - 2)
    student = (vocab - 2) / (2 * math.exp(17.0) + vocab - 2)
    # the student's share is off by 51 roundings for its power of -17 / ln 2 and some dozen for its other operations, the rest by fewer
    assert ((got - dz)[0, 2:].abs() <= 64 * 2.0 ** -24 * share * (rest + student)).all()
