"""A token that a list names several times counts once, with the sum of its entries' weights: loss and gradient are
those of the list in which they are added up."""
import math

import pytest
import torch

import teach_ref as ref
from inner_ref import assert_within

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def added_up(v, ids, vocab):
    """The lists (in 64 bits) with one entry to a token; -1 where there is none."""
    out_v, out_i = torch.zeros(v.shape, dtype=torch.float64), torch.full(ids.shape, -1, dtype=torch.int64)
    for r in range(v.shape[0]):
        weights = {}
        for t, a in zip(ids[r].tolist(), v[r].double().tolist()):
            if 0 <= t < vocab:
                weights.setdefault(t, []).append(a)
        for e, (t, a) in enumerate(weights.items()):
            out_i[r, e] = t
            out_v[r, e] = torch.logsumexp(torch.tensor(a, dtype=torch.float64), 0)
    return out_v, out_i


def run(z, v, ids, w, scale, tail):
    """Loss and gradient in one call, the loss alone, the gradient by itself."""
    from paper_2607_03011_gb300 import inner
    zc, vc, ic, wc = z.cuda(), v.cuda(), ids.cuda(), w.cuda()
    r = inner.distill(zc, vc, ic, scale=scale, tail=tail, grad_loss=wc, save=True)
    alone = inner.distill(zc, vc, ic, scale=scale, tail=tail).loss
    back = inner.distill_grad(wc, zc, vc, ic, r.saved, scale=scale, tail=tail)
    return [r.loss.cpu(), alone.cpu()], [r.grad_logits.cpu(), back.cpu()]


def check(z, v, ids, w, scale, tail):
    mv, mi = added_up(v, ids, z.shape[1])
    loss, dz = ref.distill(z, mv, mi, scale, tail, w)
    losses, grads = run(z, v, ids, w, scale, tail)
    # a token's weight is a sum of at most k terms, and what it is off by counts in its logarithm: both in loss_bound's (16 + k)
    bound = ref.loss_bound(z, v, scale)
    for got in losses:
        assert_within(got, loss, bound, "loss")
    for got in grads:
        assert_within(got, dz, ref.grad_bound(z, v, ids, scale, w, dz), "gradient")
    return losses, grads


def test_worked_rows():
    """A sure student taught by two halves of its token: 0.  A uniform student over four tokens, the weights .45 and .1 on one and
    .45 on another: .55 ln 2.2 + .45 ln 1.8."""
    z = torch.tensor([[60.0, 0.0, 0.0, 0.0], [0.0] * 4, [0.0] * 4])
    ids = torch.tensor([[0, 0, -1], [1, 1, 2], [1, 2, 1]])
    v = torch.log(torch.tensor([[0.5, 0.5, 0.5], [0.45, 0.1, 0.45], [0.45, 0.45, 0.1]]))
    want = torch.tensor([0.0, 0.55 * math.log(2.2) + 0.45 * math.log(1.8), 0.55 * math.log(2.2) + 0.45 * math.log(1.8)])
    for tail in ("drop", "rest"):
        for got in run(z, v, ids, torch.ones(3), 1.0, tail)[0]:
            # each of three logarithms off by some 8 roundings of a number below 64; q and 1 - sum q by (8 + 3) 2^-24 of 1
            assert (got - want).abs().max() < 64 * 16 * 2.0 ** -24
            assert (got > -64 * 16 * 2.0 ** -24).all()


@pytest.mark.parametrize("tail", ["drop", "rest"])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("vocab,k", [(5, 9), (600, 40), (4099, 256), (40000, 65), (70001, 33)])
def test_repeated_tokens(vocab, k, dtype, tail):
    g = torch.Generator().manual_seed(vocab + k)
    z = (torch.randn(6, vocab, generator=g) * 2).to(dtype)
    ids = torch.randint(0, vocab, (6, k), generator=g)
    ids[0] = vocab - 1                              # all of them one token
    ids[1, k // 2:] = ids[1, :k - k // 2].clone()   # in pairs, far apart
    ids[2, 1::2] = ids[2, 0:k - 1:2].clone()         # side by side
    ids[3] = torch.randint(0, 3, (k,), generator=g)
    ids[4, ::3] = -1
    v = torch.log_softmax(torch.randn(6, k + 1, generator=g) * 2, 1)[:, :k]
    v[5, 0], ids[5, -1] = -math.inf, ids[5, 0]      # the first entry of a token without weight
    check(z, v, ids, torch.rand(6, generator=g) + 0.2, 0.8, tail)


@pytest.mark.parametrize("tail", ["drop", "rest"])
def test_a_target_mixed_in(tail):
    """A hard target with weight a beside the teacher's list with weight 1 - a, whether or not the list has it: the loss is the divergence from the
    mixture, which is never negative."""
    g = torch.Generator().manual_seed(9)
    n, vocab, k, a = 32, 3000, 16, 0.3
    t = torch.randn(n, vocab, generator=g) * 2
    top = torch.log_softmax(t, 1).topk(k, 1)
    target = torch.where(torch.arange(n) % 2 == 0, top.indices[:, 3], torch.randint(0, vocab, (n,), generator=g))
    v = torch.cat([top.values + math.log(1 - a), torch.full((n, 1), math.log(a))], 1)
    ids = torch.cat([top.indices, target[:, None]], 1)
    for z in (t, t + torch.randn(n, vocab, generator=g) * 0.1, torch.randn(n, vocab, generator=g)):
        losses, _ = check(z, v, ids, torch.ones(n), 1.0, tail)
        assert (losses[0] >= -ref.loss_bound(z, v, 1.0)).all()


def test_lists_without_repeats_in_another_order():
    """One entry to a token: the order of the entries changes roundings of the sums alone."""
    g = torch.Generator().manual_seed(4)
    z, ids = torch.randn(8, 900, generator=g), torch.stack([torch.randperm(900, generator=g)[:30] for _ in range(8)])
    v = torch.log_softmax(torch.randn(8, 31, generator=g), 1)[:, :30]
    p = torch.randperm(30, generator=g)
    a, b = (run(z, v[:, q], ids[:, q], torch.ones(8), 1.0, "rest")[0][0] for q in (torch.arange(30), p))
    assert ((a - b).abs() <= 2 * ref.loss_bound(z, v, 1.0)).all()
