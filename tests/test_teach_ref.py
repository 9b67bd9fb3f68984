"""The plain implementations that the distillation and beam tests compare with: worked examples, torch's autograd and
differences."""
import math

import pytest
import torch

import teach_ref as ref


def test_a_worked_row():
    # p = (1/2, 1/4, 1/4), teacher 3/4 on token 0 and 1/8 on token 2
    z = torch.tensor([[math.log(2.0), 0.0, 0.0]], dtype=torch.float64).float()
    ids, v = torch.tensor([[0, 2]]), torch.log(torch.tensor([[0.75, 0.125]]))
    rest = ref.distill(z, v, ids, 1.0, "rest")[0].item()
    assert abs(rest - (0.75 * math.log(1.5) + 0.125 * math.log(0.5) + 0.125 * math.log(0.5))) < 1e-6
    drop = ref.distill(z, v, ids, 1.0, "drop")[0].item()
    assert abs(drop - (6 / 7 * math.log(12 / 7) + 1 / 7 * math.log(4 / 7))) < 1e-6


@pytest.mark.parametrize("tail", ["drop", "rest"])
@pytest.mark.parametrize("scale", [1.0, 0.4])
def test_gradient_against_autograd_and_differences(tail, scale):
    g = torch.Generator().manual_seed(3)
    n, vocab, k = 5, 23, 6
    z = torch.randn(n, vocab, generator=g).float()
    ids = torch.randint(-2, vocab, (n, k), generator=g)
    ids[1] = ids[1, 0]  # one token alone
    v = torch.log_softmax(torch.randn(n, k + 1, generator=g), 1)[:, :k].float()
    w = torch.rand(n, generator=g) + 0.5
    loss, dz = ref.distill(z, v, ids, scale, tail, w)

    def plain(x):
        total = 0.0
        for r in range(n):
            here = [e for e in range(k) if ids[r, e] >= 0]
            lw = v[r, here].double()
            if not here:
                continue
            q = torch.softmax(lw, 0) if tail == "drop" else lw.exp()
            lp = torch.log_softmax(x[r] * scale, 0)
            t = (q * (q.log() - lp[ids[r, here]])).sum()
            if tail == "rest" and 1 - q.sum() > 0:
                other = sorted(set(range(vocab)) - set(ids[r, here].tolist()))
                rest = 1 - q.sum()
                t = t + rest * (rest.log() - lp[other].exp().sum().log())
            total = total + w[r].double() * t
        return total

    x = z.double().requires_grad_(True)
    t = plain(x)
    assert abs((loss * w.double()).sum().item() - t.item()) < 1e-12
    assert torch.allclose(torch.autograd.grad(t, x)[0], dz, rtol=1e-9, atol=1e-12)
    for r, j in ((0, 3), (1, int(ids[1, 0])), (4, 22)):
        h, up, down = 1e-6, z.double(), z.double()
        up, down = up.clone(), down.clone()
        up[r, j] += h
        down[r, j] -= h
        assert abs((plain(up) - plain(down)).item() / (2 * h) - dz[r, j].item()) < 1e-8


def test_a_worked_selection():
    z = torch.log(torch.tensor([[[1.0, 2.0, 1.0], [4.0, 3.0, 1.0]]]))
    total, beams, tokens = ref.select(z, torch.tensor([[0.0, -0.25]]), 3)
    assert beams.tolist() == [[0, 1, 1]] and tokens.tolist() == [[1, 0, 1]]
    want = torch.tensor([[math.log(0.5), math.log(0.5) - 0.25, math.log(3 / 8) - 0.25]], dtype=torch.float64)
    assert torch.allclose(total, want, atol=1e-6)
    # a finished beam goes on with its end token, ties go to the lower beam, then the lower token
    total, beams, tokens = ref.select(z, torch.tensor([[0.0, -0.25]]), 6, torch.tensor([[False, True]]), 2)
    assert (beams[0, 0], tokens[0, 0], total[0, 0]) == (1, 2, -0.25)
    assert list(zip(beams[0].tolist(), tokens[0].tolist()))[1:] == [(0, 1), (0, 0), (0, 2), (1, 0), (1, 1)]
