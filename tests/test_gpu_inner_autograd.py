"""Autograd records nothing of these operators, as the module says: operands that require a gradient change no result, and
a torch.autograd.Function around a pair of functions is how a loss.backward() goes through them."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_outputs_require_no_gradient():
    from paper_2607_03011_gb300 import inner
    assert "autograd" in inner.__doc__
    w = torch.randn(50, 64, device="cuda").bfloat16()
    wg, wu = (torch.randn(64, 128, device="cuda") / 8).bfloat16(), (torch.randn(64, 128, device="cuda") / 8).bfloat16()
    ids = torch.arange(40, device="cuda")
    for on in (False, True):
        a, b, c = (v.detach().requires_grad_(on) for v in (w, wg, wu))
        x = inner.embed(a, ids)
        h, saved = inner.gated_ffn(x, b, c, save=True)
        r = inner.token_logprobs(h, ids, top=2, grad_logp=torch.ones(40, device="cuda"))
        d = inner.gated_ffn_grad(r.grad_logits, x, b, c, saved)
        out = [x, h, *r, *d, inner.embed_grad(d[0], ids, 50), inner.grad_norm([a, b])]
        assert not any(t.requires_grad for t in out)
        if on:
            assert all(torch.equal(p, q) for p, q in zip(out, plain))
        plain = out


def test_inside_an_autograd_function():
    from paper_2607_03011_gb300 import inner

    class Lookup(torch.autograd.Function):
        @staticmethod
        def forward(ctx, weight, ids):
            ctx.save_for_backward(ids)
            ctx.vocab = weight.shape[0]
            return inner.embed(weight, ids)

        @staticmethod
        def backward(ctx, dy):
            return inner.embed_grad(dy.contiguous(), *ctx.saved_tensors, ctx.vocab), None

    w = torch.randn(20, 32, device="cuda", requires_grad=True)
    ids = torch.randint(0, 20, (60,), device="cuda")
    v = torch.randn(60, 32, device="cuda")
    (Lookup.apply(w, ids) * v).sum().backward()
    want = torch.zeros(20, 32, device="cuda", dtype=torch.float64).index_add_(0, ids, v.double())
    # at most 60 terms of order 1 in fp32
    assert (w.grad.double() - want).abs().max() < 60 * 2.0 ** -20
