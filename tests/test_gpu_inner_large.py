"""Tensors of more than 2^31 (and 2^32) elements: the rows at the far end come out as they do alone."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def room():
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB")
    yield
    torch.cuda.empty_cache()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def test_embedding():
    from paper_2607_03011_gb300 import inner
    n, vocab, width = 4_300_000, 1000, 1024     # 4.4e9 elements
    w = torch.randn(vocab, width, generator=gen(1), device="cuda").bfloat16()
    ids = torch.randint(0, vocab - 1, (n,), generator=gen(2), device="cuda")
    ids[-5:] = vocab - 1                        # one token only at the far end
    y = inner.embed(w, ids)
    assert torch.equal(y[-1000:], w[ids[-1000:]]) and torch.equal(y[:1000], w[ids[:1000]])
    y[-5:] = torch.arange(1, 6, device="cuda", dtype=torch.bfloat16)[:, None]
    dw = inner.embed_grad(y, ids, vocab, dtype=torch.float32)
    assert torch.equal(dw[-1], torch.full((width,), 15.0, device="cuda"))


def test_gated_block():
    from paper_2607_03011_gb300 import inner, isoloco
    n, width, ff = 560_000, 64, 8192            # 4.6e9 elements in h
    x = torch.randn(n, width, generator=gen(3), device="cuda").bfloat16()
    wg = (torch.randn(width, ff, generator=gen(4), device="cuda") / 8).bfloat16()
    wu = (torch.randn(width, ff, generator=gen(5), device="cuda") / 8).bfloat16()
    h, saved = inner.gated_ffn(x, wg, wu, save=True)
    part, psaved = inner.gated_ffn(x[-512:], wg, wu, save=True)
    assert torch.equal(h[-512:], part)
    dh = h                                      # any gradient will do
    dx, _, _ = inner.gated_ffn_grad(dh, x, wg, wu, saved, need_w=False)
    pdx, _, _ = inner.gated_ffn_grad(part, x[-512:], wg, wu, psaved, need_w=False)
    assert torch.equal(dx[-512:], pdx) and inner.status() == isoloco.OK


def test_token_logprobs():
    from paper_2607_03011_gb300 import inner
    n, vocab = 36_000, 128_000                  # 4.6e9 elements
    z = torch.zeros(n, vocab, device="cuda", dtype=torch.bfloat16)
    far = torch.randn(64, vocab, generator=gen(6), device="cuda").bfloat16()
    z[-64:] = far
    t = torch.randint(0, vocab, (n,), generator=gen(7), device="cuda")
    g = torch.ones(n, device="cuda")
    r = inner.token_logprobs(z, t, top=3, grad_logp=g)
    # the same rows among as many that the same kernel takes
    few = torch.zeros(2048, vocab, device="cuda", dtype=torch.bfloat16)
    few[-64:] = far
    p = inner.token_logprobs(few, t[-2048:], top=3, grad_logp=g[-2048:])
    for a, b in ((r.logp, p.logp), (r.entropy, p.entropy), (r.top_index, p.top_index), (r.top_logp, p.top_logp),
                 (r.grad_logits, p.grad_logits)):
        assert torch.equal(a[-64:], b[-64:])
    d = inner.token_logprobs_grad(z, t, r.lse, r.entropy, g, None)
    assert torch.allclose(d[-64:].float(), r.grad_logits[-64:].float(), rtol=2.0 ** -7, atol=2.0 ** -30)


def test_clipping():
    from paper_2607_03011_gb300 import inner
    n = (1 << 32) + 12_345
    t = torch.full((n,), 0.5, device="cuda", dtype=torch.bfloat16)
    t[-1] = 1024.0
    want = (0.25 * (n - 1) + 1024.0 ** 2) ** 0.5
    norm = inner.clip_grads([t], want / 2)
    assert abs(norm.item() - want) < 1e-5 * want
    assert t[-1] == 512.0 and t[-2] == 0.25 and t[0] == 0.25 and t[1 << 31] == 0.25
