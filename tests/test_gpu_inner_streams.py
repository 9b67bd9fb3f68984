"""The inner step's operators under stream capture, and on two streams at once: the same bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def data(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def r(*s):
        return torch.randn(s, generator=g, device="cuda")

    n, vocab, d, f = 700, 5000, 256, 520
    return dict(w=r(vocab, d).bfloat16(), ids=torch.randint(0, vocab, (n,), generator=g, device="cuda"), dy=r(n, d).bfloat16(),
                wg=(r(d, f) / 16).bfloat16(), wu=(r(d, f) / 16).bfloat16(), dh=r(n, f).bfloat16(), z=r(n, vocab).bfloat16(),
                t=torch.randint(0, vocab, (n,), generator=g, device="cuda"), gl=r(n), ge=r(n), grads=[r(3_000_001), r(7)], small=[r(100)])


def step(s):
    from paper_2607_03011_gb300 import inner
    x = inner.embed(s["w"], s["ids"])
    h, saved = inner.gated_ffn(x, s["wg"], s["wu"], save=True)
    one = inner.gated_ffn(x[:1], s["wg"], s["wu"])
    back = inner.gated_ffn_grad(s["dh"], x, s["wg"], s["wu"], saved)
    p = inner.token_logprobs(s["z"], s["t"], top=6, grad_logp=s["gl"], grad_entropy=s["ge"])
    few = inner.token_logprobs(s["z"][:3], s["t"][:3])
    dz = inner.token_logprobs_grad(s["z"], s["t"], p.lse, p.entropy, s["gl"], s["ge"])
    out = [torch.empty_like(v) for v in s["grads"]]
    n = inner.clip_grads(s["grads"], 1.0, out=out)
    m = inner.grad_norm(s["small"])
    return [x, h, one, *back, *p, few.logp, few.entropy, dz, n, m, *out, inner.embed_grad(s["dy"], s["ids"], 5000, dtype=torch.float32)]


def test_captured_step():
    s = data(1)
    want = step(s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step(s)
    for v in got:
        v.zero_()
    g.replay()
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    # new inputs at the same addresses
    other = data(2)
    for k in s:
        for a, b in zip(s[k], other[k]) if isinstance(s[k], list) else [(s[k], other[k])]:
            a.copy_(b)
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, step(other)))


def test_two_streams_at_once():
    sets = [data(3), data(4)]
    want = [step(s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        got = []
        for s, st in zip(sets, streams):
            with torch.cuda.stream(st):
                got.append(step(s))
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(p, q) for p, q in zip(a, b))
