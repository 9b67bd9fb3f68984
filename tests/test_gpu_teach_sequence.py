"""Teaching and answering as they are used: a search whose beams carry states along, then a student that learns from the
teacher's top tokens along the answers; under capture, and on two streams at once."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

VOCAB, WIDTH = 401, 64


def model(seed, std=0.5):
    """A language model that looks at the last two tokens: logits from their embeddings."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    return {k: (torch.randn(s, generator=g, device="cuda") * std).bfloat16() for k, s in (("embed", (VOCAB, WIDTH)), ("head", (VOCAB, WIDTH)))}


def logits(m, last, before):
    from paper_2607_03011_gb300 import inner
    x = inner.embed(m["embed"], last).float() + 0.5 * inner.embed(m["embed"], before).float()
    return (x.bfloat16() @ m["head"].t())


def search(m, prompt, beams, steps, end):
    """The library's search: states are a cache of what the model looks at, and the tokens so far."""
    from paper_2607_03011_gb300 import inner
    batch = prompt.shape[0]
    tokens = torch.zeros(batch, beams, steps + 1, dtype=torch.int64, device="cuda")
    tokens[:, :, 0] = prompt[:, None]
    cache = torch.zeros(batch * beams, 2, steps + 1, 8, dtype=torch.bfloat16, device="cuda")
    scores = torch.full((batch, beams), -math.inf, device="cuda")
    scores[:, 0] = 0.0
    finished = torch.zeros(batch, beams, dtype=torch.bool, device="cuda")
    for i in range(steps):
        last, before = tokens[:, :, i], tokens[:, :, max(i - 1, 0)]
        cache[:, 0, i] = last.reshape(-1, 1).to(torch.bfloat16)
        cache[:, 1, i] = -last.reshape(-1, 1).to(torch.bfloat16)
        z = logits(m, last.contiguous(), before.contiguous())
        scores, came, token, finished = inner.beam_select(z, scores, finished=finished, end=end)
        inner.beam_reorder([tokens[:, :, :i + 1], cache[:, :, :i + 1]], came)
        tokens[:, :, i + 1] = token
    return scores, tokens, cache, finished


def plain_search(m, prompt, beams, steps, end):
    """The same, hypothesis by hypothesis, on the CPU (the logits are the GPU's)."""
    out = []
    for p in prompt.tolist():
        hyps = [(0.0, [p], False)]
        for i in range(steps):
            last = torch.tensor([h[1][-1] for h in hyps], device="cuda")
            before = torch.tensor([h[1][max(i - 1, 0)] for h in hyps], device="cuda")
            lp = torch.log_softmax(logits(m, last, before).double(), 1).cpu()
            more = []
            for (score, seq, done), row in zip(hyps, lp):
                if done:
                    more.append((score, seq + [end], True))
                else:
                    order = torch.sort(row, descending=True, stable=True).indices[:beams]
                    more += [(score + row[t].item(), seq + [t.item()], t.item() == end) for t in order]
            more.sort(key=lambda h: -h[0])
            hyps = more[:beams]
        out.append(hyps)
    return out


@pytest.mark.parametrize("beams", [1, 4, 9])
def test_search_finds_what_a_plain_search_finds(beams):
    m, steps, end = model(1), 6, 5
    prompt = torch.tensor([7, 300, 42], device="cuda")
    scores, tokens, cache, finished = search(m, prompt, beams, steps, end)
    want = plain_search(m, prompt, beams, steps, end)
    for b, hyps in enumerate(want):
        assert tokens[b].tolist() == [h[1] for h in hyps]
        assert finished[b].tolist() == [h[2] for h in hyps]
        # every step rounds the score to fp32 once, and each log sum is off by 2^-20 at most
        assert torch.allclose(scores[b].cpu().double(), torch.tensor([h[0] for h in hyps], dtype=torch.float64), rtol=0, atol=steps * 4 * 2.0 ** -20)
    # the cache went along with the tokens
    held = tokens[:, :, :steps].reshape(-1, steps).to(torch.bfloat16)
    assert torch.equal(cache[:, 0, :steps, 3], held) and torch.equal(cache[:, 1, :steps, 0], -held)


def taught(teacher, student, tokens, k, tail):
    """One distillation step along the answers: per-row losses, and the gradients of the student's tables."""
    from paper_2607_03011_gb300 import inner
    last, before = tokens[..., 1:].reshape(-1), tokens[..., :-1].reshape(-1)
    t = inner.token_logprobs(logits(teacher, last, before), last, top=k)
    x = inner.embed(student["embed"], last).float() + 0.5 * inner.embed(student["embed"], before).float()
    z = x.bfloat16() @ student["head"].t()
    g = torch.full((last.numel(),), 1.0 / last.numel(), device="cuda")
    r = inner.distill(z, t.top_logp, t.top_index, tail=tail, grad_loss=g, save=True)
    back = inner.distill_grad(g, z, t.top_logp, t.top_index, r.saved, tail=tail)
    dx = r.grad_logits @ student["head"]
    grads = [r.grad_logits.t() @ x.bfloat16(), inner.embed_grad(dx, last, VOCAB, dtype=torch.float32)]
    norm = inner.clip_grads(grads, 1.0)
    return [r.loss, r.saved, r.grad_logits, back, t.top_logp, t.top_index, norm, *grads], z


@pytest.mark.parametrize("tail", ["drop", "rest"])
def test_student_learns_along_the_answers(tail):
    teacher, student = model(1), model(2)
    _, tokens, _, _ = search(teacher, torch.arange(8, device="cuda") * 40, 4, 5, 5)
    (loss, _, dz, back, v, i, *_), z = taught(teacher, student, tokens, 12, tail)
    x = z.double().requires_grad_(True)
    lp = torch.log_softmax(x, 1)
    q = torch.softmax(v.double(), 1) if tail == "drop" else v.double().exp()
    want = (q * (q.log() - lp.gather(1, i))).sum(1)
    if tail == "rest":
        p = lp.gather(1, i).exp().sum(1)
        want = want + (1 - q.sum(1)) * ((1 - q.sum(1)).log() - (1 - p).log())
    assert torch.allclose(loss.double(), want, rtol=2e-5, atol=2e-5)
    d = torch.autograd.grad(want.mean(), x)[0]
    for got in (dz, back):
        # one rounding to bf16 in each entry, subnormals aside
        assert ((got.double() - d).abs() <= 2.0 ** -8 * d.abs() + 1e-7).all()


def step(s):
    scores, tokens, cache, finished = search(s["teacher"], s["prompt"], 4, 4, 5)
    out, _ = taught(s["teacher"], s["student"], tokens, 10, "rest")
    return [scores, tokens, cache, finished, *out]


def data(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return dict(teacher=model(seed), student=model(seed + 50), prompt=torch.randint(0, VOCAB, (6,), generator=g, device="cuda"))


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b)) and len(a) == len(b)


def test_captured_steps():
    s = data(3)
    want = step(s)
    torch.cuda.synchronize()
    g, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step(s)
    s2 = data(4)
    want2 = step(s2)
    torch.cuda.synchronize()
    with torch.cuda.graph(other, pool=g.pool()):   # (two graphs of one memory pool)
        got2 = step(s2)
    for _ in range(2):
        g.replay()
        torch.cuda.synchronize()
        assert same(got, want)
        other.replay()
        torch.cuda.synchronize()
        assert same(got2, want2)
    # new inputs at the same addresses
    new = data(9)
    for k in ("teacher", "student"):
        for n in s[k]:
            s[k][n].copy_(new[k][n])
    s["prompt"].copy_(new["prompt"])
    g.replay()
    torch.cuda.synchronize()
    assert same(got, step(new))


def test_two_streams_at_once():
    sets = [data(5), data(6)]
    want = [step(s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        got = []
        for s, st in zip(sets, streams):
            with torch.cuda.stream(st):
                got.append(step(s))
        torch.cuda.synchronize()
        assert all(same(a, b) for a, b in zip(got, want))


def test_the_stream_argument():
    """Work, outputs and kept inputs go to the stream that is named."""
    from paper_2607_03011_gb300 import inner
    g = torch.Generator(device="cuda").manual_seed(1)
    z = torch.randn(40, 3000, generator=g, device="cuda").bfloat16()
    v, i = torch.randn(40, 8, generator=g, device="cuda").log_softmax(1), torch.randint(0, 3000, (40, 8), generator=g, device="cuda")
    w, c = torch.rand(40, generator=g, device="cuda"), torch.randn(40, 5, generator=g, device="cuda")
    sc, beams = torch.zeros(10, 4, device="cuda"), torch.randint(0, 4, (10, 4), generator=g, device="cuda")
    torch.cuda.synchronize()
    st = torch.cuda.Stream()

    def calls(**kw):
        r = inner.distill(z, v, i, grad_loss=w, save=True, **kw)
        d = inner.distill_grad(w, z, v, i, r.saved, **kw)
        b = inner.beam_select(z.view(10, 4, 3000), sc, end=3, **kw)
        o = inner.beam_reorder(iter([c]), beams, out=(t for t in [torch.empty_like(c)]), **kw)
        return [*r, d, *b, *o]

    got = calls(stream=st)
    st.synchronize()
    want = calls()
    torch.cuda.synchronize()
    assert same(got, want)
    assert inner.status() == 0
