"""Embedding lookup and its gradient against plain 64-bit sums, and by differences."""
import pytest
import torch

import inner_ref as ref

pytestmark = pytest.mark.gpu
DT = [torch.float32, torch.bfloat16, torch.float16]


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def ids_of(kind, n, vocab, g):
    if kind == "one":     # every position the same token
        return torch.full((n,), vocab // 2, device="cuda", dtype=torch.int64)
    if kind == "none":    # nothing is a token
        return torch.where(torch.arange(n, device="cuda") % 2 == 0, -1, vocab + 3)
    if kind == "skew":
        u = torch.rand(n, generator=g, device="cuda")
        ids = (torch.exp(u * torch.log(torch.tensor(vocab + 1.0))) - 1).long().clamp(0, vocab - 1)
        ids[torch.rand(n, generator=g, device="cuda") < 0.1] = -1
        return ids
    return torch.randint(0, vocab, (n,), generator=g, device="cuda")


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("n,vocab,width,pad,id_t", [(1, 1, 1, 0, torch.int64), (7, 500, 64, 0, torch.int32),
                                                    (33, 129, 65, 0, torch.int64), (130, 1000, 1024, 8, torch.int64),
                                                    (70001, 50, 8, 3, torch.int32), (3, 40, 5000, 0, torch.int64)])
def test_lookup(dt, n, vocab, width, pad, id_t):
    from paper_2607_03011_gb300 import inner
    g = gen(n)
    w = torch.randn(vocab, width + pad, generator=g, device="cuda").to(dt)[:, :width]
    ids = ids_of("skew", n, vocab, g).to(id_t)
    for scale in (1.0, 3.7):
        y = inner.embed(w, ids, scale=scale)
        ok = ((ids >= 0) & (ids < vocab))[:, None]
        s32 = torch.tensor(scale, device="cuda")
        assert torch.equal(y, (w[ids.long().clamp(0, vocab - 1)].float() * s32 * ok).to(dt))


def test_lookup_of_any_shape_and_of_nothing():
    from paper_2607_03011_gb300 import inner
    w = torch.randn(20, 24, device="cuda")
    ids = torch.randint(0, 20, (2, 3, 5), device="cuda")
    assert torch.equal(inner.embed(w, ids), w[ids])
    assert inner.embed(w, ids[:0]).shape == (0, 3, 5, 24)
    assert inner.embed_grad(torch.empty(0, 24, device="cuda"), ids.new_empty(0), 20).abs().max() == 0


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("kind,n,vocab,width", [("any", 1, 1, 1), ("any", 31, 7, 24), ("any", 33, 300, 65), ("one", 1000, 5, 64),
                                                ("none", 100, 64, 16), ("skew", 4097, 1000, 136), ("any", 5000, 32000, 48),
                                                ("skew", 70000, 130000, 8), ("one", 40000, 3, 16), ("skew", 513, 255, 256),
                                                ("any", 2049, 256, 1025)])
def test_gradient(dt, kind, n, vocab, width):
    from paper_2607_03011_gb300 import inner
    g = gen(n + vocab)
    ids = ids_of(kind, n, vocab, g)
    dy = torch.randn(n, width, generator=g, device="cuda").to(dt)
    exact, bound = ref.embed_grad(dy, ids, vocab, 0.5)
    for out in {dt, torch.float32}:
        dw = inner.embed_grad(dy, ids, vocab, scale=0.5, dtype=out)
        assert dw.dtype == out
        ref.assert_within(dw, exact, bound, f"{kind} {out}")
        again = inner.embed_grad(dy, ids.int(), vocab, scale=0.5, dtype=out)
        assert torch.equal(dw, again)  # same bits, whatever order the blocks ran in


def test_gradient_strided_rows_and_stream():
    from paper_2607_03011_gb300 import inner
    g = gen(3)
    for pad, off in ((8, 0), (3, 1)):
        full = torch.randn(700, 64 + pad, generator=g, device="cuda")
        dy = full[:, off:off + 64]
        ids = ids_of("skew", 700, 90, g)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        dw = inner.embed_grad(dy, ids, 90, stream=s)
        s.synchronize()
        exact, bound = ref.embed_grad(dy, ids, 90, 1.0)
        ref.assert_within(dw, exact, bound)


def test_gradient_is_the_difference_quotient():
    """The lookup is linear: <dy, embed(W + V) - embed(W)> = <dW, V>."""
    from paper_2607_03011_gb300 import inner
    g = gen(5)
    w = torch.randn(40, 32, generator=g, device="cuda")
    v = torch.randn(40, 32, generator=g, device="cuda")
    ids = ids_of("skew", 300, 40, g)
    dy = torch.randn(300, 32, generator=g, device="cuda")
    lhs = (dy.double() * (inner.embed(w + v, ids, scale=2.0).double() - inner.embed(w, ids, scale=2.0).double())).sum()
    dw = inner.embed_grad(dy, ids, 40, scale=2.0)
    rhs = (dw.double() * ((w + v).double() - w.double())).sum()
    # fp32 roundings of 9600 terms of order 10: 9600 * 10 * 2^-23
    assert abs(lhs - rhs) < 9600 * 10 * 2.0 ** -23


def test_refusals():
    from paper_2607_03011_gb300 import inner, isoloco
    w = torch.randn(10, 16, device="cuda")
    ids = torch.zeros(4, dtype=torch.int64, device="cuda")
    for bad in (lambda: inner.embed(w.double(), ids), lambda: inner.embed(w, ids.float()), lambda: inner.embed(w.cpu(), ids),
                lambda: inner.embed(w.t(), ids), lambda: inner.embed(w, ids.cpu()), lambda: inner.embed(w, torch.stack([ids, ids], 1)[:, 0]),
                lambda: inner.embed_grad(torch.randn(5, 16, device="cuda"), ids, 10),
                lambda: inner.embed_grad(torch.randn(4, 16, device="cuda"), ids, 0),
                lambda: inner.embed_grad(torch.randn(4, 16, device="cuda"), ids, 10, dtype=torch.bfloat16),
                lambda: inner.embed(torch.randn(10, 0, device="cuda"), ids)):
        with pytest.raises((ValueError, isoloco.IsolocoError)):
            bad()
    torch.cuda.synchronize()
