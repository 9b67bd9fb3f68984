"""Token log probabilities, entropy, alternatives and their gradient against 64-bit formulas."""
import pytest
import torch

import inner_ref as ref

pytestmark = pytest.mark.gpu
DT = [torch.float32, torch.bfloat16, torch.float16]
INF = float("inf")


def make(dt, n, v, seed, pad=0, std=2.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn(n, v + pad, generator=g, device="cuda") * std
    z[:, v // 2] += 6.0
    t = torch.randint(0, v, (n,), generator=g, device="cuda")
    gl = torch.randn(n, generator=g, device="cuda")
    ge = torch.randn(n, generator=g, device="cuda")
    return z.to(dt)[:, :v], t, gl, ge


def check_stats(r, z, t, scale, k=0):
    """fp32 statistics: the log of a sum is good to (v + 8) 2^-23 relative in the sum (so absolutely in
    the log), and z - lse adds a rounding of each of its parts."""
    e = ref.logprobs(z, t, scale)
    v = z.shape[1]
    zmax = (z.double() * scale).masked_fill(torch.isinf(z), 0).abs().amax(1)
    base = min(1.0, ref.sum_err(v)) * 4 + 8 * 2.0 ** -23 * (1 + zmax.masked_fill(zmax > 1e30, 0))
    for name in ("logp", "lse"):
        x, y = getattr(r, name).double().view(-1), e[name]
        fin = torch.isfinite(y)
        assert torch.equal(x[~fin], y[~fin]), name
        big = 2.0 ** -22 * y[fin].abs()
        assert ((x - y)[fin].abs() <= base[fin] + big).all(), (name, (x - y)[fin].abs().max().item())
    # entropy: each of p's and log p's errors enter once per unit of probability, so the same size times
    # the entropy's own scale, log v
    tol = base * (2 + torch.log(torch.tensor(float(v) + 1)).item())
    assert ((r.entropy.double().view(-1) - e["entropy"]).abs() <= tol).all(), (r.entropy.double().view(-1) - e["entropy"]).abs().max()
    if k:
        idx = ref.top(z, k)
        assert torch.equal(r.top_index.view(-1, k), idx)
        lp = e["lp"].gather(1, idx)
        got = r.top_logp.double().view(-1, k)
        fin = torch.isfinite(lp)
        assert torch.equal(got[~fin], lp[~fin])
        assert (((got - lp).abs() <= base[:, None] + 2.0 ** -22 * lp.abs()) | ~fin).all()
    return e, base


def check_grad(d, e, base, scale, gl, ge):
    exact = ref.logprobs_grad(e, scale, gl, ge)
    # p is off by `base` relative; log p + H by `base` + the entropy's tolerance absolutely
    v = e["p"].shape[1]
    eh = base[:, None] * (3 + torch.log(torch.tensor(float(v) + 1)).item())
    lpH = torch.where(e["p"] > 0, (e["lp"] + e["entropy"][:, None]).abs(), torch.zeros_like(e["p"]))
    b = torch.zeros_like(exact)
    if gl is not None:
        hot = torch.zeros_like(exact).scatter_(1, e["t"][:, None], 1.0)
        b += gl.double().abs()[:, None] * (e["p"] * base[:, None] + 2.0 ** -22 * (hot + e["p"]))
    if ge is not None:
        b += ge.double().abs()[:, None] * e["p"] * (lpH * base[:, None] + eh + 2.0 ** -22 * lpH)
    # exponentials below fp32's normal range may flush to zero
    b += ((gl.double().abs() if gl is not None else 0) + (ge.double().abs() * 200 if ge is not None else 0))[:, None] * 2.0 ** -126
    ref.assert_within(d.view(exact.shape), exact, b * scale, "grad_logits")


SIZES = [(1, 1, 0), (1, 5, 0), (3, 33, 0), (2, 257, 3), (5, 1000, 0), (4, 1023, 0), (2, 4096, 8), (3, 4099, 0), (1, 32000, 0),
         (9, 32000, 0), (2, 50021, 0), (1, 128003, 0), (700, 515, 0), (1300, 130, 1), (2, 300007, 0)]


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("n,v,pad", SIZES)
@pytest.mark.parametrize("scale", [1.0, 0.6])
def test_statistics_and_alternatives(dt, n, v, pad, scale):
    from paper_2607_03011_gb300 import inner
    z, t, gl, ge = make(dt, n, v, n + v, pad)
    if n > 1:
        t[::3] = -100
    scale = torch.tensor(scale).item()
    r = inner.token_logprobs(z, t, scale=scale)
    assert r.top_index is None and r.grad_logits is None
    check_stats(r, z, t, scale)
    for k in sorted({1, min(5, v), min(20, v), min(32, v)}):
        check_stats(inner.token_logprobs(z, t.int(), scale=scale, top=k), z, t, scale, k)


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("n,v,pad", SIZES)
def test_gradient(dt, n, v, pad):
    from paper_2607_03011_gb300 import inner
    z, t, gl, ge = make(dt, n, v, 2 * n + v, pad)
    if n > 1:
        t[::4] = v
    for a, b, scale in ((gl, ge, 1.0), (gl, None, 0.75), (None, ge, 1.0)):
        r = inner.token_logprobs(z, t, scale=scale, grad_logp=a, grad_entropy=b)
        e, base = check_stats(r, z, t, scale)
        check_grad(r.grad_logits, e, base, scale, a, b)
        d = inner.token_logprobs_grad(z, t, r.lse, r.entropy, a, b, scale=scale)
        check_grad(d, e, base, scale, a, b)
        again = inner.token_logprobs(z, t, scale=scale, grad_logp=a, grad_entropy=b)
        assert all(torch.equal(p, q) for p, q in zip((r.logp, r.entropy, r.lse, r.grad_logits),
                                                     (again.logp, again.entropy, again.lse, again.grad_logits)))


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("v", [40, 700, 5000, 33001])
def test_masks(dt, v):
    """Rows masked by -inf or the type's lowest value: all but one entry, all but a tail, everything."""
    from paper_2607_03011_gb300 import inner
    z, t, gl, ge = make(dt, 9, v, v)
    low = torch.finfo(dt).min
    z[0, 1:] = -INF
    z[1, :-1] = -INF
    z[2, : v // 2] = -INF
    z[3] = -INF                       # nothing is left
    z[4, 1:] = low
    z[5, :-3] = low
    z[6] = low                        # all equal: uniform
    z[7] = 0.0
    z[8, ::2] = -INF
    t[0], t[1], t[2], t[3] = 0, 0, v - 1, 2
    k = min(20, v)
    r = inner.token_logprobs(z, t, top=k, grad_logp=gl, grad_entropy=ge)
    e, base = check_stats(r, z, t, 1.0, k)
    assert r.logp[0] == 0 and r.logp[1] == -INF and r.logp[3] == -INF and r.lse[3] == -INF and r.entropy[3] == 0
    assert r.entropy[0] == 0 and (r.grad_logits[3] == 0).all()
    assert torch.isfinite(r.grad_logits).all()
    check_grad(r.grad_logits, e, base, 1.0, gl, ge)
    d = inner.token_logprobs_grad(z, t, r.lse, r.entropy, gl, ge)
    assert torch.isfinite(d).all() and (d[3] == 0).all()


@pytest.mark.parametrize("v", [50, 3000, 40000])
def test_equal_logits_go_by_index(v):
    from paper_2607_03011_gb300 import inner
    g = torch.Generator(device="cuda").manual_seed(v)
    z = torch.randint(-2, 3, (12, v), generator=g, device="cuda").to(torch.bfloat16)
    z[0] = 1.0
    z[1] = torch.arange(v, device="cuda").to(torch.bfloat16)           # rising, with ties
    z[2] = -torch.arange(v, device="cuda").to(torch.bfloat16)          # falling
    z[3, :] = 0.0
    z[3, ::2] = -0.0                                                   # -0 equals 0
    t = torch.zeros(12, dtype=torch.int64, device="cuda")
    for k in (1, 7, 32):
        r = inner.token_logprobs(z, t, top=k)
        assert torch.equal(r.top_index, ref.top(z, k))


@pytest.mark.parametrize("dt", DT)
def test_invalid_values_stay_in_their_row(dt):
    from paper_2607_03011_gb300 import inner
    z, t, gl, ge = make(dt, 6, 5003, 1)
    z[1, 77] = float("nan")
    z[2, 4000] = INF
    z[4] = float("nan")
    r = inner.token_logprobs(z, t, top=8, grad_logp=gl, grad_entropy=ge)
    for i in (1, 2, 4):
        assert torch.isnan(r.lse[i]) and torch.isnan(r.entropy[i]) and torch.isnan(r.logp[i])
        assert torch.isnan(r.grad_logits[i]).any()
    assert ((r.top_index >= 0) & (r.top_index < 5003)).all()
    keep = [0, 3, 5]
    clean = z.clone()  # (the other rows stay at their addresses: the order of their sums goes by those)
    clean[[1, 2, 4]] = 0.0
    sub = inner.token_logprobs(clean, t, top=8, grad_logp=gl, grad_entropy=ge)
    for a, b in zip((r.logp, r.entropy, r.lse, r.top_logp, r.top_index, r.grad_logits), sub):
        assert torch.equal(a[keep], b[keep])


def test_gradient_by_differences():
    from paper_2607_03011_gb300 import inner
    z, t, gl, ge = make(torch.float32, 6, 40, 4)
    r = inner.token_logprobs(z, t, scale=0.5, grad_logp=gl, grad_entropy=ge)

    def f(x):
        e = ref.logprobs(x, t, 0.5)
        return (gl.double() * e["logp"] + ge.double() * e["entropy"]).sum()

    w = torch.randn(6, 40, generator=torch.Generator(device="cuda").manual_seed(8), device="cuda", dtype=torch.float64)
    e = 1e-5
    quot = (f(z.double() + e * w) - f(z.double() - e * w)) / (2 * e)
    # fp32 gradient entries: some tens of roundings each; the quotient itself is good to ~1e-9
    assert abs((r.grad_logits.double() * w).sum() - quot) < 64 * 2.0 ** -23 * r.grad_logits.double().norm() * w.norm() + 1e-8


def test_leading_dimensions_no_rows_and_stream():
    from paper_2607_03011_gb300 import inner
    z, t, gl, ge = make(torch.bfloat16, 12, 520, 6)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    r = inner.token_logprobs(z.view(3, 4, 520), t.view(3, 4), top=3, grad_logp=gl.view(3, 4), stream=s)
    s.synchronize()
    assert r.logp.shape == (3, 4) and r.top_index.shape == (3, 4, 3) and r.grad_logits.shape == (3, 4, 520)
    check_stats(r, z, t, 1.0, 3)
    r0 = inner.token_logprobs(z[:0], t[:0], top=3)
    assert r0.logp.shape == (0,) and r0.top_index.shape == (0, 3)


def test_refusals():
    from paper_2607_03011_gb300 import inner, isoloco
    z, t, gl, ge = make(torch.float32, 4, 40, 2)
    for bad in (lambda: inner.token_logprobs(z.double(), t), lambda: inner.token_logprobs(z, t[:3]),
                lambda: inner.token_logprobs(z, t.float()), lambda: inner.token_logprobs(z, t, top=33),
                lambda: inner.token_logprobs(z, t, top=-1), lambda: inner.token_logprobs(z[:, :4], t, top=5),
                lambda: inner.token_logprobs(z, t, scale=0.0), lambda: inner.token_logprobs(z, t, scale=float("nan")),
                lambda: inner.token_logprobs(z, t, scale=float("inf")), lambda: inner.token_logprobs(z.t(), t),
                lambda: inner.token_logprobs(z, t, grad_logp=gl[:2]), lambda: inner.token_logprobs(z, t, grad_entropy=ge.double()),
                lambda: inner.token_logprobs_grad(z, t, gl[:1], ge, gl, ge),
                lambda: inner.token_logprobs_grad(z, t, gl, None, gl, ge)):
        with pytest.raises((ValueError, isoloco.IsolocoError)):
            bad()
    torch.cuda.synchronize()
