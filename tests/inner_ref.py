"""Plain 64-bit implementations of the inner step's operators, from their formulas, and the bounds
the tests hold the kernels to.

U[dtype] is half the spacing of the type's numbers relative to their size: one rounding changes a value
by at most U |value| (plus half the smallest subnormal).  A sum of n products held in fp32, in any
order, is off by at most (n + 8) 2^-23 times the sum of the products' magnitudes: 2^-24 per
addition for rounding to nearest, 2^-23 where the tensor core truncates instead.
"""
import torch

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}


def sum_err(n):
    return (n + 8) * 2.0 ** -23


def assert_within(got, exact, bound, what=""):
    """|got - exact| <= bound + one rounding to got's type, entry by entry."""
    g = got.double()
    lim = bound + U[got.dtype] * (exact.abs() + bound) + TINY[got.dtype]
    bad = ~((g - exact).abs() <= lim)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst by " \
                          f"{((g - exact).abs() / lim).nan_to_num(nan=float('inf')).max().item():.3g} of the bound"


def rel(got, exact):
    return ((got.double() - exact).norm() / exact.norm().clamp_min(1e-300)).item()


def embed_grad(dy, ids, vocab, scale):
    ids = ids.reshape(-1)
    ok = (ids >= 0) & (ids < vocab)
    dw = torch.zeros(vocab, dy.shape[-1], dtype=torch.float64, device=dy.device)
    mag = torch.zeros_like(dw)
    cnt = torch.zeros(vocab, dtype=torch.float64, device=dy.device)
    d = dy.reshape(-1, dy.shape[-1]).double()[ok] * scale
    dw.index_put_((ids[ok].long(),), d, accumulate=True)
    mag.index_put_((ids[ok].long(),), d.abs(), accumulate=True)
    cnt.index_put_((ids[ok].long(),), torch.ones(int(ok.sum()), dtype=torch.float64, device=dy.device), accumulate=True)
    return dw, sum_err(cnt)[:, None] * mag


def act(g, kind):
    """(value, first derivative); the second derivative of both is below 1 in magnitude, the first
    below 1.2."""
    if kind == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    c = (2 / torch.pi) ** 0.5
    t = torch.tanh(c * (g + 0.044715 * g ** 3))
    return g * (1 + t) / 2, (1 + t) / 2 + g / 2 * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)


def gated_ffn(x, wg, wu, kind, dh=None):
    """h with its bound; with dh also dx, dwg, dwu with theirs (dict name -> (exact, bound))."""
    x, wg, wu, u16 = x.double(), wg.double(), wu.double(), U[x.dtype]
    k = x.shape[1]
    g, u = x @ wg, x @ wu
    eg, eu = sum_err(k) * (x.abs() @ wg.abs()), sum_err(k) * (x.abs() @ wu.abs())
    a, s = act(g, kind)
    # the activation itself is good to a few units in fp32
    ea = 1.2 * eg + 16 * 2.0 ** -24 * (a.abs() + g.abs() * 2.0 ** -10 + 2.0 ** -10)
    out = {"h": (a * u, ea * (u.abs() + eu) + a.abs() * eu + 2.0 ** -23 * (a * u).abs())}
    if dh is None:
        return out
    dh = dh.double()
    # g and u are kept rounded; dg and du are rounded once more (subnormals: TINY)
    eg, eu = eg + u16 * (g.abs() + eg), eu + u16 * (u.abs() + eu)
    dg, du = dh * u * s, dh * a
    edg = dh.abs() * (eu * 1.2 + (u.abs() + eu) * (eg + 16 * 2.0 ** -24))
    edu = dh.abs() * (1.2 * eg + 16 * 2.0 ** -24 * (a.abs() + 2.0 ** -10))
    tiny = TINY[torch.float16] if u16 == U[torch.float16] else 0.0
    edg, edu = edg + u16 * (dg.abs() + edg) + tiny, edu + u16 * (du.abs() + edu) + tiny
    n, f = x.shape[0], wg.shape[1]
    mg, mu = dg.abs() + edg, du.abs() + edu
    out["dx"] = (dg @ wg.T + du @ wu.T,
                 edg @ wg.abs().T + edu @ wu.abs().T + sum_err(2 * f) * (mg @ wg.abs().T + mu @ wu.abs().T))
    out["dwg"] = (x.T @ dg, x.abs().T @ edg + sum_err(n) * (x.abs().T @ mg))
    out["dwu"] = (x.T @ du, x.abs().T @ edu + sum_err(n) * (x.abs().T @ mu))
    return out


def logprobs(z, targets, scale):
    """Dict of exact logp, entropy, lse, p, lp (rows of -inf alone as the entry point says)."""
    v = z.shape[1]
    x = z.double() * scale
    m = x.amax(1, keepdim=True)
    none = (m == -float("inf"))
    e = torch.exp(x - torch.where(none, torch.zeros_like(m), m))
    s = e.sum(1, keepdim=True)
    lse = torch.where(none, m, m + torch.log(s))
    lp = torch.where(none, torch.full_like(x, -float("inf")), (x - m) - torch.log(s))  # (lse alone may have lost log s)
    p = torch.where(none, torch.zeros_like(x), e / s)
    ent = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(1)
    given = (targets >= 0) & (targets < v)
    t = targets.long().clamp(0, v - 1)
    logp = torch.where(given, lp.gather(1, t[:, None])[:, 0], torch.zeros_like(ent))
    return dict(logp=logp, entropy=ent, lse=lse[:, 0], p=p, lp=lp, given=given, t=t, none=none[:, 0])


def logprobs_grad(r, scale, gl, ge):
    d = torch.zeros_like(r["p"])
    if gl is not None:
        g = torch.where(r["given"], gl.double(), torch.zeros_like(r["logp"]))[:, None]
        d -= g * r["p"]
        d.scatter_add_(1, r["t"][:, None], g)
    if ge is not None:
        h = torch.where(r["p"] > 0, r["lp"] + r["entropy"][:, None], torch.zeros_like(r["p"]))
        d -= ge.double()[:, None] * r["p"] * h
    d[r["none"]] = 0.0
    return d * scale


def top(z, k):
    """Indices of the k largest, the lowest index first among equals."""
    return torch.sort(z.double(), dim=1, descending=True, stable=True).indices[:, :k]
