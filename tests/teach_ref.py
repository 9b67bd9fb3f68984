"""Plain 64-bit implementations of distillation from top logits and of a beam search's selection, from their
formulas, and the bounds that the tests hold the kernels to."""
import math

import torch

from inner_ref import U

LOWEST = {torch.float32: torch.finfo(torch.float32).min, torch.bfloat16: torch.finfo(torch.bfloat16).min,
          torch.float16: torch.finfo(torch.float16).min}
INF = math.inf


def masked(z):
    """Logits in 64 bits, masked ones -inf."""
    x = z.double()
    return torch.where(x <= LOWEST[z.dtype], torch.full_like(x, -INF), x)


def distill(z, v, ids, scale, tail, g=None):
    """loss and (with g) the gradient by the logits, row by row from the definitions."""
    x, v = masked(z), v.double()
    n, vocab = x.shape
    loss = torch.zeros(n, dtype=torch.float64)
    dz = torch.zeros(n, vocab, dtype=torch.float64)
    for r in range(n):
        here = [(int(ids[r, e]), v[r, e].item()) for e in range(ids.shape[1]) if 0 <= int(ids[r, e]) < vocab]
        if not here:
            continue
        tokens = torch.tensor([t for t, _ in here])
        w = torch.tensor([a for _, a in here], dtype=torch.float64)
        bad = bool(torch.isnan(x[r]).any() or (x[r] == INF).any() or torch.isnan(w).any() or (w == INF).any())
        if tail == "drop" and (w == -INF).all():
            continue
        if bad:
            loss[r] = math.nan
            dz[r] = math.nan
            continue
        outside = torch.ones(vocab, dtype=torch.bool)
        outside[tokens] = False
        logq = w - torch.logsumexp(w, 0) if tail == "drop" else w
        q = logq.exp()
        zz = x[r] * scale
        lse = torch.logsumexp(zz, 0)
        others = torch.logsumexp(zz[outside], 0) if outside.any() else torch.tensor(-INF, dtype=torch.float64)
        rest = max(0.0, 1.0 - q.sum().item()) if tail == "rest" and others > -INF else 0.0
        if lse == -INF:
            loss[r] = INF if q.sum() > 0 else 0.0
            continue
        lp = zz - lse
        total = sum(a.item() * (b.item() - lp[t].item()) for a, b, t in zip(q, logq, tokens) if a > 0)
        if rest > 0:
            total += rest * (math.log(rest) - (others - lse).item())
        loss[r] = total
        d = lp.exp() * (q.sum() + rest)
        if rest > 0:
            d[outside] -= rest * (zz[outside] - others).exp()
        d.index_put_((tokens,), -q, accumulate=True)
        dz[r] = d * scale
    return (loss, dz * g.double()[:, None]) if g is not None else loss


# How far the kernels may be off.  An exponent d = (x - m) c, in units of ln 2, carries the roundings of the difference, of
# c and of the product: 3 * 2^-24 |d|, so the power 2^d is off by (3 * 2^-24 ln 2 |d| + 2^-22) of itself, the latter by its
# own approximation.  |d| 2^d is at most 0.54, and a sum of powers about its largest is at least 1: together with the additions' own
# roundings (in chains of at most 8 + length / 64, of positive terms) a sum is off by less than SUM(length) of itself.
def sum_of_powers(length):
    return 2.0 ** -20 + (8 + length / 64) * 2.0 ** -24


def _size(z, v, scale):
    """The largest magnitude that a logarithm in a row's loss may have: the logits' range, the list's, and 32 for the rest."""
    x = masked(z) * scale
    fine = torch.isfinite(x)
    hi = torch.where(fine, x, torch.full_like(x, -1e300)).amax(1)
    lo = torch.where(fine, x, torch.full_like(x, 1e300)).amin(1)
    return (hi - lo).clamp_min(0.0) + torch.nan_to_num(v.double(), nan=0.0, posinf=0.0, neginf=0.0).abs().amax(1) + 32


def loss_bound(z, v, scale):
    """q (ln q - z + lse), summed over k entries and the rest: each factor q and 1 - sum q is off by (8 + k) 2^-24 of 1 in sum, each logarithm by
    a few roundings of its size, the log of a sum by the sum's share."""
    k, vocab = v.shape[1], z.shape[1]
    return (16 + k) * 2.0 ** -24 * _size(z, v, scale) + 4 * sum_of_powers(vocab)


def grad_bound(z, v, ids, scale, g, dz):
    """An entry is a difference p Q - q, or p Q - r p / P: each part is off by its factors' share of itself (powers and sums of them; for q also the
    rounding of its exponent, of the list's size), and r by (8 + k) 2^-24 of 1.  Each part is at most the difference and twice the smaller part, p Q.
    A power below 2^-126, fp32's smallest normal number, counts as 0; what it is multiplied by is at most 1.01 w (sums are at least 1)."""
    k, vocab = v.shape[1], z.shape[1]
    x = masked(z) * scale
    none = (x.amax(1, keepdim=True) == -INF) | torch.isnan(x).any(1, keepdim=True) | (x == INF).any(1, keepdim=True)
    p = torch.softmax(torch.where(none, torch.zeros_like(x), x), 1)
    outside = torch.ones(x.shape[0], vocab + 1, dtype=torch.float64)
    outside.scatter_(1, torch.where((ids >= 0) & (ids < vocab), ids.long(), torch.full_like(ids.long(), vocab)), 0.0)
    po = p * outside[:, :vocab]
    share = po / po.sum(1, keepdim=True).clamp_min(1e-300)
    w = scale * g.double().abs()[:, None]
    rel = 4 * sum_of_powers(vocab) + (_size(z, v, scale)[:, None] + 16 + k) * 2.0 ** -23
    return torch.where(none, torch.full_like(p, 0.0), rel * (torch.nan_to_num(dz).abs() + 2 * w * p * 1.01) + (8 + k) * 2.0 ** -23 * w * share + 1.01 * w * 2.0 ** -126)


def select(z, scores, keep, finished=None, end=None, scale=1.0):
    """(totals, beams, tokens) of each batch entry, from a full ranking."""
    b, w, vocab = z.shape
    out = ([], [], [])
    for i in range(b):
        rows = []
        for j in range(w):
            c = scores[i, j].double().item()
            raw, x = z[i, j].double(), masked(z[i, j])
            done = finished is not None and bool(finished[i, j])
            bad = math.isnan(c) or c == INF or (c != -INF and not done and bool(torch.isnan(raw).any() or (raw == INF).any()))
            if bad or c == -INF or (not done and bool((x == -INF).all())):
                rows += [(-INF, j, 0.0, t, bad) for t in range(min(keep, vocab))]
            elif done:
                rows += [(c if t == end else -INF, j, 0.0, t, False) for t in sorted({*range(min(keep + 1, vocab)), end})]
            else:
                lse = torch.logsumexp(x * scale, 0)
                total = c + (x * scale - lse)
                order = torch.sort(raw, descending=True, stable=True).indices[:keep]
                rows += [(total[t].item(), j, raw[t].item() + 0.0, t.item(), False) for t in order]
        rows.sort(key=lambda e: (-e[0], e[1], -e[2], e[3]))
        rows = rows[:keep]
        out[0].append([math.nan if e[4] else e[0] for e in rows])
        out[1].append([e[1] for e in rows])
        out[2].append([e[3] for e in rows])
    return (torch.tensor(out[0], dtype=torch.float64), torch.tensor(out[1]), torch.tensor(out[2]))


def reorder(s, beams):
    """state[b, beams[b, w]] of a state whose first two dimensions are batch and beams."""
    b, w = beams.shape
    own = torch.arange(w).expand(b, w)
    src = torch.where((beams >= 0) & (beams < w), beams.long(), own)
    return torch.stack([s[i, src[i]] for i in range(b)])
