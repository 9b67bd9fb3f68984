"""Token log probabilities: every entry of a row counts.  Rows whose result changes by far more than the bounds
if any one entry is left out, at the sizes where rows are cut into vectors, batches, threads' and CTAs' shares."""
import math

import pytest
import torch

import inner_ref as ref
from test_gpu_token_logprobs import check_grad, make

pytestmark = pytest.mark.gpu
DT = [torch.float32, torch.bfloat16, torch.float16]
# rows at once: clusters of 8, 4 and 2 CTAs per row, and one CTA per row (where the row is long enough)
ROWS = [1, 19, 38, 76, 200]
WIDE = [1, 7, 64, 65, 515, 1023, 4096, 5003, 8192, 8193, 16385, 33001, 50021, 128003, 300007]


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("v", WIDE)
def test_equal_entries(dt, v):
    """A row of equal logits: the exponentials are 1 exactly and their sum v exactly (below 2^24), so that the
    entropy is logf(v), good to one unit in the last place (at most 2^-23 relative), and the log probability minus
    that.  One entry left out changes either by 1 / v, more than twice as much at every size here."""
    from paper_2607_03011_gb300 import inner
    ln = math.log(v)
    bound = 2.0 ** -23 * ln
    assert v == 1 or 1.0 / v > 2 * bound
    for n in ROWS:
        for c, off in ((0.0, 0), (2.5, 3), (-3.0, 1)):
            z = torch.full((n, v + off), c, device="cuda", dtype=dt)[:, off:]
            t = torch.arange(n, device="cuda") * 7919 % v
            for top in (0, min(3, v)):
                r = inner.token_logprobs(z, t, top=top, grad_logp=torch.ones(n, device="cuda"))
                assert ((r.entropy.double() - ln).abs() <= bound).all(), (n, c, top)
                assert ((r.logp.double() + ln).abs() <= bound).all(), (n, c, top)
                # c + ln v rounded once more
                assert ((r.lse.double() - (c + ln)).abs() <= bound + 2.0 ** -24 * abs(c + ln) + 2.0 ** -30).all()
                if top:
                    assert torch.equal(r.top_index, torch.arange(top, device="cuda").expand(n, top))
                exact = torch.full((n, v), -1.0 / v, device="cuda", dtype=torch.float64)
                exact.scatter_add_(1, t[:, None], torch.ones(n, 1, device="cuda", dtype=torch.float64))
                # 1 / s and its product with the gradient: a few roundings
                ref.assert_within(r.grad_logits, exact, 8 * 2.0 ** -24 * exact.abs() + (8 * 2.0 ** -24 if v > 1 else 2.0 ** -22) / v)


def positions(v):
    """Places where a share, a batch of vectors, a vector or the row's head and tail begin and end, and others."""
    if v <= 5003:
        return torch.arange(v)
    at = [torch.arange(300), v - 1 - torch.arange(300)]
    edge = []
    for split in (2, 4, 8):
        per = (-(-v // split) + 63) // 64 * 64
        edge += [per * k for k in range(1, split)]
    for threads in (64, 128, 256):
        for per_vec in (4, 8):
            edge += list(range(0, v, threads * per_vec * 4))[:40] + [v // (threads * per_vec * 4) * threads * per_vec * 4]
    e = torch.tensor(edge)
    at += [e + d for d in range(-9, 10)]
    at.append(torch.randint(0, v, (500,), generator=torch.Generator().manual_seed(v)))
    at = torch.unique(torch.cat(at))
    return at[(at >= 0) & (at < v)]


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("v", [64, 515, 5003, 33001, 50021, 128003])
@pytest.mark.parametrize("rows", [1, 19, 76, 100000])
def test_one_entry_holds_the_mass(dt, v, rows):
    """All logits -20 but one of 10: its probability is 1 to 1e-7 (v e^-30 in all for the others, 1.2e-8 at most), so
    the results are lse 10, log probability 0 and entropy 0 to 1e-5, where a row without it gives -20 + ln v."""
    from paper_2607_03011_gb300 import inner
    js = positions(v).cuda()
    if rows < 100:
        js = js[torch.randperm(len(js), generator=torch.Generator().manual_seed(rows))[:rows * 40].cuda()]
    for part in js.split(min(rows, 2000)):
        n = len(part)
        z = torch.full((n, v), -20.0, device="cuda", dtype=dt)
        z.scatter_(1, part[:, None], 10.0)
        other = (part + v // 2) % v
        gl = torch.ones(n, device="cuda")
        for top in (0, 2):
            r = inner.token_logprobs(z, part, top=top)
            assert ((r.lse - 10).abs() < 1e-5).all() and (r.logp.abs() < 1e-5).all() and (r.entropy.abs() < 1e-5).all()
            if top:
                assert torch.equal(r.top_index[:, 0], part) and torch.equal(r.top_index[:, 1], (part == 0).long())
            # the gradient of the log probability of another token: 1 there, -1 at the entry, 0 elsewhere
            r = inner.token_logprobs(z, other, top=top, grad_logp=gl)
            d = inner.token_logprobs_grad(z, other, r.lse, r.entropy, gl, None)
            for g in (r.grad_logits, d):
                want = torch.zeros(n, v, device="cuda")
                want.scatter_(1, other[:, None], 1.0)
                want.scatter_(1, part[:, None], -1.0)
                assert (g.float() - want).abs().max() < 1e-5


def tight(v, e):
    """What the kernel's own order of summation can be off by: a thread adds at most v / 64 entries (64 threads at least
    up to 8192 entries, 128 up to 16384 and with alternatives, else 256; two sums each), so v / 128 additions, and at most
    20 more in the merges, each 2^-24; an exponential is good to 2^-22, and its argument, of three roundings, to
    2^-22 |d| (|d| on average below log2 v + 1); a running maximum that rises multiplies by one more such power, some
    ten times in a thread and three in the merges."""
    depth = v / 128 + 20
    base = depth * 2.0 ** -24 + 16 * 2.0 ** -22 + (math.log2(v) + 1) * 2.0 ** -22
    return base + 4 * 2.0 ** -24 * (1 + e["lse"].abs())


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("n,v", [(3, 1000), (200, 1003), (3, 8192), (300, 8200), (200, 16385), (2, 32000), (200, 32000), (3, 50021),
                                 (200, 50021), (1, 128003), (160, 128003), (2, 300007), (160, 300007)])
def test_random_rows(dt, n, v):
    """Statistics and gradient to a few 1e-5: a thread's share left out changes a row's lse by some 4e-3."""
    from paper_2607_03011_gb300 import inner
    z, t, gl, ge = make(dt, n, v, 3 * n + v)
    e = ref.logprobs(z, t, 1.0)
    base = tight(v, e)
    for top in (0, 5):
        r = inner.token_logprobs(z, t, top=top, grad_logp=gl, grad_entropy=ge)
        # of the target's logit: z - lse, with a rounding of each part
        assert ((r.lse.double() - e["lse"]).abs() <= base).all(), ((r.lse.double() - e["lse"]).abs() / base).max()
        assert ((r.logp.double() - e["logp"]).abs() <= base + 2.0 ** -22 * e["logp"].abs()).all()
        # w / s: both sums' errors times the mean |d|, at most log v, once each
        assert ((r.entropy.double() - e["entropy"]).abs() <= base * (3 + 2 * math.log(v))).all()
        check_grad(r.grad_logits, e, 2 * base, 1.0, gl, ge)
    d = inner.token_logprobs_grad(z, t, r.lse, r.entropy, gl, ge)
    check_grad(d, e, 4 * base, 1.0, gl, ge)


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("n,v,pad", [(1, 5, 0), (300, 515, 0), (300, 1003, 5), (2, 32000, 0), (3, 50021, 0), (200, 50021, 3),
                                     (2, 300007, 0)])
def test_gradient_over_the_logits(dt, n, v, pad):
    """grad_logits may be the logits themselves: the bits that a buffer of its own gets."""
    from paper_2607_03011_gb300 import isoloco
    z, t, gl, ge = make(dt, n, v, n + v, pad)
    own = torch.empty(n, v + pad, dtype=dt, device="cuda")[:, :v]
    code = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}[dt]
    out = []
    for top in (0, min(4, v)):
        for grad in (own, z.clone() if not pad else torch.empty_like(own.new_empty(n, v + pad))[:, :v].copy_(z)):
            src = z if grad is own else grad
            s = [torch.empty(n, device="cuda") for _ in range(3)]
            tl, ti = torch.empty(n, max(top, 1), device="cuda"), torch.empty(n, max(top, 1), device="cuda", dtype=torch.int64)
            rc = isoloco.lib().isoloco_token_logprobs(src.data_ptr(), v + pad, code, n, v, t.data_ptr(), 8, 1.0, *(q.data_ptr() for q in s),
                                                      top, tl.data_ptr(), ti.data_ptr(), gl.data_ptr(), ge.data_ptr(), grad.data_ptr(),
                                                      v + pad, torch.cuda.current_stream().cuda_stream)
            assert rc == isoloco.OK
            out.append([grad.clone(), *s] + ([tl, ti] if top else []))
        assert all(torch.equal(a, b) for a, b in zip(out[-2], out[-1]))
