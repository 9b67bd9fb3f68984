"""Distillation from a teacher's top logits against the 64-bit implementation, row by row."""
import math

import pytest
import torch

import teach_ref as ref
from inner_ref import assert_within

pytestmark = pytest.mark.gpu

INF = math.inf
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def make(n, vocab, k, dtype, vdtype=F32, idt=torch.int64, seed=0, missing=0.0, pad=0, distinct=True):
    g = torch.Generator().manual_seed(seed * 1000 + n + vocab + k)
    z = torch.randn(n, vocab + pad, generator=g) * 2.0
    if distinct and k <= vocab:
        ids = torch.stack([torch.randperm(vocab, generator=g)[:k] for _ in range(n)])
    else:
        ids = torch.randint(0, vocab, (n, k), generator=g)
    z[:, :vocab].scatter_add_(1, ids[:, :4], torch.rand(n, min(k, 4), generator=g) * 6)
    v = torch.log_softmax(torch.randn(n, k + 1, generator=g) * 2, 1)[:, :k]
    ids[torch.rand(n, k, generator=g) < missing] = -1
    w = torch.rand(n, generator=g) * 2 - 0.5
    return z.to(dtype), v.to(vdtype), ids.to(idt), w


def check(z, v, ids, w, vocab, scale=1.0, tail="drop", twice=True):
    """Loss alone, loss with gradient, and the gradient by itself, all against the definition."""
    from paper_2607_03011_gb300 import inner
    zc = z.cuda()[:, :vocab]
    vc, ic, wc = v.cuda(), ids.cuda(), w.cuda()
    zr = z[:, :vocab]
    loss, dz = ref.distill(zr, v, ids, scale, tail, w)
    bound = ref.loss_bound(zr, v, scale)
    r = inner.distill(zc, vc, ic, scale=scale, tail=tail, grad_loss=wc, save=True)
    alone = inner.distill(zc, vc, ic, scale=scale, tail=tail)
    assert alone.saved is None and alone.grad_logits is None
    back = inner.distill_grad(wc, zc, vc, ic, r.saved, scale=scale, tail=tail)
    fine = torch.isfinite(loss)
    for got in (r.loss.cpu(), alone.loss.cpu()):
        assert torch.equal(torch.isnan(got), torch.isnan(loss)) and torch.equal(got == INF, loss == INF)
        assert_within(got[fine], loss[fine], bound[fine], "loss")
    for name, d in (("gradient", r.grad_logits), ("gradient by itself", back)):
        assert d.shape == zr.shape and d.dtype == z.dtype
        d = d.cpu()
        assert torch.equal(torch.isnan(d), torch.isnan(dz)), name
        ok = ~torch.isnan(dz)
        assert_within(d[ok], dz[ok], ref.grad_bound(zr, v, ids, scale, w, dz)[ok], name)
    if twice:  # same inputs, same bits
        again = inner.distill(zc, vc, ic, scale=scale, tail=tail, grad_loss=wc, save=True)
        for a, b in zip(r, again):
            assert torch.equal(a.reshape(-1).view(torch.uint8) if a.is_contiguous() else a, b.reshape(-1).view(torch.uint8) if b.is_contiguous() else b)
    return r


SIZES = [(1, 1, 1), (1, 7, 3), (3, 40, 40), (2, 513, 5), (5, 1000, 1), (4, 1003, 33), (9, 4099, 64), (3, 8200, 129), (2, 20011, 256), (2, 33000, 20)]


@pytest.mark.parametrize("tail", ["drop", "rest"])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n,vocab,k", SIZES)
def test_sizes(n, vocab, k, dtype, tail):
    check(*make(n, vocab, k, dtype), vocab, tail=tail)


@pytest.mark.parametrize("vdtype", [F32, BF16, F16])
@pytest.mark.parametrize("idt", [torch.int32, torch.int64])
@pytest.mark.parametrize("tail", ["drop", "rest"])
def test_list_types(vdtype, idt, tail):
    check(*make(6, 777, 12, BF16, vdtype, idt), 777, tail=tail, scale=0.5)


@pytest.mark.parametrize("dtype,vocab,rows", [(F32, 128001, 2), (BF16, 128001, 3), (F16, 262144, 1), (F32, 262147, 1), (BF16, 500000, 2)])
@pytest.mark.parametrize("tail", ["drop", "rest"])
def test_long_rows(dtype, vocab, rows, tail):
    check(*make(rows, vocab, 50, dtype), vocab, tail=tail)


@pytest.mark.parametrize("rows,vocab,dtype", [(330, 50021, F16), (170, 80003, BF16), (170, 40000, F32)])
def test_many_rows_of_several_ctas(rows, vocab, dtype):
    check(*make(rows, vocab, 6, dtype, missing=0.3), vocab, tail="rest", twice=False)


def test_rows_beyond_shared_memory():
    check(*make(2, 1200001, 9, F32), 1200001, tail="rest", twice=False)


@pytest.mark.parametrize("rows", [1, 151, 153, 700])
@pytest.mark.parametrize("vocab", [64, 1001, 5003])
def test_many_rows(rows, vocab):
    check(*make(rows, vocab, 8, BF16, missing=0.3), vocab, tail="rest")


@pytest.mark.parametrize("pad", [0, 1, 3, 8])
@pytest.mark.parametrize("offset", [0, 1, 5])
@pytest.mark.parametrize("dtype", [F32, F16])
def test_pitches_and_offsets(pad, offset, dtype):
    vocab = 901
    z, v, ids, w = make(7, vocab, 11, dtype, pad=pad + offset)
    from paper_2607_03011_gb300 import inner
    part = z.cuda()[:, offset:offset + vocab]
    zr = z[:, offset:offset + vocab]
    # lists in the columns of wider tensors, too
    wide_v, wide_i = torch.zeros(7, 17).cuda(), torch.full((7, 13), 3).cuda()
    wide_v[:, 2:13], wide_i[:, 1:12] = v.cuda(), ids.cuda()
    r = inner.distill(part, wide_v[:, 2:13], wide_i[:, 1:12], tail="rest", grad_loss=w.cuda())
    loss, dz = ref.distill(zr, v, ids, 1.0, "rest", w)
    assert_within(r.loss.cpu(), loss, ref.loss_bound(zr, v, 1.0), "loss")
    assert_within(r.grad_logits.cpu(), dz, ref.grad_bound(zr, v, ids, 1.0, w, dz), "gradient")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", [4096, 4101, 50001, 70000, 80001])
def test_gradient_over_the_logits_and_elsewhere(dtype, vocab):
    """Through the C entry point: the gradient over the logits themselves, and into rows of another alignment whose
    neighbours stay as they are."""
    from paper_2607_03011_gb300 import inner, isoloco
    z, v, ids, w = make(5, vocab, 16, dtype, missing=0.2)
    zc, vc, ic, wc = z.cuda(), v.cuda(), ids.cuda(), w.cuda()
    want = inner.distill(zc, vc, ic, grad_loss=wc, tail="rest")
    L, code, loss = isoloco.lib(), inner._DTYPE[dtype], torch.empty(5, device="cuda")

    def call(out, ld):
        rc = L.isoloco_distill(zin.data_ptr(), vocab, code, 5, vocab, vc.data_ptr(), 16, 0, ic.data_ptr(), 16, 8, 16, 1.0, 1,
                               loss.data_ptr(), None, wc.data_ptr(), out.data_ptr(), ld, torch.cuda.current_stream().cuda_stream)
        assert rc == 0, isoloco.last_error()

    zin = zc
    for shift in (1, 2, 3):
        wide = torch.full((5 * (vocab + 5) + 8,), 7.0, dtype=dtype, device="cuda")
        call(wide[shift:], vocab + 5)
        rows = wide[shift:shift + 5 * (vocab + 5)].view(5, vocab + 5)
        assert torch.equal(rows[:, :vocab], want.grad_logits) and (rows[:, vocab:] == 7.0).all() and (wide[:shift] == 7.0).all()
    zin = zc.clone()
    call(zin, vocab)
    assert torch.equal(zin, want.grad_logits) and torch.equal(loss, want.loss)


@pytest.mark.parametrize("tail", ["drop", "rest"])
def test_the_same_token_twice(tail):
    z, v, ids, w = make(8, 600, 40, BF16, seed=2)
    ids[0] = 5                      # all of them
    ids[1, 20:] = ids[1, :20]       # in pairs, far apart
    ids[2, 1::2] = ids[2, 0::2]     # side by side
    ids[3] = torch.randint(0, 4, (40,))
    if tail == "rest":
        v = v - 3.0
    check(z, v, ids, w, 600, tail=tail)


@pytest.mark.parametrize("tail", ["drop", "rest"])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_masks_and_empty_rows(dtype, tail):
    z, v, ids, w = make(14, 300, 10, dtype, seed=4)
    low = ref.LOWEST[dtype]
    ids[0] = -1                                    # no list
    ids[1] = 300                                   # the first index past the vocabulary
    ids[2, :9] = torch.tensor([-5, 301, 2 ** 40, -2 ** 40, 10 ** 9, 400, -1, -1, 999])
    z[3] = -INF                                    # nothing is left of the row
    z[4] = low
    z[5, ids[5, 0]] = -INF                         # a token of the list is masked
    z[6, ids[6, 1]] = low
    m = torch.ones(300, dtype=torch.bool)
    m[ids[7]] = False
    z[7, m] = -INF                                 # nothing but the list is left
    z[8, m.scatter(0, ids[8], False)] = low
    v[9] = -INF                                    # entries without weight
    v[10, 1:] = -INF
    z[11, ids[11]] = -INF                          # nothing but other tokens is left
    z[12, ::2] = -INF
    z[13, 50:] = low
    check(z, v, ids, w, 300, tail=tail)


@pytest.mark.parametrize("tail", ["drop", "rest"])
def test_nan_and_infinities(tail):
    z, v, ids, w = make(12, 200, 6, F32, seed=5)
    other = [j for j in range(200) if j not in ids[1].tolist()][0]
    z[0, ids[0, 2]] = math.nan
    z[1, other] = math.nan
    z[2, ids[2, 0]] = INF
    z[3, [j for j in range(200) if j not in ids[3].tolist()][7]] = INF
    v[4, 3] = math.nan
    v[5, 1] = INF
    v[6, 2], ids[6, 2] = math.nan, -1              # an entry that is not there
    z[7], ids[7] = math.nan, -1                    # a row without a list
    z[8] = -INF
    z[8, [j for j in range(200) if j not in ids[8].tolist()][3]] = math.nan
    z[9] = math.nan
    v[10] = -INF
    z[10, 0] = math.nan
    check(z, v, ids, w, 200, tail=tail)


def test_a_sure_student():
    """The others' share of the student is far below what a difference of sums could hold."""
    z, v, ids, w = make(6, 500, 4, F32, seed=6)
    for r, gap in enumerate((10.0, 20.0, 40.0, 80.0, 120.0, 300.0)):
        z[r] -= gap
        z[r, ids[r]] += gap
    check(z, v, ids, w, 500, tail="rest")


@pytest.mark.parametrize("scale", [0.05, 1.0, 7.0])
def test_large_logits_and_scales(scale):
    z, v, ids, w = make(4, 900, 7, F32, seed=7)
    z[0] = z[0] * 1e4
    z[1] = z[1] + 3e6
    z[2] = z[2] * 1e-6
    check(z, v, ids, w, 900, tail="drop", scale=scale)


def test_gradient_against_differences():
    """The kernel's gradient against differences of the definition in 64 bits, in some entries of every row."""
    from paper_2607_03011_gb300 import inner
    z, v, ids, w = make(4, 50, 5, F32, seed=8)
    d = inner.distill(z.cuda(), v.cuda(), ids.cuda(), tail="rest", grad_loss=w.cuda()).grad_logits.cpu().double()
    for r in range(4):
        for j in (int(ids[r, 0]), 0, 49):
            h = 1e-3  # (z stays in fp32, where a step of 1e-3 is good to 2e-4 of itself)
            up, down = z.clone(), z.clone()
            up[r, j] += h
            down[r, j] -= h
            step = up[r, j].double() - down[r, j].double()
            diff = (ref.distill(up, v, ids, 1.0, "rest") - ref.distill(down, v, ids, 1.0, "rest"))[r] / step * w[r].double()
            # third derivatives of a log sum are below 1: h^2 / 6 of them
            assert abs(diff.item() - d[r, j].item()) <= 2 * h * h / 6 + 1e-6


def test_leading_dimensions_and_no_rows():
    from paper_2607_03011_gb300 import inner
    z, v, ids, w = make(6, 100, 4, BF16, seed=9)
    flat = inner.distill(z.cuda(), v.cuda(), ids.cuda(), grad_loss=w.cuda())
    deep = inner.distill(z.cuda().view(2, 3, 100), v.cuda().view(2, 3, 4), ids.cuda().view(2, 3, 4), grad_loss=w.cuda().view(2, 3))
    assert deep.loss.shape == (2, 3) and deep.grad_logits.shape == (2, 3, 100)
    assert torch.equal(deep.loss.view(-1), flat.loss) and torch.equal(deep.grad_logits.view(6, 100), flat.grad_logits)
    none = inner.distill(z.cuda()[:0], v.cuda()[:0], ids.cuda()[:0], grad_loss=w.cuda()[:0], save=True)
    assert none.loss.shape == (0,) and none.grad_logits.shape == (0, 100)
    assert inner.distill_grad(w.cuda()[:0], z.cuda()[:0], v.cuda()[:0], ids.cuda()[:0], none.saved).shape == (0, 100)


def test_refusals():
    from paper_2607_03011_gb300 import inner
    z, v, ids, w = (t.cuda() for t in make(4, 100, 6, BF16))
    r = inner.distill(z, v, ids, save=True)
    for args, kw in [((z.double(), v, ids), {}), ((z.cpu(), v, ids), {}), ((z, v.cpu(), ids), {}), ((z, v, ids.cpu()), {}),
                     ((z, v, ids.float()), {}), ((z, v[:3], ids), {}), ((z, v, ids[:, :5]), {}), ((z, v[:, :0], ids[:, :0]), {}),
                     ((z, v, ids), dict(tail="all")), ((z, v, ids), dict(grad_loss=w[:3])), ((z, v, ids), dict(grad_loss=w.half())),
                     ((z.t(), v, ids), {}), ((z, v.t().contiguous().t(), ids), {}),
                     ((z, v.repeat(1, 50), ids.repeat(1, 50)), {})]:
        with pytest.raises(ValueError):
            inner.distill(*args, **kw)
    for scale in (0.0, -1.0, math.nan, INF):
        with pytest.raises(inner.IsolocoError):
            inner.distill(z, v, ids, scale=scale)
    for saved in (r.saved[:3], r.saved.half(), r.saved.cpu()):
        with pytest.raises(ValueError):
            inner.distill_grad(w, z, v, ids, saved)
    with pytest.raises(ValueError):
        inner.distill_grad(None, z, v, ids, r.saved)
