"""Gated feed-forward block and its gradient against plain 64-bit products, and by differences."""
import pytest
import torch

import inner_ref as ref

pytestmark = pytest.mark.gpu
DT = [torch.bfloat16, torch.float16]

# (tokens, width, ff): one token, a few, tile edges crossed by one, widths that are no multiple of 8
SIZES = [(1, 64, 64), (1, 1024, 2816), (2, 8, 8), (3, 130, 70), (5, 513, 1000), (8, 256, 520), (9, 256, 520), (17, 2048, 384),
         (33, 1024, 264), (64, 72, 136), (127, 320, 136), (129, 64, 264), (257, 512, 392), (300, 1000, 129), (300, 129, 1000),
         (513, 264, 776), (1, 1, 1), (260, 7, 5), (2048, 256, 512), (700, 1032, 1544)]


def operands(dt, n, d, f, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(n, d, generator=g, device="cuda").to(dt)
    wg = (torch.randn(d, f, generator=g, device="cuda") / d ** 0.5).to(dt)
    wu = (torch.randn(d, f, generator=g, device="cuda") / d ** 0.5).to(dt)
    dh = torch.randn(n, f, generator=g, device="cuda").to(dt)
    return x, wg, wu, dh


def check(got, x, wg, wu, dh, kind):
    r = ref.gated_ffn(x, wg, wu, kind, dh)
    u16 = ref.U[x.dtype]
    for name, v in got.items():
        exact, bound = r[name]
        ref.assert_within(v, exact, bound, f"{name} {tuple(x.shape)} x {wg.shape[1]}")
        # roundings are independent: the output's, and for gradients those of g, u and dg or du, each
        # below U; together below 4 U in the norm (fp32 sums add far less)
        if exact.numel() >= 64:
            assert ref.rel(v, exact) < 4 * u16, name


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("n,d,f", SIZES)
def test_forward_and_backward(dt, n, d, f):
    from paper_2607_03011_gb300 import inner, isoloco
    kind = "silu" if (n + d + f) % 2 == 0 else "gelu_tanh"
    x, wg, wu, dh = operands(dt, n, d, f, n + d + f)
    h = inner.gated_ffn(x, wg, wu, act=kind)
    h2, saved = inner.gated_ffn(x, wg, wu, act=kind, save=True)
    dx, dwg, dwu = inner.gated_ffn_grad(dh, x, wg, wu, saved, act=kind)
    check({"h": h, "dx": dx, "dwg": dwg, "dwu": dwu}, x, wg, wu, dh, kind)
    check({"h": h2}, x, wg, wu, dh, kind)
    again = inner.gated_ffn_grad(dh, x, wg, wu, saved, act=kind)
    assert all(torch.equal(a, b) for a, b in zip(again, (dx, dwg, dwu)))
    assert inner.status() == isoloco.OK


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("kind", ["silu", "gelu_tanh"])
def test_one_token_is_a_row_of_the_batch(dt, kind):
    """Serving a token by itself gives what the batch gives, to the roundings of either."""
    from paper_2607_03011_gb300 import inner
    x, wg, wu, _ = operands(dt, 40, 264, 528, 11)
    r = ref.gated_ffn(x, wg, wu, kind)["h"]
    for n in (1, 2, 3, 4, 7, 8, 12, 16, 24, 40):
        h = inner.gated_ffn(x[:n], wg, wu, act=kind)
        ref.assert_within(h, r[0][:n], r[1][:n], f"{n} tokens")


@pytest.mark.parametrize("dt", DT)
def test_strides_and_offsets(dt):
    """Rows with a pitch, weights that are columns of a wider matrix, addresses off 16 bytes."""
    from paper_2607_03011_gb300 import inner
    for n, d, f, pad, off in ((70, 128, 192, 8, 8), (70, 128, 192, 5, 3), (1, 128, 192, 5, 1), (300, 256, 264, 24, 16)):
        x, wg, wu, dh = operands(dt, n, d, f, 7)
        xs = torch.zeros(n, d + pad, device="cuda", dtype=dt)[:, :d]
        xs.copy_(x)
        ws = torch.zeros(d, 2 * f + pad + off, device="cuda", dtype=dt)
        a, b = ws[:, off:off + f], ws[:, off + f:off + 2 * f]
        a.copy_(wg), b.copy_(wu)
        dhs = torch.zeros(n, f + pad, device="cuda", dtype=dt)[:, pad:]
        dhs.copy_(dh)
        h, saved = inner.gated_ffn(xs, a, b, save=True)
        dx, dwg, dwu = inner.gated_ffn_grad(dhs, xs, a, b, saved)
        check({"h": h, "dx": dx, "dwg": dwg, "dwu": dwu}, x, wg, wu, dh, "silu")


def test_parts_of_the_gradient_leading_dimensions_and_no_tokens():
    from paper_2607_03011_gb300 import inner
    x, wg, wu, dh = operands(torch.bfloat16, 60, 64, 128, 3)
    _, saved = inner.gated_ffn(x, wg, wu, save=True)
    dx, dwg, dwu = inner.gated_ffn_grad(dh, x, wg, wu, saved)
    a = inner.gated_ffn_grad(dh, x, wg, wu, saved, need_w=False)
    b = inner.gated_ffn_grad(dh, x, wg, wu, saved, need_x=False)
    assert torch.equal(a[0], dx) and a[1] is None and a[2] is None
    assert b[0] is None and torch.equal(b[1], dwg) and torch.equal(b[2], dwu)
    h3 = inner.gated_ffn(x.view(3, 4, 5, 64), wg, wu)
    assert h3.shape == (3, 4, 5, 128) and torch.equal(h3.view(60, 128), inner.gated_ffn(x, wg, wu))
    h0, s0 = inner.gated_ffn(x[:0], wg, wu, save=True)
    assert h0.shape == (0, 128)
    dx0, dwg0, dwu0 = inner.gated_ffn_grad(dh[:0], x[:0], wg, wu, s0)
    assert dx0.shape == (0, 64) and dwg0.abs().max() == 0 and dwu0.abs().max() == 0


@pytest.mark.parametrize("n", [2, 200])
def test_large_and_invalid_values(n):
    """A NaN row stays in its row; an fp16 product past the type's range saturates h and leaves the
    gradient finite; a large negative gate gives zeros."""
    from paper_2607_03011_gb300 import inner
    x, wg, wu, dh = operands(torch.float16, n, 64, 64, 9)
    x[1, 5] = float("nan")
    h = inner.gated_ffn(x, wg, wu)
    assert torch.isnan(h[1]).all() and torch.isfinite(h[0]).all() and torch.isfinite(h[2:]).all()
    x[1] = 30000.0
    wg.fill_(-1.0)
    wu.fill_(1.0)
    h, saved = inner.gated_ffn(x, wg, wu, save=True)
    assert (h[1] == 0).all()
    dx, dwg, dwu = inner.gated_ffn_grad(dh, x, wg, wu, saved)
    assert torch.isfinite(dx).all() and torch.isfinite(dwg).all() and torch.isfinite(dwu).all()


@pytest.mark.parametrize("exponent", [-28, -12, 12, 28])
def test_scales_far_from_one(exponent):
    """bf16 keeps g and u in a form of its own: small and large products keep their accuracy, and beyond its range
    the gradient is NaN, not some number."""
    from paper_2607_03011_gb300 import inner
    x, wg, wu, dh = operands(torch.bfloat16, 300, 64, 72, 17)
    wu = (wu.float() * 2.0 ** exponent).bfloat16()
    if exponent < 0:
        wg = (wg.float() * 2.0 ** exponent).bfloat16()
    h, saved = inner.gated_ffn(x, wg, wu, save=True)
    dx, dwg, dwu = inner.gated_ffn_grad(dh, x, wg, wu, saved)
    check({"h": h, "dx": dx, "dwg": dwg, "dwu": dwu}, x, wg, wu, dh, "silu")
    wu.fill_(2.0 ** 40)
    x[7] = 1.0
    _, saved = inner.gated_ffn(x, wg, wu, save=True)
    dx, _, _ = inner.gated_ffn_grad(dh, x, wg, wu, saved)
    assert torch.isnan(dx[7]).all()


@pytest.mark.parametrize("kind", ["silu", "gelu_tanh"])
def test_gradient_by_differences(kind):
    """<dh, f(v + e w) - f(v - e w)> / 2e against <grad, w>, f in 64 bits, for each operand."""
    from paper_2607_03011_gb300 import inner
    x, wg, wu, dh = operands(torch.float16, 20, 24, 40, 13)
    _, saved = inner.gated_ffn(x, wg, wu, act=kind, save=True)
    grads = inner.gated_ffn_grad(dh, x, wg, wu, saved, act=kind)
    ops = [x.double(), wg.double(), wu.double()]

    def f(o):
        return ((ref.act(o[0] @ o[1], kind)[0] * (o[0] @ o[2])) * dh.double()).sum()

    for i in range(3):
        g = torch.Generator(device="cuda").manual_seed(i)
        w = torch.randn(ops[i].shape, generator=g, device="cuda", dtype=torch.float64)
        e = 1e-5
        up, dn = list(ops), list(ops)
        up[i], dn[i] = ops[i] + e * w, ops[i] - e * w
        quot = (f(up) - f(dn)) / (2 * e)
        got = (grads[i].double() * w).sum()
        # each entry is off by 4 U in the norm (as above), so the product by at most that times both norms
        assert abs(got - quot) < 4 * ref.U[torch.float16] * grads[i].double().norm() * w.norm()


def test_stream():
    from paper_2607_03011_gb300 import inner
    x, wg, wu, dh = operands(torch.bfloat16, 300, 128, 256, 21)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    h, saved = inner.gated_ffn(x, wg, wu, save=True, stream=s)
    dx, dwg, dwu = inner.gated_ffn_grad(dh, x, wg, wu, saved, stream=s)
    s.synchronize()
    check({"h": h, "dx": dx, "dwg": dwg, "dwu": dwu}, x, wg, wu, dh, "silu")


def test_refusals():
    from paper_2607_03011_gb300 import inner, isoloco
    x, wg, wu, dh = operands(torch.bfloat16, 4, 16, 32, 1)
    _, saved = inner.gated_ffn(x, wg, wu, save=True)
    for bad in (lambda: inner.gated_ffn(x.float(), wg.float(), wu.float()), lambda: inner.gated_ffn(x, wg, wu.half()),
                lambda: inner.gated_ffn(x, wg, wu, act="relu"), lambda: inner.gated_ffn(x, wg[:8], wu[:8]),
                lambda: inner.gated_ffn(x, wg, wu[:, :16]), lambda: inner.gated_ffn(x.t(), wg, wu),
                lambda: inner.gated_ffn(x.cpu(), wg, wu), lambda: inner.gated_ffn_grad(dh[:3], x, wg, wu, saved),
                lambda: inner.gated_ffn_grad(dh, x, wg, wu, saved[:-16]), lambda: inner.gated_ffn_grad(dh.half(), x, wg, wu, saved)):
        with pytest.raises((ValueError, isoloco.IsolocoError)):
            bad()
    torch.cuda.synchronize()
