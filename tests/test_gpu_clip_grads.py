"""Global gradient norm and clipping against 64-bit sums."""
import math

import pytest
import torch

import inner_ref as ref

pytestmark = pytest.mark.gpu
DT = [torch.float32, torch.bfloat16, torch.float16]


def tensors(sizes, dts, seed, offset=0, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        base = torch.randn(n + offset, generator=g, device="cuda") * std
        out.append(base.to(dts[i % len(dts)])[offset:])
    return out


def exact_norm(ts):
    return math.sqrt(sum(float(t.double().square().sum()) for t in ts))


def norm_tol(ts):
    # squares and their fp32 partial sums over at most 2^10 terms per thread and chunk, halved by the root
    return (1024 + 8) * 2.0 ** -24


SETS = [[1], [0, 5, 0], [7, 8, 9], [64 * 64, 64 * 256, 64, 256], [8192], [8193, 16385, 3], [100003, 1, 2_000_001],
        [17] * 300, [5] * 1300 + [40000], [3_000_000]]


@pytest.mark.parametrize("sizes", SETS, ids=lambda s: f"{len(s)}x{max(s)}")
@pytest.mark.parametrize("dts", [[torch.float32], [torch.bfloat16], [torch.float16], DT], ids=["f32", "bf16", "f16", "mixed"])
@pytest.mark.parametrize("offset", [0, 1, 5])
def test_norm_and_clip(sizes, dts, offset):
    from paper_2607_03011_gb300 import inner
    ts = tensors(sizes, dts, len(sizes), offset)
    want = exact_norm(ts)
    n = inner.grad_norm(ts)
    assert n.dim() == 0 and abs(n.item() - want) <= norm_tol(ts) * want
    assert torch.equal(n, inner.grad_norm(ts))
    for factor in (0.3, 2.0):
        outs = [torch.full_like(t, 9.0) for t in ts]
        m = inner.clip_grads(ts, factor * want, out=outs)
        assert torch.equal(m, n)
        coef = min(1.0, factor)
        for o, t in zip(outs, ts):
            # the coefficient carries the norm's error and two roundings
            ref.assert_within(o, t.double() * coef, t.double().abs() * coef * (norm_tol(ts) + 2.0 ** -22))
            if factor > 1:
                assert torch.equal(o, t)
        # copies at the same offset from a 16-byte boundary: which thread adds which entry goes by that
        inp = [torch.empty(t.numel() + offset, dtype=t.dtype, device="cuda")[offset:].copy_(t) for t in ts]
        m = inner.clip_grads(inp, factor * want)
        assert torch.equal(m, n) and all(torch.equal(a, b) for a, b in zip(inp, outs))


def test_outputs_at_other_addresses_modulo_16_and_the_inputs_own():
    from paper_2607_03011_gb300 import inner
    ts = tensors([100_001, 4097], [torch.bfloat16], 2)
    want = [t.clone() for t in ts]
    inner.clip_grads(want, 1.0)
    outs = [torch.empty(t.numel() + 3, dtype=t.dtype, device="cuda")[3:] for t in ts]
    inner.clip_grads(ts, 1.0, out=outs)
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    inner.clip_grads(ts, 1.0, out=[ts[0], outs[1]])
    assert torch.equal(ts[0], want[0]) and torch.equal(outs[1], want[1])


def test_neighbours_are_left_alone():
    from paper_2607_03011_gb300 import inner
    buf = torch.ones(5000, device="cuda")
    ts = [buf[1:14], buf[20:4099]]
    inner.clip_grads(ts, 0.5)
    assert buf[0] == 1 and (buf[14:20] == 1).all() and (buf[4099:] == 1).all() and (buf[1:14] != 1).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), 3e38])
def test_a_norm_that_is_not_finite_scales_nothing(bad):
    from paper_2607_03011_gb300 import inner
    ts = tensors([1000, 2000], [torch.float32], 3)
    ts[1][77] = bad
    keep = [t.clone() for t in ts]
    outs = [torch.empty_like(t) for t in ts]
    n = inner.clip_grads(ts, 1.0, out=outs)
    assert not torch.isfinite(n)
    inner.clip_grads(ts, 1.0)
    for a, b, c in zip(ts, keep, outs):
        assert torch.equal(a.view(torch.int32), b.view(torch.int32)) and torch.equal(c.view(torch.int32), b.view(torch.int32))


def test_zero_gradient_no_tensors_and_stream():
    from paper_2607_03011_gb300 import inner
    z = [torch.zeros(100, device="cuda"), torch.zeros(0, device="cuda")]
    assert inner.clip_grads(z, 1.0).item() == 0 and z[0].abs().max() == 0
    assert inner.grad_norm([]).item() == 0 and inner.clip_grads([], 1.0).item() == 0
    s = torch.cuda.Stream()
    ts = tensors([70000], [torch.float32], 5)
    s.wait_stream(torch.cuda.current_stream())
    n = inner.clip_grads(ts, 1.0, stream=s)
    s.synchronize()
    assert abs(n.item() - math.sqrt(70000)) < 10
    assert abs(exact_norm(ts) - 1.0) < 1e-5


def test_refusals():
    from paper_2607_03011_gb300 import inner, isoloco
    t = torch.randn(100, device="cuda")
    for bad in (lambda: inner.grad_norm([t.double()]), lambda: inner.grad_norm([t.cpu()]), lambda: inner.grad_norm([t[::2]]),
                lambda: inner.clip_grads([t], 0.0), lambda: inner.clip_grads([t], float("nan")),
                lambda: inner.clip_grads([t], -1.0), lambda: inner.clip_grads([t], 1.0, out=[]),
                lambda: inner.clip_grads([t], 1.0, out=[t[:50]]), lambda: inner.clip_grads([t], 1.0, out=[t.half()])):
        with pytest.raises((ValueError, isoloco.IsolocoError)):
            bad()
    torch.cuda.synchronize()
