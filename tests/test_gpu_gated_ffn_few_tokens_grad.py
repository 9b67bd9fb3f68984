"""The gated block's gradient for few tokens is as exact as its outputs' type allows: a sum of few products does not
average the roundings of its operands out, so that those count in full."""
import pytest
import torch

import inner_ref as ref
from test_gpu_gated_ffn import DT, check, operands

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("kind", ["silu", "gelu_tanh"])
@pytest.mark.parametrize("n,d,f", [(1, 67, 223), (1, 216, 1072), (1, 208, 2728), (2, 640, 448), (3, 749, 136), (4, 88, 184), (6, 66, 3706),
                                   (13, 1328, 384), (32, 160, 480), (37, 350, 551), (64, 64, 64), (65, 225, 128), (127, 129, 70),
                                   (128, 1024, 264)])
def test_one_rounding(dt, kind, n, d, f):
    """The outputs' own rounding, and for bf16 what g and u are kept in: a fourth of it each, so together below
    sqrt(1 + 2 / 16) = 1.06 of it in the norm; up to 1.25 for the few entries of the smallest cases."""
    from paper_2607_03011_gb300 import inner, isoloco
    x, wg, wu, dh = operands(dt, n, d, f, n + d)
    exact = ref.gated_ffn(x, wg, wu, kind, dh)
    _, saved = inner.gated_ffn(x, wg, wu, act=kind, save=True)
    got = dict(zip(("dx", "dwg", "dwu"), inner.gated_ffn_grad(dh, x, wg, wu, saved, act=kind)))
    check(got, x, wg, wu, dh, kind)
    for name, v in got.items():
        e = exact[name][0]
        assert ref.rel(v, e) < 1.25 * ref.rel(e.to(dt), e), name
    # each part by itself, and the same bits again
    dx, _, _ = inner.gated_ffn_grad(dh, x, wg, wu, saved, act=kind, need_w=False)
    _, dwg, dwu = inner.gated_ffn_grad(dh, x, wg, wu, saved, act=kind, need_x=False)
    assert torch.equal(dx, got["dx"]) and torch.equal(dwg, got["dwg"]) and torch.equal(dwu, got["dwu"])
    assert inner.status() == isoloco.OK


@pytest.mark.parametrize("n", [5, 128, 129])
def test_values_past_fp16(n):
    """A dg or du past fp16's range is inf there and has no rest: its products are inf or NaN, the others' finite."""
    from paper_2607_03011_gb300 import inner
    x, wg, wu, dh = operands(torch.float16, n, 64, 72, 4)
    x[1], wg[:, 3], wu[:, 3] = 40.0, 1.0, 1.0   # g = u = 2560 in that column
    dh[1, 3] = 60.0                             # du = 153600
    _, saved = inner.gated_ffn(x, wg, wu, save=True)
    dx, dwg, dwu = inner.gated_ffn_grad(dh, x, wg, wu, saved)
    assert not torch.isfinite(dx[1]).any() and torch.isfinite(dx[0]).all() and torch.isfinite(dx[2:]).all()
    rest = torch.arange(72, device="cuda") != 3
    assert torch.isfinite(dwg[:, rest]).all() and torch.isfinite(dwu[:, rest]).all()
    assert torch.isinf(dwu[:, 3]).all()
