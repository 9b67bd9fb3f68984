"""The gated block's gradient over many tokens: sums of one sign keep their accuracy, and no token is left out where
the sums over all tokens are cut into slices of 65536."""
import pytest
import torch

import inner_ref as ref
from test_gpu_gated_ffn import DT, check, operands

pytestmark = pytest.mark.gpu


def weight_grads(x, wg, wu, dh):
    from paper_2607_03011_gb300 import inner, isoloco
    _, saved = inner.gated_ffn(x, wg, wu, save=True)
    dx, dwg, dwu = inner.gated_ffn_grad(dh, x, wg, wu, saved)
    _, a, b = inner.gated_ffn_grad(dh, x, wg, wu, saved, need_x=False)
    assert torch.equal(a, dwg) and torch.equal(b, dwu) and inner.status() == isoloco.OK
    return {"dx": dx, "dwg": dwg, "dwu": dwu}


@pytest.mark.parametrize("n", [1 << 16, 1 << 18, 1 << 20])
def test_sums_of_one_sign(n):
    """One rounding of the output, and what a slice's sum may lose: 6e-9 of it per product, 4e-4 over 2^16 (a rounding to
    bf16 is some 1.4e-3 in the norm here: together 1.04 times that; roundings of single products average out)."""
    x, wg, wu, dh = (v.abs() for v in operands(torch.bfloat16, n, 64, 64, 3))
    got = weight_grads(x, wg, wu, dh)
    exact = ref.gated_ffn(x, wg, wu, "silu", dh)
    for name in ("dwg", "dwu"):
        e = exact[name][0]
        assert ref.rel(got[name], e) < 1.25 * ref.rel(e.bfloat16(), e), name


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("n,d,f", [(65536, 40, 72), (65537, 40, 72), (131072, 24, 136), (131073, 129, 70), (200003, 300, 40),
                                   (262144 - 63, 264, 8)])
def test_around_the_slices(dt, n, d, f):
    x, wg, wu, dh = operands(dt, n, d, f, n)
    check(weight_grads(x, wg, wu, dh), x, wg, wu, dh, "silu")


@pytest.mark.parametrize("dt", DT)
def test_tokens_at_the_slices_ends_count(dt):
    """All but a few tokens have no gradient: each of those is a good part of the sums."""
    n, d, f = 200003, 40, 72
    x, wg, wu, dh = operands(dt, n, d, f, 8)
    at = torch.tensor([0, 63, 64, 65535, 65536, 65599, 131071, 131072, 196607, 196608, n - 1], device="cuda")
    few = torch.zeros_like(dh)
    few[at] = dh[at]
    got = weight_grads(x, wg, wu, few)
    r = ref.gated_ffn(x[at], wg, wu, "silu", dh[at])
    for name in ("dwg", "dwu"):
        assert ref.rel(got[name], r[name][0]) < 4 * ref.U[dt], name
