"""The gated block's gradient where g = x w_gate or u = x w_up are far below one: bf16 keeps them in a form of
its own, whose lower end is fp32's, so that no gradient is lost while its own value is within bf16's range."""
import pytest
import torch

import inner_ref as ref
from test_gpu_gated_ffn import operands

pytestmark = pytest.mark.gpu


def grads(x, wg, wu, dh, kind):
    from paper_2607_03011_gb300 import inner
    _, saved = inner.gated_ffn(x, wg, wu, act=kind, save=True)
    return dict(zip(("dx", "dwg", "dwu"), inner.gated_ffn_grad(dh, x, wg, wu, saved, act=kind)))


@pytest.mark.parametrize("n", [2, 300])  # the kernel for few tokens, and the pair GEMM
@pytest.mark.parametrize("kind", ["silu", "gelu_tanh"])
@pytest.mark.parametrize("which", ["up", "gate", "both"])
@pytest.mark.parametrize("exponent", [-31, -34, -38, -42, -50, -58])
def test_small_products(n, kind, which, exponent):
    x, wg, wu, dh = operands(torch.bfloat16, n, 64, 72, n - exponent)
    if which != "gate":
        wu = (wu.float() * 2.0 ** exponent).bfloat16()
    if which != "up":
        wg = (wg.float() * 2.0 ** exponent).bfloat16()
    exact = ref.gated_ffn(x, wg, wu, kind, dh)
    for name, v in grads(x, wg, wu, dh, kind).items():
        # roundings of g or u, of dg or du and of the output, each below U and independent: below 4 U in the norm
        assert ref.rel(v, exact[name][0]) < 4 * ref.U[torch.bfloat16], name


@pytest.mark.parametrize("kind", ["silu", "gelu_tanh"])
def test_columns_of_different_scales(kind):
    """Every column of dw_gate depends on its own column of w_up alone, and keeps its accuracy beside columns 2^80
    times as large."""
    x, wg, wu, dh = operands(torch.bfloat16, 300, 64, 136, 5)
    scale = 2.0 ** torch.linspace(-60, 20, 136, device="cuda").round()
    wu = (wu.float() * scale).bfloat16()
    exact, got = ref.gated_ffn(x, wg, wu, kind, dh)["dwg"][0], grads(x, wg, wu, dh, kind)["dwg"].double()
    err = (got - exact).norm(dim=0) / exact.norm(dim=0)
    assert (err < 4 * ref.U[torch.bfloat16]).all(), err.max().item()


def test_the_upper_end():
    """Products of some 2^28."""
    x, wg, wu, dh = operands(torch.bfloat16, 300, 64, 72, 6)
    wu = (wu.float() * 2.0 ** 28).bfloat16()
    exact = ref.gated_ffn(x, wg, wu, "silu", dh)
    for name, v in grads(x, wg, wu, dh, "silu").items():
        assert ref.rel(v, exact[name][0]) < 4 * ref.U[torch.bfloat16], name
