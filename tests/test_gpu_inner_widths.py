"""The inner step's operators at the widths of the framework's own shape sets."""
import pytest
import torch

import inner_ref as ref
from test_gpu_gated_ffn import check, operands

pytestmark = pytest.mark.gpu


def widths(name):
    from paper_2607_03011_gb300.workloads import SPECS
    shapes = {s[0]: s[1:] for s in SPECS[name].shapes}
    return next(v for k, v in shapes.items() if k.endswith("w_gate"))


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("name", ["llama_180m_k8", "llama_1b_k8", "llama_3b_k4"])
@pytest.mark.parametrize("n", [1, 2, 65, 300])
def test_block(dt, name, n):
    from paper_2607_03011_gb300 import inner, isoloco
    x, wg, wu, dh = operands(dt, n, *widths(name), n)
    h, saved = inner.gated_ffn(x, wg, wu, save=True)
    dx, dwg, dwu = inner.gated_ffn_grad(dh, x, wg, wu, saved)
    check({"h": h, "dx": dx, "dwg": dwg, "dwu": dwu}, x, wg, wu, dh, "silu")
    assert inner.status() == isoloco.OK


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("name", ["llama_180m_k8", "llama_1b_k8", "llama_3b_k4"])
def test_lookup_and_table_gradient(dt, name):
    from paper_2607_03011_gb300 import inner
    d, vocab, n = widths(name)[0], 4001, 2050
    g = torch.Generator(device="cuda").manual_seed(d)
    w = torch.randn(vocab, d, generator=g, device="cuda").to(dt)
    ids = (torch.rand(n, generator=g, device="cuda") ** 3 * vocab).long()
    assert torch.equal(inner.embed(w, ids), w[ids])
    dy = torch.randn(n, d, generator=g, device="cuda").to(dt)
    exact, bound = ref.embed_grad(dy, ids, vocab, 1.0)
    for out in {dt, torch.float32}:
        ref.assert_within(inner.embed_grad(dy, ids, vocab, dtype=out), exact, bound, f"{name} {out}")
