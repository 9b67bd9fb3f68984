"""Sizes past an entry point's limits are refused as the module says, before anything is allocated for them."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def room():
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    yield
    torch.cuda.empty_cache()


def refused():
    from paper_2607_03011_gb300 import isoloco
    return pytest.raises((ValueError, isoloco.IsolocoError), match=r"2\^\d+")  # (the limit is named)


def test_a_gradient_tensor_of_too_many_entries():
    from paper_2607_03011_gb300 import inner
    t = torch.empty((1 << 33) + 1, dtype=torch.bfloat16, device="cuda")
    with refused():
        inner.grad_norm([t])
    with refused():
        inner.clip_grads([t], 1.0)


def test_too_many_tokens():
    from paper_2607_03011_gb300 import inner
    n = 1 << 31
    x = torch.empty(n, 1, dtype=torch.bfloat16, device="cuda")
    w = torch.empty(1, 1, dtype=torch.bfloat16, device="cuda")
    for save in (False, True):
        with refused():
            inner.gated_ffn(x, w, w, save=save)
    with refused():
        inner.gated_ffn_grad(x, x, w, w, torch.empty(16, dtype=torch.uint8, device="cuda"))
    ids = torch.empty(n, dtype=torch.int32, device="cuda")
    with refused():
        inner.embed_grad(x, ids, 10)
