"""The logits' gradient takes the room its rows need, whatever the logits' pitch is."""
import pytest
import torch

from test_gpu_token_logprobs import check_grad, check_stats, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("length,v", [(1, 1000), (7, 1003), (50, 1000), (3, 5)])
def test_last_position_of_every_sequence(dt, length, v):
    """logits[:, -1] of a batch x length x vocabulary tensor: rows length x vocabulary apart."""
    from paper_2607_03011_gb300 import inner
    batch = 5
    z, _, _, _ = make(dt, batch * length, v, v + length)
    _, t, gl, ge = make(dt, batch, v, 3)
    z = z.reshape(batch, length, v)[:, -1]
    r = inner.token_logprobs(z, t, grad_logp=gl, grad_entropy=ge)
    e, base = check_stats(r, z, t, 1.0)
    d = inner.token_logprobs_grad(z, t, r.lse, r.entropy, gl, ge)
    es = z.element_size()
    for g in (r.grad_logits, d):
        assert g.shape == z.shape and g.dtype == dt
        check_grad(g, e, base, 1.0, gl, ge)
        assert g.untyped_storage().nbytes() <= batch * (v * es + 16)
        # rows start as far from a 16-byte boundary as the logits' do
        first = z.data_ptr() - g.data_ptr()
        assert all((z[i].data_ptr() - g[i].data_ptr() - first) % 16 == 0 for i in range(batch))


def test_small_pitches_stay():
    from paper_2607_03011_gb300 import inner
    z, t, gl, _ = make(torch.bfloat16, 6, 1003, 2, pad=5)
    r = inner.token_logprobs(z, t, grad_logp=gl)
    assert r.grad_logits.stride() == z.stride() == (1008, 1)
