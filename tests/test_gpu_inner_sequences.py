"""Gradients given as any iterable: the tensors are kept for the stream that works on them."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture
def recorded(monkeypatch):
    seen = []
    plain = torch.Tensor.record_stream

    def record(t, stream):
        seen.append((t.data_ptr(), stream.cuda_stream))
        return plain(t, stream)

    monkeypatch.setattr(torch.Tensor, "record_stream", record)
    return seen


FORMS = [list, tuple, iter, lambda v: dict(enumerate(v)).values(), lambda v: (t for t in v)]


@pytest.mark.parametrize("form", FORMS, ids=["list", "tuple", "iterator", "dict values", "generator"])
def test_tensors_are_recorded_on_the_stream(recorded, form):
    from paper_2607_03011_gb300 import inner
    ts, outs = [torch.ones(100 * i, device="cuda") for i in (1, 2, 3)], [torch.empty(100 * i, device="cuda") for i in (1, 2, 3)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    n = inner.grad_norm(form(ts), stream=s)
    assert {p for p, q in recorded if q == s.cuda_stream} >= {t.data_ptr() for t in ts}
    recorded.clear()
    m = inner.clip_grads(form(ts), 1.0, out=form(outs), stream=s)
    assert {p for p, q in recorded if q == s.cuda_stream} >= {t.data_ptr() for t in ts + outs}
    s.synchronize()
    assert abs(n.item() - 600 ** 0.5) < 1e-4 and m.item() == n.item()
    assert all(abs(o.double().square().sum().item() - len(o) / 600) < 1e-5 for o in outs)
