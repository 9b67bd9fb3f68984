"""Gradients over the logits themselves, of both entry points: the same bits as into other memory."""
import pytest
import torch

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def made(n, vocab, k, dtype, borders=()):
    g = torch.Generator(device="cuda").manual_seed(n + vocab)
    z = (torch.randn(n, vocab, generator=g, device="cuda") * 2).to(dtype)
    ids = torch.randint(-1, vocab, (n, k), generator=g, device="cuda")
    for e, t in enumerate(t for t in borders if t < vocab):
        ids[:, e] = t
    v = torch.log_softmax(torch.randn(n, k + 1, generator=g, device="cuda"), 1)[:, :k].contiguous()
    return z, v, ids, torch.rand(n, generator=g, device="cuda") + 0.5


def stream():
    return torch.cuda.current_stream().cuda_stream


@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("dtype,vocab", [(F32, 901), (BF16, 70001), (F16, 131075), (F32, 40003)])
def test_by_itself(dtype, vocab, tail):
    """Several spans of a row (65536 entries of 16 bits, 32768 of 32), with tokens of the list at their ends."""
    from paper_2607_03011_gb300 import inner, isoloco
    n, k = 7, 24
    z, v, ids, w = made(n, vocab, k, dtype, (0, 32767, 32768, 65535, 65536, 65537, 131071, 131072, vocab - 1))
    name = ("drop", "rest")[tail]
    r = inner.distill(z, v, ids, tail=name, save=True)
    want = inner.distill_grad(w, z, v, ids, r.saved, tail=name)
    rc = isoloco.lib().isoloco_distill_grad(w.data_ptr(), z.data_ptr(), vocab, inner._DTYPE[dtype], n, vocab, v.data_ptr(), k, 0,
                                            ids.data_ptr(), k, 8, k, 1.0, tail, r.saved.data_ptr(), z.data_ptr(), vocab, stream())
    assert rc == 0, isoloco.last_error()
    assert torch.equal(z, want)


@pytest.mark.parametrize("rows,vocab,dtype", [
    (700, 5003, BF16), (400, 20011, F16), (330, 50021, F16),         # one CTA a row, of 64, 128 and 512 threads, three rows or more to an SM
    (170, 40003, F32), (170, 30011, F32), (160, 70001, BF16)])       # several CTAs a row
@pytest.mark.parametrize("tail", [0, 1])
def test_many_rows(rows, vocab, dtype, tail):
    """Rows that share 16-byte pieces with their neighbours, of which some are read while others are written."""
    from paper_2607_03011_gb300 import inner, isoloco
    k = 12
    z, v, ids, w = made(rows, vocab, k, dtype)
    want = inner.distill(z, v, ids, tail=("drop", "rest")[tail], grad_loss=w, save=True)
    loss, saved = torch.empty(rows, device="cuda"), torch.empty(rows, 6, device="cuda")
    rc = isoloco.lib().isoloco_distill(z.data_ptr(), vocab, inner._DTYPE[dtype], rows, vocab, v.data_ptr(), k, 0, ids.data_ptr(), k, 8, k, 1.0,
                                       tail, loss.data_ptr(), saved.data_ptr(), w.data_ptr(), z.data_ptr(), vocab, stream())
    assert rc == 0, isoloco.last_error()
    assert torch.equal(loss, want.loss) and torch.equal(z, want.grad_logits) and torch.equal(saved, want.saved)


def test_several_ctas_a_row_against_the_definition():
    """Many rows of sizes that are split between CTAs: fp32 above 27648 entries, 16 bits above 55000."""
    import teach_ref as ref
    from inner_ref import assert_within
    from paper_2607_03011_gb300 import inner
    for rows, vocab, dtype in ((160, 30011, F32), (160, 55021, F16)):
        z, v, ids, w = made(rows, vocab, 6, dtype)
        ids = torch.stack([torch.randperm(vocab)[:6] for _ in range(rows)]).cuda()
        r = inner.distill(z, v, ids, tail="rest", grad_loss=w)
        zc, vc, ic, wc = z.cpu(), v.cpu(), ids.cpu(), w.cpu()
        loss, dz = ref.distill(zc, vc, ic, 1.0, "rest", wc)
        assert_within(r.loss.cpu(), loss, ref.loss_bound(zc, vc, 1.0), "loss")
        assert_within(r.grad_logits.cpu(), dz, ref.grad_bound(zc, vc, ic, 1.0, wc, dz), "gradient")
