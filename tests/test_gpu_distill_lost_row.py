"""A row whose copy does not arrive: the bounded wait gives up, the call's rows are NaN, the status says so, and the next call
is as before.  (On the host's request the kernel does not start the copy.)"""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tail", ["drop", "rest"])
@pytest.mark.parametrize("rows,vocab,dtype", [(3, 700, torch.bfloat16), (2, 40000, torch.float32), (200, 30001, torch.float16)])
def test_a_wait_that_gives_up(rows, vocab, dtype, tail):
    from paper_2607_03011_gb300 import inner, isoloco
    g = torch.Generator(device="cuda").manual_seed(rows)
    z = (torch.randn(rows, vocab, generator=g, device="cuda") * 2).to(dtype)
    ids = torch.randint(0, vocab, (rows, 9), generator=g, device="cuda")
    v = torch.log_softmax(torch.randn(rows, 10, generator=g, device="cuda"), 1)[:, :9]
    w = torch.ones(rows, device="cuda")
    ids[1] = -1                                     # no list: 0 whatever the logits

    def call():
        return inner.distill(z, v, ids, tail=tail, grad_loss=w, save=True)

    inner.status()
    want = call()
    assert inner.status() == isoloco.OK
    assert isoloco.lib().isoloco_debug_lose_rows(1) == isoloco.OK
    lost = call()
    assert inner.status() == isoloco.ERR_TIMEOUT
    with_list = torch.arange(rows, device="cuda") != 1
    assert torch.isnan(lost.loss[with_list]).all() and torch.isnan(lost.grad_logits[with_list]).all()
    assert lost.loss[1] == 0 and (lost.grad_logits[1] == 0).all()
    back = inner.distill_grad(w, z, v, ids, lost.saved, tail=tail)
    assert torch.isnan(back[with_list]).all() and (back[1] == 0).all()
    again = call()
    assert inner.status() == isoloco.OK
    assert torch.equal(again.loss, want.loss) and torch.equal(again.grad_logits, want.grad_logits)
    assert torch.equal(again.saved, want.saved)
