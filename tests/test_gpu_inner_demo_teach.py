"""The demo's teaching and answering: they run, and the student's gradients are the formula's."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def parameters(spec, seed):
    from paper_2607_03011_gb300 import inner_demo as demo
    g = torch.Generator(device="cuda").manual_seed(seed)
    flat = torch.randn(sum(r * c for _, r, c in spec), generator=g, device="cuda")
    for name, v in demo.views(flat, spec).items():
        v.mul_(1.0 if name == "embed" else v.shape[0] ** -0.5 if name != "head" else v.shape[1] ** -0.5)
    return flat.bfloat16().float()


def test_gradients_of_the_student():
    from paper_2607_03011_gb300 import inner, inner_demo as demo
    big, small = demo.shapes(300, 64, 128), demo.shapes(300, 32, 64)
    teacher, student = parameters(big, 1), parameters(small, 2)
    ids = torch.randint(0, 300, (500,), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    loss, grads = demo.taught(student, small, teacher, big, ids, top=8)
    t = inner.token_logprobs(demo.forward(demo.views(teacher, big), ids, save=False)[0], ids, top=8)
    top_logp, top_index, ids = t.top_logp.cpu().double(), t.top_index.cpu(), ids.cpu()
    p = {k: v.cpu().double().requires_grad_(True) for k, v in demo.views(student, small).items()}
    x = p["embed"][ids]
    y = x + (torch.nn.functional.silu(x @ p["w_gate"]) * (x @ p["w_up"])) @ p["w_down"]
    lp = torch.log_softmax(y @ p["head"].t(), 1)
    q = top_logp.exp()
    rest, share = 1 - q.sum(1), 1 - lp.gather(1, top_index).exp().sum(1)
    want = ((q * (q.log() - lp.gather(1, top_index))).sum(1) + rest * (rest.log() - share.log())).mean()
    assert abs(loss.item() - want.item()) < 2e-2 * want.item()
    for k, d in zip(p, torch.autograd.grad(want, list(p.values()))):
        # some eight roundings to bf16 (2^-8 each) lie between the definition and a gradient
        assert ((grads[k].cpu().double() - d).norm() / d.norm()).item() < 8 * 2.0 ** -8, k


def test_answers():
    from paper_2607_03011_gb300 import inner_demo as demo
    spec = demo.shapes(300, 64, 128)
    theta = parameters(spec, 4)
    prompts = torch.tensor([5, 77, 299], device="cuda")
    scores, tokens = demo.answer(theta, spec, prompts, beams=4, length=5)
    assert (scores[:, :-1] >= scores[:, 1:]).all() and (tokens[:, :, 0] == prompts[:, None]).all()
    # a score is the sum of its tokens' log probabilities
    logits, _ = demo.forward(demo.views(theta, spec), tokens[:, :, :-1].reshape(-1), save=False)
    lp = torch.log_softmax(logits.double(), 1).gather(1, tokens[:, :, 1:].reshape(-1, 1)).view(3, 4, 5).sum(2)
    assert torch.allclose(scores.double(), lp, rtol=0, atol=5 * 4 * 2.0 ** -20)
    assert len({tuple(t) for t in tokens[0].tolist()}) == 4
