"""A small IsoLoCo run, inner and outer steps on one GPU: ``python -m paper_2607_03011_gb300.inner_demo``.

K workers train replicas of a one-block language model on their own shards of a synthetic text (each
token is followed by a fixed other one most of the time).  A replica's inner step runs the operators of
`inner` in order: embedding, gated block, log probabilities with their gradient, the block's and the
embedding's gradients, clipping; the plain products around them are torch's.  After `inner_steps` steps the
replicas go through the outer step of `isoloco` (Alg. 2), and the merged model is scored on held-out text
with `token_logprobs`: loss, entropy, and how often the next token is among the five likeliest.
"""
from __future__ import annotations

import math
from typing import Dict, List

import torch

from . import inner, isoloco
from .workloads import param_table


def shapes(vocab: int, width: int, ff: int):
    return [("embed", vocab, width), ("w_gate", width, ff), ("w_up", width, ff), ("w_down", ff, width),
            ("head", vocab, width)]


def views(flat: torch.Tensor, spec) -> Dict[str, torch.Tensor]:
    return {name: flat[off:off + r * c].view(r, c) for (name, _, _), (off, r, c) in zip(spec, param_table(spec))}


def forward(p: Dict[str, torch.Tensor], ids: torch.Tensor, save: bool):
    """Logits (bf16) and what the backward pass needs."""
    w = {name: v.bfloat16() for name, v in p.items()}
    x = inner.embed(w["embed"], ids)
    h = inner.gated_ffn(x, w["w_gate"], w["w_up"], save=save)
    h, saved = h if save else (h, None)
    y = x + h @ w["w_down"]
    return y @ w["head"].t(), (w, x, h, saved, y)


def inner_step(replica: torch.Tensor, spec, ids: torch.Tensor, targets: torch.Tensor, lr: float, max_norm: float):
    """One clipped gradient step on the mean negative log likelihood, in place; returns (loss, norm)."""
    p = views(replica, spec)
    logits, (w, x, h, saved, y) = forward(p, ids, save=True)
    n = ids.numel()
    r = inner.token_logprobs(logits, targets, grad_logp=torch.full((n,), -1.0 / n, device=ids.device))
    g: Dict[str, torch.Tensor] = {"head": r.grad_logits.t() @ y}
    dy = r.grad_logits @ w["head"]
    g["w_down"] = h.t() @ dy
    dx, g["w_gate"], g["w_up"] = inner.gated_ffn_grad(dy @ w["w_down"].t(), x, w["w_gate"], w["w_up"], saved)
    g["embed"] = inner.embed_grad(dx + dy, ids, w["embed"].shape[0], dtype=torch.float32)
    grads = [g[name].contiguous() for name, _, _ in spec]
    norm = inner.clip_grads(grads, max_norm)
    for (name, _, _), d in zip(spec, grads):
        p[name].sub_(lr * d.float())
    return -r.logp.mean(), norm


def evaluate(theta: torch.Tensor, spec, ids: torch.Tensor, targets: torch.Tensor):
    """(loss, entropy, share of targets among the five likeliest) on held-out text."""
    logits, _ = forward(views(theta, spec), ids, save=False)
    r = inner.token_logprobs(logits, targets, top=5)
    hit = (r.top_index == targets[:, None]).any(1).float().mean()
    return -r.logp.mean().item(), r.entropy.mean().item(), hit.item()


def text(follow: torch.Tensor, n: int, gen: torch.Generator):
    """n tokens and their successors: `follow` nine times in ten, else any."""
    vocab, dev = follow.numel(), follow.device
    ids = torch.randint(0, vocab, (n,), generator=gen, device=dev)
    noise = torch.randint(0, vocab, (n,), generator=gen, device=dev)
    return ids, torch.where(torch.rand(n, generator=gen, device=dev) < 0.9, follow[ids], noise)


def run(workers: int = 4, rounds: int = 4, inner_steps: int = 12, tokens: int = 2048, vocab: int = 512, width: int = 128,
        ff: int = 256, lr: float = 1.0, max_norm: float = 1.0, seed: int = 0, report=print) -> List[float]:
    """Held-out losses before the first and after every outer step."""
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    spec = shapes(vocab, width, ff)
    table = param_table(spec)
    n = table[-1][0] + table[-1][1] * table[-1][2]
    theta = torch.empty(n, device=dev)
    for name, v in views(theta, spec).items():
        v.copy_(torch.randn(v.shape, generator=gen, device=dev) * (1.0 if name == "embed" else 1.0 / math.sqrt(width)))
    momentum = torch.zeros_like(theta)
    follow = torch.randperm(vocab, generator=gen, device=dev)
    held_out = text(follow, 4 * tokens, gen)
    plan = isoloco.Plan(table, n, workers)
    losses = [evaluate(theta, spec, *held_out)[0]]
    report(f"{n} parameters, {workers} workers; held-out loss {losses[0]:.3f} (uniform: {math.log(vocab):.3f})")
    for rnd in range(rounds):
        replicas = theta.repeat(workers, 1)
        for k in range(workers):
            for _ in range(inner_steps):
                loss, norm = inner_step(replicas[k], spec, *text(follow, tokens, gen), lr=lr, max_norm=max_norm)
        plan.outer_step(theta, momentum, replicas, isoloco.make_opts(outer_lr=0.7, momentum=0.5, sync=True))
        held = evaluate(theta, spec, *held_out)
        losses.append(held[0])
        report(f"round {rnd}: last inner loss {loss.item():.3f}, gradient norm {norm.item():.2f}; merged model: held-out loss "
               f"{held[0]:.3f}, entropy {held[1]:.3f}, in the top five {100 * held[2]:.1f} %")
    if inner.status() != isoloco.OK:
        raise isoloco.IsolocoError(inner.status(), isoloco.last_error())
    plan.close()
    return losses


if __name__ == "__main__":
    run()
