"""Performance cases of the operators with which a model is taught by another and answers.

The merged model teaches: a worker, or a smaller model, learns from the likeliest tokens that
`token_logprobs(top=k)` recorded of it.  And it answers: beams of continuations are searched, and what is kept
for each beam follows it.  A case is one pass through one of these operators of `paper_2607_03011_gb300.inner`:

* `distill`: per row the divergence of the student's distribution from the teacher's, which is given by k tokens and
  their log probabilities; either the teacher renormalised over these tokens (tail "drop") or with one further outcome
  for all others (tail "rest"); and (train) the logits' gradient, in the same call or (split) in a later one;
* `select`: the `keep` continuations of the largest total log probability over the beams and the vocabulary;
* `reorder`: the caches and token histories of the beams that were continued, into the new beams' places.

Sizes are those of the shape sets of `workloads.py` (vocabulary 32000, 16 heads of 64 in 12 layers) or generic ones.
"""
from __future__ import annotations

import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}

_LISTED = [
    # Learning while answering: six positions, a step that only its latency matters for.
    dict(name="distill_6_rows", op="distill", T=6, V=32000, K=16, dtype="bf16", vdtype="f32", ids=64, tail="drop", scale=1.0,
         train=True, split=False, pad=0, none=0.0),
    # A micro-batch of odd length over an odd vocabulary (rows start at odd addresses), in fp16, with all other tokens as
    # one outcome; a tenth of the rows are prompt, and lists end early.
    dict(name="distill_train_odd", op="distill", T=2047, V=50021, K=20, dtype="f16", vdtype="f16", ids=32, tail="rest",
         scale=1.0, train=True, split=False, pad=0, none=0.1),
    # How far a student is from the teacher on held-out text: no gradient, fp32 logits, a temperature.
    dict(name="distill_eval", op="distill", T=4096, V=32000, K=32, dtype="f32", vdtype="f32", ids=64, tail="drop", scale=0.5,
         train=False, split=False, pad=0, none=0.0),
    # The loss of a full micro-batch with its gradient at the ~180M set's head.
    dict(name="distill_train", op="distill", T=8192, V=32000, K=32, dtype="bf16", vdtype="f32", ids=64, tail="drop",
         scale=1.0, train=True, split=False, pad=0, none=0.1),
    # The largest: a large vocabulary, long lists, the backward pass in a call of its own.
    dict(name="distill_train_large", op="distill", T=8192, V=128000, K=64, dtype="bf16", vdtype="bf16", ids=32, tail="rest",
         scale=1.0, train=True, split=True, pad=0, none=0.0),
    # One prompt, four beams: latency.
    dict(name="select_one_prompt", op="select", B=1, W=4, V=32000, keep=4, dtype="bf16", scale=1.0, done=0.0, first=False),
    # Odd vocabulary; twice as many continuations as beams are asked for, a fifth of the beams have ended.
    dict(name="select_16_odd", op="select", B=16, W=8, V=50021, keep=16, dtype="f16", scale=0.8, done=0.2, first=False),
    # A batch of prompts in fp32, five beams each.
    dict(name="select_64_f32", op="select", B=64, W=5, V=32000, keep=5, dtype="f32", scale=1.0, done=0.0, first=False),
    # A batch over a large vocabulary, many beams.
    dict(name="select_large", op="select", B=64, W=16, V=128000, keep=16, dtype="bf16", scale=1.0, done=0.1, first=False),
    # One prompt's four beams, a few tokens in.
    dict(name="reorder_one_prompt", op="reorder", B=1, W=4, layers=2, H=2, L=17, Lmax=64, D=32, dtype="bf16"),
    # Five beams of odd length, heads of an odd width, in fp32.
    dict(name="reorder_odd", op="reorder", B=3, W=5, layers=6, H=7, L=333, Lmax=401, D=33, dtype="f32"),
    # The ~180M set's caches of sixteen prompts with eight beams.
    dict(name="reorder_180m", op="reorder", B=16, W=8, layers=12, H=16, L=500, Lmax=512, D=64, dtype="bf16"),
]


def listed():
    return [dict(c) for c in _LISTED]


def _distinct(W):
    """How many of W sources are expected to be continued (see `prepare`)."""
    return sum(1.0 - (1.0 - (math.sqrt((w + 1) / W) - math.sqrt(w / W))) ** W for w in range(W))


def work(case):
    b, op = _BYTES[case["dtype"]], case["op"]
    if op == "distill":
        T, V, K = case["T"], case["V"], case["K"]
        lists = T * K * (_BYTES[case["vdtype"]] + case["ids"] // 8)
        n = T * V * b * (2 if case["train"] else 1) + lists + 4 * T * (2 if case["train"] else 1)
        return {"bytes": float(n), "flops": float(T * V * (8 if case["train"] else 4))}
    if op == "select":
        B, W, V = case["B"], case["W"], case["V"]
        live = 1 if case["first"] else W * (1.0 - case["done"])
        return {"bytes": B * live * V * b + B * (4 * W + 20 * case["keep"]), "flops": 4.0 * B * live * V}
    B, W = case["B"], case["W"]
    row = 2 * case["layers"] * case["H"] * case["L"] * case["D"] * b + 8 * case["L"]
    return {"bytes": float(B * row * (W + _distinct(W)) + 8 * B * W), "flops": 0.0}


def _cost(case):
    w = work(case)
    return w["bytes"] / 6e12 + w["flops"] / 3e13


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size between lo and hi over its logarithm: a multiple of 64, one of 8, or any."""
    n = _log(rng, lo, hi)
    step = rng.choice([64, 8, 1, 1])
    return max(lo, n // step * step)


def draw(rng):
    """Any operator; rows from one to the largest listed number, vocabularies and lengths over their logarithm,
    odd ones among them; every type, tail and direction."""
    limit = max(_cost(c) for c in _LISTED)
    while True:
        op = rng.choice(["distill", "distill", "distill", "select", "select", "reorder"])
        dt = rng.choice(["f32", "bf16", "f16"])
        if op == "distill":
            train = rng.random() < 0.7
            c = dict(op=op, T=_log(rng, 1, 8192), V=_size(rng, 500, 128000), K=_log(rng, 1, 128), dtype=dt,
                     vdtype=rng.choice(["f32", "f32", "bf16", "f16"]), ids=rng.choice([32, 64]),
                     tail=rng.choice(["drop", "rest"]), scale=rng.choice([1.0, 0.5]), train=train,
                     split=train and rng.random() < 0.4, pad=rng.choice([0, 0, 24]), none=rng.choice([0.0, 0.3]))
        elif op == "select":
            W = rng.choice([1, 2, 3, 4, 5, 6, 8, 10, 12, 16])
            c = dict(op=op, B=_log(rng, 1, 64), W=W, V=_size(rng, 500, 128000), keep=rng.choice([W, 2 * W]), dtype=dt,
                     scale=rng.choice([1.0, 0.7]), done=rng.choice([0.0, 0.3]), first=rng.random() < 0.2)
        else:
            L = _log(rng, 1, 2048)
            c = dict(op=op, B=_log(rng, 1, 32), W=rng.choice([2, 3, 4, 5, 8, 10, 16]), layers=rng.randint(1, 24),
                     H=_log(rng, 1, 16), L=L, Lmax=L + rng.choice([0, 1, 64]), D=rng.choice([16, 33, 64, 80, 128]), dtype=dt)
        if _cost(c) <= limit:
            return c


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dt, op = _DT[case["dtype"]], case["op"]

    def randn(*shape, std=1.0):
        return torch.randn(shape, generator=g, device="cuda") * std

    def rand(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    def fill(rows, V, pad, places):
        """Logits of `rows` rows: noise, a few tokens that stand out as a trained model's do, and unused tokens."""
        full = torch.empty(rows, V + pad, dtype=dt, device="cuda")
        for r in range(0, rows, 1024):
            n = min(1024, rows - r)
            z = randn(n, V + pad, std=2.0)
            z.scatter_add_(1, places[r:r + n], randn(*places[r:r + n].shape, std=5.0).abs())
            z[:, V - V // 100:V] = -math.inf  # rows of the head that no token uses
            full[r:r + n] = z.to(dt)
        return full[:, :V]

    st = {"case": case}
    if op == "distill":
        T, V, K = case["T"], case["V"], case["K"]
        used = V - V // 100
        # k different tokens a row, one of each stretch of the vocabulary, in any order
        ids = ((torch.arange(K, device="cuda") + 0.999 * rand(T, K)) * (used / K)).long().clamp_(max=used - 1)
        low = (torch.arange(K, device="cuda") * (used / K)).ceil().long()
        ids = torch.maximum(ids, low).gather(1, rand(T, K).argsort(1))
        # the student has learned some of them, and some others
        other = torch.randint(0, used, (T, 4), generator=g, device="cuda")
        st["logits"] = fill(T, V, case["pad"], torch.cat([ids[:, :8], other], 1))
        t = torch.sort(randn(T, K, std=2.0), dim=1, descending=True).values
        rest = torch.log(rand(T, 1) * 0.2 + 0.01) + torch.logsumexp(t, 1, keepdim=True)
        st["top_logp"] = (t - torch.logaddexp(torch.logsumexp(t, 1, keepdim=True), rest)).to(_DT[case["vdtype"]])
        if case["none"]:
            # lists that end early, and rows without any
            count = (K * (1.0 - rand(T, 1) * 0.5)).ceil().long()
            count[rand(T, 1) < case["none"]] = 0
            ids[torch.arange(K, device="cuda") >= count] = -1
        st["top_index"] = ids.to(torch.int32 if case["ids"] == 32 else torch.int64)
        if case["train"]:
            st["g"] = (randn(T).abs() + 0.1) * 4.0  # weights of the rows, times a loss scale
    elif op == "select":
        B, W, V = case["B"], case["W"], case["V"]
        places = torch.randint(0, V - V // 100, (B * W, 8), generator=g, device="cuda")
        st["logits"] = fill(B * W, V, 0, places).view(B, W, V)
        st["scores"] = -(rand(B, W) * 6.0 + rand(B, 1) * 40.0)
        st["finished"] = (rand(B, W) < case["done"]) if case["done"] else None
        if case["first"]:
            st["scores"][:, 1:] = -math.inf  # all beams are the prompt: one of them is continued
            st["scores"][:, 0] = 0.0
            st["finished"] = None
        st["end"] = 2 if case["done"] and not case["first"] else None
    else:
        B, W, H, L, Lmax, D = (case[k] for k in ("B", "W", "H", "L", "Lmax", "D"))
        st["states"], st["out"] = [], []
        for _ in range(2 * case["layers"]):
            st["states"].append(torch.empty(B * W, H, Lmax, D, dtype=dt, device="cuda").normal_(generator=g)[:, :, :L])
            st["out"].append(torch.empty(B * W, H, Lmax, D, dtype=dt, device="cuda")[:, :, :L])
        st["states"].append(torch.randint(0, 32000, (B, W, L), generator=g, device="cuda"))
        st["out"].append(torch.empty_like(st["states"][-1]))
        # good beams are continued more often than others
        st["beams"] = (rand(B, W).square() * W).long().clamp_(max=W - 1)
    return st


# ------------------------------------------------------------------ the framework's operators

def _run_own(st):
    from paper_2607_03011_gb300 import inner

    case = st["case"]
    op = case["op"]
    if op == "distill":
        args = (st["logits"], st["top_logp"], st["top_index"])
        if not case["train"]:
            return {"loss": inner.distill(*args, scale=case["scale"], tail=case["tail"]).loss}
        if case["split"]:
            r = inner.distill(*args, scale=case["scale"], tail=case["tail"], save=True)
            dz = inner.distill_grad(st["g"], *args, r.saved, scale=case["scale"], tail=case["tail"])
            return {"loss": r.loss, "dlogits": dz}
        r = inner.distill(*args, scale=case["scale"], tail=case["tail"], grad_loss=st["g"])
        return {"loss": r.loss, "dlogits": r.grad_logits}
    if op == "select":
        r = inner.beam_select(st["logits"], st["scores"], keep=case["keep"], finished=st["finished"], end=st["end"],
                              scale=case["scale"])
        return {"scores": r.scores, "beams": r.beams, "tokens": r.tokens}
    inner.beam_reorder(st["states"], st["beams"], out=st["out"])
    return st["out"]


# ------------------------------------------------------------------ their plain forms

def _ordered(x):
    """fp32 values as whole numbers of the same order."""
    x = torch.where(x == 0, torch.zeros_like(x), x)  # -0 and 0 are equal
    i = x.view(torch.int32).long()
    return torch.where(i < 0, -(i & 0x7FFFFFFF), i)


def _run_plain(st):
    case = st["case"]
    op, dt = case["op"], _DT[case["dtype"]]
    if op == "distill":
        T, V = case["T"], case["V"]
        ids, v = st["top_index"].long(), st["top_logp"].float()
        there = (ids >= 0) & (ids < V)
        any_there = there.any(1)
        at = torch.where(there, ids, torch.full_like(ids, V))
        x = st["logits"].float() * case["scale"]
        m = x.amax(1, keepdim=True)
        e = torch.exp(x - m)
        s = e.sum(1, keepdim=True)
        lp = (x - m).gather(1, at.clamp(max=V - 1)) - torch.log(s)  # the student's log probabilities of the list's tokens
        w = torch.where(there, torch.exp(v), torch.zeros_like(v))
        outside = None
        if case["tail"] == "drop":
            q = w / w.sum(1, keepdim=True).clamp(min=1e-30)
            rest = torch.zeros_like(m)
        else:
            q = w
            rest = torch.where(any_there[:, None], (1.0 - q.sum(1, keepdim=True)).clamp(min=0.0), torch.zeros_like(m))
            outside = torch.ones(T, V + 1, device="cuda").scatter_(1, at, 0.0)[:, :V]
            others = (e * outside).sum(1, keepdim=True)
            rest = torch.where(others > 0, rest, torch.zeros_like(rest))
            share = torch.where(others > 0, others / s, torch.ones_like(s))
        loss = torch.where(q > 0, q * (torch.log(q) - lp), torch.zeros_like(q)).sum(1)
        if outside is not None:
            loss = loss + torch.where(rest > 0, rest * (torch.log(rest) - torch.log(share)), torch.zeros_like(rest))[:, 0]
        o = {"loss": loss}
        if case["train"]:
            d = (e / s) * (q.sum(1, keepdim=True) + rest)
            if outside is not None:
                d = d - e * outside * torch.where(others > 0, rest / others, torch.zeros_like(rest))
            full = torch.zeros(T, V + 1, device="cuda").scatter_add_(1, at, q)
            o["dlogits"] = ((d - full[:, :V]) * (st["g"] * case["scale"])[:, None]).to(dt)
        return o
    if op == "select":
        # in 64 bits: totals of different beams that are close to each other are ranked
        B, W, V, keep = case["B"], case["W"], case["V"], case["keep"]
        sc = float(torch.tensor(case["scale"], dtype=torch.float32))
        z = st["logits"].float()
        if st["finished"] is not None:
            only = torch.full((V,), -math.inf, device="cuda")
            only[st["end"]] = 0.0
            z = torch.where(st["finished"][:, :, None], only, z)
        z = torch.where(st["scores"][:, :, None] > -math.inf, z, torch.full_like(z, -math.inf))
        # a beam's likeliest tokens, the lowest index first among equal ones; then the likeliest of all beams'
        k = min(keep, V)
        at = (_ordered(z) * 2 ** 24 + (V - 1 - torch.arange(V, device="cuda"))).topk(k, dim=2).indices
        x = z.double() * sc
        m = x.amax(2, keepdim=True).clamp(min=-1e300)
        lse = m + torch.log(torch.exp(x - m).sum(2, keepdim=True))
        total = (st["scores"].double()[:, :, None] + (x.gather(2, at) - lse)).nan_to_num(nan=-math.inf, neginf=-math.inf)
        val, place = torch.sort(total.view(B, W * k), dim=1, descending=True, stable=True)
        place = place[:, :keep].contiguous()
        return {"scores": val[:, :keep].float(), "beams": place // k, "tokens": at.view(B, W * k).gather(1, place)}
    B, W = case["B"], case["W"]
    rows = (torch.arange(B, device="cuda")[:, None] * W + st["beams"]).view(-1)
    moved = [s[rows] for s in st["states"][:-1]]
    last = st["states"][-1]
    return moved + [last.view(B * W, -1)[rows].view(last.shape)]


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------ the definitions in 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    sc = float(torch.tensor(case.get("scale", 1.0), dtype=torch.float32))
    if op == "distill":
        V, parts = case["V"], []
        for r in range(0, case["T"], 512):  # rows are independent
            z = st["logits"][r:r + 512].double()
            ids, v = st["top_index"][r:r + 512].long(), st["top_logp"][r:r + 512].double()
            given = (ids >= 0) & (ids < V)
            v = torch.where(given, v, torch.full_like(v, -math.inf))
            has = given.any(1)
            if case["train"]:
                z.requires_grad_(True)
            lp = torch.log_softmax(z * sc, 1)
            mine = torch.where(given, lp.gather(1, torch.where(given, ids, torch.zeros_like(ids))), torch.zeros_like(v))
            if case["tail"] == "drop":
                logq = torch.log_softmax(torch.where(has[:, None], v, torch.zeros_like(v)), 1)
                logq = torch.where(has[:, None], logq, torch.full_like(logq, -math.inf))
            else:
                logq = v
            q = logq.exp()
            loss = (q * (torch.where(given, logq, torch.zeros_like(logq)) - mine)).sum(1)
            if case["tail"] == "rest":
                rest = torch.where(has, 1.0 - q.sum(1), torch.zeros_like(loss)).clamp(min=0.0)
                hidden = torch.zeros(z.shape[0], V + 1, dtype=torch.bool, device="cuda")
                hidden.scatter_(1, torch.where(given, ids, torch.full_like(ids, V)), True)
                log_share = torch.logsumexp(lp.masked_fill(hidden[:, :V], -math.inf), 1)
                on = rest > 0
                log_rest = torch.where(on, rest, torch.ones_like(rest)).log()
                loss = loss + torch.where(on, rest * (log_rest - log_share), torch.zeros_like(rest))
            part = [loss.detach()]
            if case["train"]:
                part.append(torch.autograd.grad(loss, z, st["g"][r:r + 512].double())[0])
            parts.append(part)
        cols = [torch.cat(c) for c in zip(*parts)]
        return dict(zip(["loss", "dlogits"], cols))
    if op == "select":
        B, W, V, keep = case["B"], case["W"], case["V"], case["keep"]
        found = []
        for b in range(B):
            lp = torch.log_softmax(st["logits"][b].double() * sc, 1)
            if st["finished"] is not None:
                lp[st["finished"][b]] = -math.inf
                lp[st["finished"][b], st["end"]] = 0.0
            total = (lp + st["scores"][b].double()[:, None]).reshape(-1)
            order = torch.sort(-total, stable=True).indices[:keep]
            found.append((total[order], order.div(V, rounding_mode="floor"), order.remainder(V)))
        return dict(zip(["scores", "beams", "tokens"], (torch.stack(c) for c in zip(*found))))
    B, W = case["B"], case["W"]
    o = []
    for s in st["states"]:
        own_shape = s.reshape(B, W, -1)
        there = st["beams"][:, :, None].expand(-1, -1, own_shape.shape[2])
        moved = own_shape.gather(1, there).reshape(s.shape)
        o.append(moved.double() if moved.is_floating_point() else moved)
    return o
