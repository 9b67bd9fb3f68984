"""Performance cases of the operators of a worker's inner step.

Between two outer steps every worker trains its replica: it looks tokens up in its embedding, runs
gated feed-forward blocks, scores the next tokens from the head's logits, and clips the gradient's
global norm; the merged model is then scored on held-out text.  A case is one pass through one of
these four operators of `paper_2607_03011_gb300.inner`:

* `embed`: rows of an embedding times a scale, and (train) the gradient of the whole table;
* `ffn`: h = act(x Wg) * (x Wu) with Wg, Wu of width x ff, and (train) the gradients of x, Wg, Wu;
* `logp`: log probability of each row's given token, entropy and the `top` likeliest tokens, and
  (train) the logits' gradient for given gradients of the log probabilities and entropies;
* `clip`: the norm over all tensors of a gradient, and the gradient scaled down to `max_norm`.

Sizes are those of the shape sets of `workloads.py` (widths 64, 1024 and 2048, ff 256, 2816 and
5632, vocabulary 32000) or generic ones.
"""
from __future__ import annotations

import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}

_LISTED = [
    # Eight sequences that each add one token: a lookup that only its latency matters for.
    dict(name="embed_8_tokens", op="embed", T=8, V=32000, D=1024, dtype="bf16", scale=1.0, train=False, none=0.0),
    # A worker's micro-batch on the ~180M set's embedding: lookup and table gradient.
    dict(name="embed_train_180m", op="embed", T=8192, V=32000, D=1024, dtype="bf16", scale=1.0, train=True, none=0.0),
    # A long batch of odd length on a wide fp32 table with a large vocabulary, rows scaled by
    # sqrt(width), some positions padded.
    dict(name="embed_train_large", op="embed", T=65533, V=128000, D=2048, dtype="f32", scale=45.2548, train=True,
         none=0.02),
    # One token through the ~1.1B set's block: reading the weights is all there is.
    dict(name="ffn_token", op="ffn", T=1, D=2048, F=5632, dtype="bf16", act="silu", train=False),
    # A small odd batch of sequences that each add a token, fp16, the ~180M set's block.
    dict(name="ffn_33_tokens", op="ffn", T=33, D=1024, F=2816, dtype="f16", act="gelu_tanh", train=False),
    # A short micro-batch of odd length, forward and backward, the ~180M set's block.
    dict(name="ffn_train_180m", op="ffn", T=2047, D=1024, F=2816, dtype="bf16", act="silu", train=True),
    # The largest: a full micro-batch, forward and backward, the ~1.1B set's block.
    dict(name="ffn_train_1b", op="ffn", T=16384, D=2048, F=5632, dtype="bf16", act="silu", train=True),
    # Sampling: the log probability of the sampled token of four sequences and 20 alternatives.
    dict(name="logp_sample", op="logp", T=4, V=32000, dtype="f32", top=20, scale=1.25, train=False, pad=0, none=0.0),
    # Held-out text through the merged model: an odd vocabulary (rows that start at odd addresses),
    # five alternatives.
    dict(name="logp_eval", op="logp", T=2049, V=50021, dtype="bf16", top=5, scale=1.0, train=False, pad=0, none=0.0),
    # The loss of a micro-batch with its gradient; a tenth of the targets are prompt tokens (none).
    dict(name="logp_train", op="logp", T=8192, V=32000, dtype="bf16", top=0, scale=1.0, train=True, pad=0, none=0.1),
    # The unit-test-sized set: launch latency.
    dict(name="clip_tiny", op="clip", d=64, ff=256, layers=1, vocab=0, dtype="f32", clip=0.5),
    # The ~180M set's gradient in fp32.
    dict(name="clip_180m", op="clip", d=1024, ff=2816, layers=12, vocab=32000, dtype="f32", clip=0.25),
]


def listed():
    return [dict(c) for c in _LISTED]


def _shapes(case):
    d, ff, vocab = case["d"], case["ff"], case["vocab"]
    s = [(vocab, d)] if vocab else []
    for _ in range(case["layers"]):
        s += [(d,), (d, d), (d, d), (d, d), (d, d), (d,), (d, ff), (d, ff), (ff, d)]
    if vocab:
        s.append((vocab, d))
    return s


def work(case):
    b = _BYTES[case["dtype"]]
    op = case["op"]
    if op == "embed":
        T, V, D = case["T"], case["V"], case["D"]
        n = min(T, V) * D + T * D + (T * D + V * D if case["train"] else 0)
        return {"bytes": float(n * b + 8 * T), "flops": float(T * D * (2 if case["train"] else 1))}
    if op == "ffn":
        T, D, F = case["T"], case["D"], case["F"]
        if case["train"]:
            # x, Wg, Wu and dh in; h and the three gradients out; two products forward, four back
            return {"bytes": float(b * (2 * T * D + 4 * D * F + 2 * T * F)), "flops": 12.0 * T * D * F}
        return {"bytes": float(b * (T * D + 2 * D * F + T * F)), "flops": 4.0 * T * D * F}
    if op == "logp":
        T, V = case["T"], case["V"]
        n = T * V * b * (2 if case["train"] else 1) + T * (16 + 8 * case["top"] + (8 if case["train"] else 0))
        return {"bytes": float(n), "flops": float(T * V * (9 if case["train"] else 5))}
    n = sum(math.prod(s) for s in _shapes(case))
    return {"bytes": float(2 * n * b + 4), "flops": 3.0 * n}


def _cost(case):
    w = work(case)
    return w["bytes"] / 6e12 + w["flops"] / 6e13 * (1.0 if case["op"] == "ffn" else 0.05)


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size between lo and hi over its logarithm: a multiple of 64, one of 8, or any."""
    n = _log(rng, lo, hi)
    step = rng.choice([64, 8, 8, 1])
    return max(step, n // step * step)


def draw(rng):
    """Any operator; tokens from one to the largest listed length, widths and vocabularies over
    their logarithm, odd ones among them; every type, activation and direction."""
    limit = max(_cost(c) for c in _LISTED)
    while True:
        op = rng.choice(["embed", "ffn", "ffn", "logp", "logp", "clip"])
        dt = rng.choice(["f32", "bf16", "f16"])
        if op == "embed":
            c = dict(op=op, T=_log(rng, 1, 65536), V=_log(rng, 500, 128000), D=_size(rng, 64, 4096), dtype=dt,
                     scale=rng.choice([1.0, 27.5]), train=rng.random() < 0.7, none=rng.choice([0.0, 0.1]))
        elif op == "ffn":
            c = dict(op=op, T=_log(rng, 1, 16384), D=_size(rng, 64, 4096), F=_size(rng, 128, 8192),
                     dtype=rng.choice(["bf16", "f16"]), act=rng.choice(["silu", "gelu_tanh"]),
                     train=rng.random() < 0.6)
        elif op == "logp":
            train = rng.random() < 0.5
            c = dict(op=op, T=_log(rng, 1, 8192), V=_log(rng, 500, 128000), dtype=dt,
                     top=0 if train else rng.choice([0, 1, 5, 20]), scale=rng.choice([1.0, 0.7]), train=train,
                     pad=rng.choice([0, 0, 24]), none=rng.choice([0.0, 0.3]))
        else:
            c = dict(op=op, d=_log(rng, 24, 2048), ff=_log(rng, 64, 5632), layers=rng.randint(1, 16),
                     vocab=rng.choice([0, 10007, 32000]), dtype=dt, clip=rng.choice([0.1, 0.9, 2.0]))
        if 3072 not in c.values() and _cost(c) <= limit:
            return c


def _ids(g, T, V, none):
    """Token ids whose frequency falls with their rank, as text's do; a share `none` is -1."""
    u = torch.rand(T, generator=g, device="cuda")
    ids = (torch.exp(u * math.log(V + 1.0)) - 1.0).long().clamp_(0, V - 1)
    if none:
        ids[torch.rand(T, generator=g, device="cuda") < none] = -1
    return ids


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dt, op = _DT[case["dtype"]], case["op"]

    def randn(*shape, std=1.0):
        return torch.randn(shape, generator=g, device="cuda") * std

    st = {"case": case}
    if op == "embed":
        T, V, D = case["T"], case["V"], case["D"]
        st["weight"] = randn(V, D, std=0.02).to(dt)
        st["ids"] = _ids(g, T, V, case["none"])
        if case["train"]:
            st["dy"] = randn(T, D, std=2.0 ** -6).to(dt)
    elif op == "ffn":
        T, D, F = case["T"], case["D"], case["F"]
        st["x"] = randn(T, D).to(dt)
        st["wg"], st["wu"] = randn(D, F, std=0.7 / math.sqrt(D)).to(dt), randn(D, F, std=0.7 / math.sqrt(D)).to(dt)
        if case["train"]:
            st["dh"] = randn(T, F, std=2.0 ** -6).to(dt)
    elif op == "logp":
        T, V = case["T"], case["V"]
        full = torch.empty(T, V + case["pad"], dtype=dt, device="cuda")
        for r in range(0, T, 1024):
            n = min(1024, T - r)
            z = randn(n, V + case["pad"], std=2.0)
            # a few tokens stand out in most rows, as a trained model's do
            z.scatter_add_(1, torch.randint(0, V, (n, 8), generator=g, device="cuda"), randn(n, 8, std=5.0).abs())
            full[r:r + n] = z.to(dt)
        st["logits"] = full[:, :V]
        st["logits"][:, V - V // 100:] = -math.inf  # rows of the head that no token uses
        st["targets"] = torch.randint(0, max(1, V - V // 100), (T,), generator=g, device="cuda")
        if case["none"]:
            st["targets"][torch.rand(T, generator=g, device="cuda") < case["none"]] = -1
        if case["train"]:
            # weighted log likelihoods and an entropy bonus, times a loss scale
            st["g_logp"] = -(randn(T).abs() + 0.1)
            st["g_entropy"] = randn(T, std=0.1)
    else:
        shapes = _shapes(case)
        n = sum(math.prod(s) for s in shapes)
        flat, out = randn(n, std=1e-3).to(dt), torch.empty(n, dtype=dt, device="cuda")
        cut = [math.prod(s) for s in shapes]
        st["grads"] = [v.view(s) for v, s in zip(flat.split(cut), shapes)]
        st["out"] = [v.view(s) for v, s in zip(out.split(cut), shapes)]
        st["flat"] = out  # all of "out", one after the other
        st["max_norm"] = case["clip"] * 1e-3 * math.sqrt(n)
    return st


# ------------------------------------------------------------------ the framework's operators

def _run_own(st):
    from paper_2607_03011_gb300 import inner

    case = st["case"]
    op = case["op"]
    if op == "embed":
        y = inner.embed(st["weight"], st["ids"], scale=case["scale"])
        if not case["train"]:
            return {"y": y}
        return {"y": y, "dw": inner.embed_grad(st["dy"], st["ids"], case["V"], scale=case["scale"])}
    if op == "ffn":
        if not case["train"]:
            return {"h": inner.gated_ffn(st["x"], st["wg"], st["wu"], act=case["act"])}
        h, saved = inner.gated_ffn(st["x"], st["wg"], st["wu"], act=case["act"], save=True)
        dx, dwg, dwu = inner.gated_ffn_grad(st["dh"], st["x"], st["wg"], st["wu"], saved, act=case["act"])
        return {"h": h, "dx": dx, "dwg": dwg, "dwu": dwu}
    if op == "logp":
        if case["train"]:
            r = inner.token_logprobs(st["logits"], st["targets"], scale=case["scale"], grad_logp=st["g_logp"],
                                     grad_entropy=st["g_entropy"])
            return {"logp": r.logp, "entropy": r.entropy, "dlogits": r.grad_logits}
        r = inner.token_logprobs(st["logits"], st["targets"], scale=case["scale"], top=case["top"])
        o = {"logp": r.logp, "entropy": r.entropy}
        if case["top"]:
            o.update(top_logp=r.top_logp, top_index=r.top_index)
        return o
    norm = inner.clip_grads(st["grads"], st["max_norm"], out=st["out"])
    return {"norm": norm, "grads": st["flat"]}


# ------------------------------------------------------------------ their plain forms

def _act(g, kind):
    if kind == "silu":
        return g * torch.sigmoid(g)
    return 0.5 * g * (1.0 + torch.tanh(0.7978845608028654 * (g + 0.044715 * g * g * g)))


def _act_grad(g, kind):
    if kind == "silu":
        s = torch.sigmoid(g)
        return s * (1.0 + g * (1.0 - s))
    t = torch.tanh(0.7978845608028654 * (g + 0.044715 * g * g * g))
    return 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * 0.7978845608028654 * (1.0 + 0.134145 * g * g)


def _ordered(x):
    """fp32 values as whole numbers of the same order."""
    x = torch.where(x == 0, torch.zeros_like(x), x)  # -0 and 0 are equal
    i = x.view(torch.int32).long()
    return torch.where(i < 0, -(i & 0x7FFFFFFF), i)


def _run_plain(st):
    case = st["case"]
    op, dt = case["op"], _DT[case["dtype"]]
    if op == "embed":
        ids = st["ids"]
        ok = (ids >= 0) & (ids < case["V"])
        w = st["weight"][ids.clamp(0, case["V"] - 1)].float()
        o = {"y": (w * case["scale"] * ok[:, None]).to(dt)}
        if case["train"]:
            dw = torch.zeros(case["V"], case["D"], device="cuda")
            dw.index_add_(0, ids.clamp(0, case["V"] - 1), st["dy"].float() * ok[:, None])
            o["dw"] = (dw * case["scale"]).to(dt)
        return o
    if op == "ffn":
        x, wg, wu = st["x"].float(), st["wg"].float(), st["wu"].float()
        g, u = x @ wg, x @ wu
        a = _act(g, case["act"])
        o = {"h": (a * u).to(dt)}
        if case["train"]:
            dh = st["dh"].float()
            du, dg = dh * a, dh * u * _act_grad(g, case["act"])
            o["dx"] = (dg @ wg.t() + du @ wu.t()).to(dt)
            o["dwg"], o["dwu"] = (x.t() @ dg).to(dt), (x.t() @ du).to(dt)
        return o
    if op == "logp":
        V, t = case["V"], st["targets"]
        given = (t >= 0) & (t < V)
        x = st["logits"].float() * case["scale"]
        m = x.amax(1, keepdim=True)
        e = torch.exp(x - m)
        s = e.sum(1, keepdim=True)
        lse = m + torch.log(s)
        lp = x - lse
        p = e / s
        plp = torch.where(p > 0, p * lp, torch.zeros_like(p))
        ent = -plp.sum(1)
        tt = t.clamp(0, V - 1)[:, None]
        o = {"logp": torch.where(given, lp.gather(1, tt)[:, 0], torch.zeros_like(ent)), "entropy": ent}
        if case["top"]:
            # the lowest index among equal logits comes first
            key = _ordered(st["logits"].float()) * 2 ** 24 + (V - 1 - torch.arange(V, device="cuda"))
            idx = key.topk(case["top"], dim=1).indices
            o["top_logp"], o["top_index"] = lp.gather(1, idx), idx
        if case["train"]:
            gl = torch.where(given, st["g_logp"], torch.zeros_like(ent))[:, None]
            d = -gl * p - st["g_entropy"][:, None] * (plp + p * ent[:, None])
            d.scatter_add_(1, tt, gl)
            o["dlogits"] = (d * case["scale"]).to(dt)
        return o
    total = torch.zeros((), device="cuda")
    for v in st["grads"]:
        total = total + (v.float() * v.float()).sum()
    norm = torch.sqrt(total)
    coef = torch.clamp(st["max_norm"] / norm, max=1.0)
    for o, v in zip(st["out"], st["grads"]):
        o.copy_((v.float() * coef).to(dt))
    return {"norm": norm, "grads": st["flat"]}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------ the definitions in 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    op, sc = case["op"], float(torch.tensor(case.get("scale", 1.0), dtype=torch.float32))
    if op == "embed":
        ids, V = st["ids"], case["V"]
        table = torch.cat([st["weight"].double() * sc, torch.zeros(1, case["D"], device="cuda").double()])
        row = torch.where((ids < 0) | (ids >= V), torch.full_like(ids, V), ids)
        o = {"y": table[row]}
        if case["train"]:
            dw = torch.zeros_like(table)
            dw.index_put_((row,), st["dy"].double() * sc, accumulate=True)
            o["dw"] = dw[:V]
        return o
    if op == "ffn":
        x, wg, wu = st["x"].double(), st["wg"].double(), st["wu"].double()
        if case["train"]:
            for v in (x, wg, wu):
                v.requires_grad_(True)
        g, u = x.mm(wg), x.mm(wu)
        if case["act"] == "silu":
            a = torch.nn.functional.silu(g)
        else:
            a = torch.nn.functional.gelu(g, approximate="tanh")
        h = a * u
        o = {"h": h.detach()}
        if case["train"]:
            o["dx"], o["dwg"], o["dwu"] = torch.autograd.grad(h, (x, wg, wu), st["dh"].double())
        return o
    if op == "logp":
        V, parts = case["V"], []
        for r in range(0, case["T"], 1024):  # rows are independent
            z = st["logits"][r:r + 1024].double()
            t = st["targets"][r:r + 1024]
            given = (t >= 0) & (t < V)
            if case["train"]:
                z.requires_grad_(True)
            lp = torch.log_softmax(z * sc, 1)
            p = lp.exp()
            ent = -(p * lp.clamp(min=-1e300)).sum(1)
            logp = lp.gather(1, t.clamp(0, V - 1)[:, None])[:, 0] * given
            part = [logp.detach(), ent.detach()]
            if case["top"]:
                order = torch.sort(z.detach(), dim=1, descending=True, stable=True).indices[:, :case["top"]]
                part += [lp.gather(1, order), order]
            if case["train"]:
                # gradients of the row's log probability and entropy, from their definitions
                with torch.no_grad():
                    gl = (st["g_logp"][r:r + 1024].double() * given)[:, None]
                    ge = st["g_entropy"][r:r + 1024].double()[:, None]
                    hot = torch.zeros_like(p).scatter_(1, t.clamp(0, V - 1)[:, None], 1.0)
                    part.append(sc * (gl * (hot - p) - ge * p * (lp.clamp(min=-1e300) + ent[:, None])))
            parts.append(part)
        cols = [torch.cat(c) for c in zip(*parts)]
        names = ["logp", "entropy"] + (["top_logp", "top_index"] if case["top"] else [])
        return dict(zip(names + (["dlogits"] if case["train"] else []), cols))
    norm = math.sqrt(sum(float(v.double().square().sum()) for v in st["grads"]))
    coef = min(1.0, st["max_norm"] / norm)
    return {"norm": torch.tensor(norm, dtype=torch.float64, device="cuda"),
            "grads": torch.cat([v.double().reshape(-1) for v in st["grads"]]) * coef}
