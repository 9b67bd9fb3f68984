"""Operators of a worker's inner step, over the C ABI of libisoloco (include/isoloco.h).

Between two outer steps a worker looks tokens up in its embedding (`embed`), runs gated feed-forward
blocks (`gated_ffn`), scores the next tokens from the head's logits (`token_logprobs`) and clips the
global norm of its gradient (`clip_grads`); the `*_grad` functions are the backward passes.  A merged model also
teaches: from its top tokens, as `token_logprobs` gives them, another learns (`distill`).  And it answers: by a search over
beams (`beam_select`, `beam_reorder`).

Argument marshalling only, as in `isoloco`: tensors are torch CUDA tensors on the current device, in
fp32, bf16 or fp16 (the gated block: bf16 or fp16), whose last dimension is contiguous; other strides
are free as long as the leading dimensions fold into one.  Every function takes `stream` (default: the
current stream): work is enqueued and outputs and workspaces are allocated there.  Inputs made on another stream have to be
ordered before the call by the caller.  Bad arguments raise ValueError (shapes and types) or
IsolocoError (what the library refuses) before anything is launched.

Nothing here is recorded by autograd, as nothing in `isoloco` is: tensors that require a gradient are taken as they
are, outputs never require one, and a loss.backward() through them reaches no operand.  Gradients come from the
`*_grad` functions (and grad_logits of `token_logprobs` and `distill`) alone, called by the training step itself as `inner_demo`
does, or by a torch.autograd.Function around them.
"""
from __future__ import annotations

import array
from typing import Iterable, List, NamedTuple, Optional

import torch

from . import isoloco
from .isoloco import IsolocoError, _check, lib  # noqa: F401  (IsolocoError: what these functions raise)

_DTYPE = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_HALF = {torch.bfloat16: 1, torch.float16: 2}
_ACT = {"silu": 0, "gelu_tanh": 1}
_INT = {torch.int32: 4, torch.int64: 8}
_TAIL = {"drop": 0, "rest": 1}
MAX_TOP = 32
MAX_LIST = 256
MAX_BEAMS = 32

# The smallest of these calls take a few microseconds on the GPU, so the way there is kept short: the
# current stream's handle and the device's number without objects made for them, where torch has these names.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_empty = torch.empty
_data_ptr, _numel = torch.Tensor.data_ptr, torch.Tensor.numel
_is_contiguous, _get_device = torch.Tensor.is_contiguous, torch.Tensor.get_device
_stride = torch.Tensor.stride


def _on(stream, f, *args):
    """The call f(*args) with `stream` as the current stream: its outputs and workspaces are allocated there, and
    inputs freed before it has run are not given out again until then."""
    if not hasattr(stream, "cuda_stream"):
        stream = torch.cuda.ExternalStream(int(stream))
    for a in args:
        for t in a if isinstance(a, (list, tuple)) else (a,):
            if isinstance(t, torch.Tensor) and t.is_cuda:
                t.record_stream(stream)
    with torch.cuda.stream(stream):
        return f(*args)


def _rows(t: torch.Tensor, what: str, dtypes=_DTYPE):
    """(t as rows x columns, rows, columns, pitch): leading dimensions folded, without a copy."""
    if t.dtype not in dtypes or t.get_device() != _current_device():
        names = ", ".join(str(d).replace("torch.", "") for d in dtypes)
        raise ValueError(f"{what}: a tensor of {names} on the current CUDA device is needed")
    shape = t.shape
    if len(shape) != 2:
        if len(shape) < 1 or shape[-1] == 0:
            raise ValueError(f"{what}: at least one column is needed")
        n = shape[-1]
        try:
            t = t.view(t.numel() // n, n)
        except RuntimeError:
            raise ValueError(f"{what}: the leading dimensions do not fold into rows of one pitch") from None
        shape = t.shape
    rows, cols = shape
    ld, step = t.stride()
    if cols == 0:
        raise ValueError(f"{what}: at least one column is needed")
    if step != 1 and cols > 1:
        raise ValueError(f"{what}: the last dimension must be contiguous")
    if rows < 2:
        ld = cols
    elif ld < cols:
        raise ValueError(f"{what}: rows overlap")
    return t, rows, cols, ld


def _tokens(ids: torch.Tensor, what: str, count: Optional[int] = None) -> int:
    """The ids' element size."""
    size = _INT.get(ids.dtype)
    if size is None or ids.get_device() != _current_device():
        raise ValueError(f"{what}: a tensor of int32 or int64 on the current CUDA device is needed")
    if not ids.is_contiguous():
        raise ValueError(f"{what}: must be contiguous")
    if count is not None and ids.numel() != count:
        raise ValueError(f"{what}: {count} entries expected, got {ids.numel()}")
    return size


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _buffer(need: int, what: str, dev):
    """Uninitialised bytes, as many as `what` asked for (none: None); what it refuses raises."""
    if need < 0:
        _check(need, what)
    return _empty(need, dtype=torch.uint8, device=dev) if need else None


def embed(weight: torch.Tensor, ids: torch.Tensor, scale: float = 1.0, stream=None) -> torch.Tensor:
    """scale * weight[ids] (vocab x width by ids of any shape); zeros where an id is outside
    [0, vocab)."""
    if stream is not None:
        return _on(stream, embed, weight, ids, scale)
    w, vocab, width, ld = _rows(weight, "weight")
    size = _tokens(ids, "ids")
    dev = w.device
    y = _empty((*ids.shape, width), dtype=w.dtype, device=dev)
    rc = lib().isoloco_embed(w.data_ptr(), ld, _DTYPE[w.dtype], vocab, width, ids.data_ptr(), size, ids.numel(), scale,
                             y.data_ptr(), width, _raw_stream(dev.index))
    if rc:
        _check(rc, "isoloco_embed")
    return y


def embed_grad(grad: torch.Tensor, ids: torch.Tensor, vocab: int, scale: float = 1.0, dtype=None,
               stream=None) -> torch.Tensor:
    """The lookup's gradient by the whole table (vocab x width, of `dtype`: grad's or fp32), from
    grad = d loss / d embed(weight, ids, scale)."""
    if stream is not None:
        return _on(stream, embed_grad, grad, ids, vocab, scale, dtype)
    dy, n, width, ld = _rows(grad, "grad")
    size = _tokens(ids, "ids", n)
    dtype = dtype or dy.dtype
    if dtype not in (dy.dtype, torch.float32):
        raise ValueError("dtype: grad's type or fp32")
    L, dev = lib(), dy.device
    need = L.isoloco_embed_grad_workspace(vocab, width, n)
    ws = _buffer(need, "isoloco_embed_grad_workspace", dev)
    dw = _empty((vocab, width), dtype=dtype, device=dev)
    rc = L.isoloco_embed_grad(dy.data_ptr(), ld, _DTYPE[dy.dtype], vocab, width, ids.data_ptr(), size, n, scale,
                              dw.data_ptr(), width, _DTYPE[dtype], ws.data_ptr(), need, _raw_stream(dev.index))
    if rc:
        _check(rc, "isoloco_embed_grad")
    return dw


def _ffn_operands(x, w_gate, w_up, act):
    """x's rows, their number, width, ff, pitches, the activation's code, and whether all addresses and
    pitches, outputs' included, are multiples of 16 bytes."""
    x2, n, width, ldx = _rows(x, "x", _HALF)
    wg, rows, ff, ldw = _rows(w_gate, "w_gate", _HALF)
    wu, rows_u, ff_u, ldu = _rows(w_up, "w_up", _HALF)
    if wg.dtype != x2.dtype or wu.dtype != x2.dtype:
        raise ValueError("x, w_gate and w_up must be of one type")
    if rows != width or rows_u != width or ff != ff_u:
        raise ValueError(f"w_gate, w_up: width x ff matrices expected for width {width}")
    if ldw != ldu and rows > 1:
        raise ValueError("w_gate and w_up must have the same pitch")
    if act not in _ACT:
        raise ValueError(f"act: one of {sorted(_ACT)}")
    px, pg, pu = x2.data_ptr(), wg.data_ptr(), wu.data_ptr()
    aligned = (px | pg | pu) % 16 == 0 and (ldx | ldw | width | ff) % 8 == 0
    return n, width, ff, (px, ldx, pg, pu, ldw, _HALF[x2.dtype], n, width, ff, _ACT[act]), aligned


def gated_ffn(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, act: str = "silu", save: bool = False,
              stream=None):
    """h = act(x w_gate) * (x w_up); w_gate and w_up are width x ff.  With save=True returns
    (h, saved), where `saved` is what gated_ffn_grad needs besides the operands."""
    if stream is not None:
        return _on(stream, gated_ffn, x, w_gate, w_up, act, save)
    n, width, ff, args, aligned = _ffn_operands(x, w_gate, w_up, act)
    L, dev, dt = lib(), x.device, x.dtype
    saved = _buffer(L.isoloco_gated_ffn_saved_bytes(n, ff, _HALF[dt]), "isoloco_gated_ffn_saved_bytes", dev) if save else None
    need = 0 if aligned else L.isoloco_gated_ffn_workspace(n, width, ff, 0)
    ws = _buffer(need, "isoloco_gated_ffn_workspace", dev)
    h = _empty((*x.shape[:-1], ff), dtype=dt, device=dev)
    rc = L.isoloco_gated_ffn(*args, h.data_ptr(), ff, _ptr(saved), _ptr(ws), need, _raw_stream(dev.index))
    if rc:
        _check(rc, "isoloco_gated_ffn")
    return (h, saved) if save else h


def gated_ffn_grad(grad: torch.Tensor, x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, saved: torch.Tensor,
                   act: str = "silu", need_x: bool = True, need_w: bool = True, stream=None):
    """(dx, dw_gate, dw_up) for grad = d loss / d h; None for what is not needed."""
    if stream is not None:
        return _on(stream, gated_ffn_grad, grad, x, w_gate, w_up, saved, act, need_x, need_w)
    n, width, ff, args, aligned = _ffn_operands(x, w_gate, w_up, act)
    dh, rows, cols, ldh = _rows(grad, "grad", _HALF)
    L, dev, dt = lib(), x.device, x.dtype
    if dh.dtype != dt or rows != n or cols != ff:
        raise ValueError(f"grad: {n} rows of {ff} of x's type expected")
    need = L.isoloco_gated_ffn_grad_workspace(n, width, ff, aligned)
    _check(need, "isoloco_gated_ffn_grad_workspace")
    if saved.dtype != torch.uint8 or not saved.is_contiguous() or saved.device != dev or \
            saved.numel() != L.isoloco_gated_ffn_saved_bytes(n, ff, _HALF[dt]):
        raise ValueError("saved: not what gated_ffn(save=True) returned for these sizes")
    dx = _empty(x.shape, dtype=dt, device=dev) if need_x else None
    dwg = _empty((width, ff), dtype=dt, device=dev) if need_w else None
    dwu = _empty((width, ff), dtype=dt, device=dev) if need_w else None
    ws = _buffer(need, "isoloco_gated_ffn_grad_workspace", dev)
    rc = L.isoloco_gated_ffn_grad(dh.data_ptr(), ldh, *args, saved.data_ptr(), _ptr(dx), width, _ptr(dwg), _ptr(dwu),
                                  ff, _ptr(ws), need, _raw_stream(dev.index))
    if rc:
        _check(rc, "isoloco_gated_ffn_grad")
    return dx, dwg, dwu


class TokenLogprobs(NamedTuple):
    logp: torch.Tensor                     # fp32, one per row; 0 where the target is no token
    entropy: torch.Tensor                  # fp32, one per row
    lse: torch.Tensor                      # fp32, one per row
    top_logp: Optional[torch.Tensor]       # fp32, rows x top
    top_index: Optional[torch.Tensor]      # int64, rows x top
    grad_logits: Optional[torch.Tensor]    # of the logits' type and shape; rows a little apart where the logits' are


def _per_row(t: Optional[torch.Tensor], n: int, what: str):
    if t is None:
        return None
    if t.dtype != torch.float32 or t.get_device() != _current_device() or not t.is_contiguous() or t.numel() != n:
        raise ValueError(f"{what}: {n} contiguous fp32 entries on the current CUDA device expected")
    return t.data_ptr()


def _like_rows(z, shape, vocab, ld, dev):
    """(an empty tensor of the logits' shape, its pitch): the smallest pitch with which rows start as far from a
    16-byte boundary as the logits' do (both are then read and written 16 bytes at a time)."""
    pitch = vocab + (ld - vocab) % (16 // z.element_size())
    if pitch == vocab:
        return _empty(shape, dtype=z.dtype, device=dev), vocab
    return _empty((*shape[:-1], pitch), dtype=z.dtype, device=dev)[..., :vocab], pitch


def token_logprobs(logits: torch.Tensor, targets: torch.Tensor, scale: float = 1.0, top: int = 0,
                   grad_logp: Optional[torch.Tensor] = None, grad_entropy: Optional[torch.Tensor] = None,
                   stream=None) -> TokenLogprobs:
    """Log probability of each row's target under softmax(scale * logits), the rows' entropies and
    logarithms of the sum of exponentials, and the `top` likeliest tokens (ties: the lowest index).
    With grad_logp or grad_entropy (a gradient per row, known in advance as for a weighted sum of log
    probabilities) the same call returns the gradient by the logits."""
    if stream is not None:
        return _on(stream, token_logprobs, logits, targets, scale, top, grad_logp, grad_entropy)
    z, n, vocab, ld = _rows(logits, "logits")
    size = _tokens(targets, "targets", n)
    if not 0 <= top <= min(vocab, MAX_TOP):
        raise ValueError(f"top: 0 .. {min(vocab, MAX_TOP)}")
    gl, ge = _per_row(grad_logp, n, "grad_logp"), _per_row(grad_entropy, n, "grad_entropy")
    shape, dev = logits.shape, z.device
    lead = shape[:-1]
    logp = _empty(lead, dtype=torch.float32, device=dev)
    ent = _empty(lead, dtype=torch.float32, device=dev)
    lse = _empty(lead, dtype=torch.float32, device=dev)
    tl = _empty((*lead, top), dtype=torch.float32, device=dev) if top else None
    ti = _empty((*lead, top), dtype=torch.int64, device=dev) if top else None
    gz, ldg = _like_rows(z, shape, vocab, ld, dev) if gl is not None or ge is not None else (None, ld)
    rc = lib().isoloco_token_logprobs(z.data_ptr(), ld, _DTYPE[z.dtype], n, vocab, targets.data_ptr(), size, scale,
                                      logp.data_ptr(), ent.data_ptr(), lse.data_ptr(), top, _ptr(tl), _ptr(ti), gl, ge,
                                      _ptr(gz), ldg, _raw_stream(dev.index))
    if rc:
        _check(rc, "isoloco_token_logprobs")
    return TokenLogprobs(logp, ent, lse, tl, ti, gz)


def token_logprobs_grad(logits: torch.Tensor, targets: torch.Tensor, lse: torch.Tensor, entropy: Optional[torch.Tensor],
                        grad_logp: Optional[torch.Tensor], grad_entropy: Optional[torch.Tensor],
                        scale: float = 1.0, stream=None) -> torch.Tensor:
    """The gradient by the logits alone, from the lse and entropy of token_logprobs (backward pass of
    an autograd step, where the rows' gradients come later)."""
    if stream is not None:
        return _on(stream, token_logprobs_grad, logits, targets, lse, entropy, grad_logp, grad_entropy, scale)
    z, n, vocab, ld = _rows(logits, "logits")
    size = _tokens(targets, "targets", n)
    dev = z.device
    gz, ldg = _like_rows(z, logits.shape, vocab, ld, dev)
    rc = lib().isoloco_token_logprobs_grad(z.data_ptr(), ld, _DTYPE[z.dtype], n, vocab, targets.data_ptr(), size, scale,
                                           _per_row(lse, n, "lse"), _per_row(entropy, n, "entropy"),
                                           _per_row(grad_logp, n, "grad_logp"),
                                           _per_row(grad_entropy, n, "grad_entropy"), gz.data_ptr(), ldg,
                                           _raw_stream(dev.index))
    if rc:
        _check(rc, "isoloco_token_logprobs_grad")
    return gz


class Distilled(NamedTuple):
    loss: torch.Tensor                     # fp32, one per row
    saved: Optional[torch.Tensor]          # fp32, rows x 6: what distill_grad needs besides the operands
    grad_logits: Optional[torch.Tensor]    # as of TokenLogprobs


def _distill_operands(logits, top_logp, top_index, tail):
    z, n, vocab, ld = _rows(logits, "logits")
    v, rows, k, ldv = _rows(top_logp, "top_logp")
    i, rows_i, k_i, ldi = _rows(top_index, "top_index", _INT)
    if rows != n or rows_i != n or k != k_i:
        raise ValueError(f"top_logp, top_index: {n} rows of one length expected")
    if k > MAX_LIST:
        raise ValueError(f"top_logp: at most {MAX_LIST} columns")
    code = _TAIL.get(tail)
    if code is None:
        raise ValueError(f"tail: one of {sorted(_TAIL)}")
    return z, n, vocab, ld, (v.data_ptr(), ldv, _DTYPE[v.dtype], i.data_ptr(), ldi, _INT[i.dtype], k), code


def distill(logits: torch.Tensor, top_logp: torch.Tensor, top_index: torch.Tensor, scale: float = 1.0, tail: str = "drop",
            grad_loss: Optional[torch.Tensor] = None, save: bool = False, stream=None) -> Distilled:
    """Each row's divergence KL(q || softmax(scale * logits)) from a teacher that is given by k tokens (top_index,
    int32 or int64; an index that is no token is no entry) and its log probabilities for them (top_logp), as
    token_logprobs(teacher_logits, ..., scale, top=k) returns them.  tail="drop" renormalises the teacher over the row's list;
    tail="rest" adds one outcome, any other token, with what the list leaves of the teacher's probability.  Entries of
    one token add up, so a target that is mixed in is one more entry with the logarithm of its weight.
    With grad_loss (the gradient by each row's loss, known in advance) the same call returns the gradient by the logits; with
    save=True what distill_grad needs."""
    if stream is not None:
        return _on(stream, distill, logits, top_logp, top_index, scale, tail, grad_loss, save)
    z, n, vocab, ld, lists, code = _distill_operands(logits, top_logp, top_index, tail)
    g = _per_row(grad_loss, n, "grad_loss")
    dev, shape = z.device, logits.shape
    loss = _empty(shape[:-1], dtype=torch.float32, device=dev)
    saved = _empty((n, 6), dtype=torch.float32, device=dev) if save else None
    gz, ldg = _like_rows(z, shape, vocab, ld, dev) if g is not None else (None, ld)
    rc = lib().isoloco_distill(z.data_ptr(), ld, _DTYPE[z.dtype], n, vocab, *lists, scale, code, loss.data_ptr(),
                               _ptr(saved), g, _ptr(gz), ldg, _raw_stream(dev.index))
    if rc:
        _check(rc, "isoloco_distill")
    return Distilled(loss, saved, gz)


def distill_grad(grad_loss: torch.Tensor, logits: torch.Tensor, top_logp: torch.Tensor, top_index: torch.Tensor,
                 saved: torch.Tensor, scale: float = 1.0, tail: str = "drop", stream=None) -> torch.Tensor:
    """The gradient by the logits alone, for grad_loss = d loss / d distill(...).loss and what the call saved."""
    if stream is not None:
        return _on(stream, distill_grad, grad_loss, logits, top_logp, top_index, saved, scale, tail)
    z, n, vocab, ld, lists, code = _distill_operands(logits, top_logp, top_index, tail)
    if grad_loss is None or saved is None:
        raise ValueError("grad_loss, saved: needed")
    g, kept = _per_row(grad_loss, n, "grad_loss"), _per_row(saved, 6 * n, "saved")
    dev = z.device
    gz, ldg = _like_rows(z, logits.shape, vocab, ld, dev)
    rc = lib().isoloco_distill_grad(g, z.data_ptr(), ld, _DTYPE[z.dtype], n, vocab, *lists, scale, code, kept,
                                    gz.data_ptr(), ldg, _raw_stream(dev.index))
    if rc:
        _check(rc, "isoloco_distill_grad")
    return gz


class BeamSelection(NamedTuple):
    scores: torch.Tensor                   # fp32, ... x keep, largest first
    beams: torch.Tensor                    # int64: the beam that each continues
    tokens: torch.Tensor                   # int64: with this token
    finished: Optional[torch.Tensor]       # bool: its beam was finished, or the token is `end` (None without `end`)


def beam_select(logits: torch.Tensor, scores: torch.Tensor, keep: Optional[int] = None,
                finished: Optional[torch.Tensor] = None, end: Optional[int] = None, scale: float = 1.0,
                stream=None) -> BeamSelection:
    """The `keep` (default: as many as beams) largest of scores[..., w] + log softmax(scale * logits[..., w, :])[t] over
    the beams w and tokens t of each batch entry; logits are ... x beams x vocab, scores fp32 ... x beams.  Ties: the lower
    beam, then the larger logit, then the lower token.  Beams where `finished` (bool) is set go on with the token `end` alone, at their own
    score.  A first step starts from one beam: scores of -inf for the others."""
    if stream is not None:
        return _on(stream, beam_select, logits, scores, keep, finished, end, scale)
    rows_of = logits.shape[:-1]
    if not rows_of:
        raise ValueError("logits: ... x beams x vocab expected")
    z, n, vocab, ld = _rows(logits, "logits")
    beams, dev = rows_of[-1], z.device
    if not 1 <= beams <= MAX_BEAMS:
        raise ValueError(f"logits: 1 .. {MAX_BEAMS} beams")
    if keep is None:
        keep = beams
    if not 1 <= keep <= min(beams * vocab, MAX_TOP):
        raise ValueError(f"keep: 1 .. {min(beams * vocab, MAX_TOP)}")
    if scores.shape != rows_of:
        raise ValueError("scores: one per row of logits expected")
    ps, pf, pe, code = _per_row(scores, n, "scores"), None, None, -1
    shape = (*rows_of[:-1], keep)
    f = None
    if end is not None:
        if not 0 <= end < vocab:
            raise ValueError(f"end: 0 .. {vocab - 1}")
        f = _empty(shape, dtype=torch.bool, device=dev)
        pe, code = f.data_ptr(), end
    if finished is not None:
        if finished.dtype != torch.bool or finished.shape != rows_of or not finished.is_contiguous() or \
                finished.get_device() != _current_device():
            raise ValueError("finished: contiguous bools on the current CUDA device expected, one per score")
        if end is None:
            raise ValueError("finished: needs the token `end`")
        pf = finished.data_ptr()
    s = _empty(shape, dtype=torch.float32, device=dev)
    b = _empty(shape, dtype=torch.int64, device=dev)
    t = _empty(shape, dtype=torch.int64, device=dev)
    rc = lib().isoloco_beam_select(z.data_ptr(), ld, _DTYPE[z.dtype], n // beams, beams, vocab, ps, pf, code, scale, keep,
                                   s.data_ptr(), b.data_ptr(), t.data_ptr(), pe, _raw_stream(dev.index))
    if rc:
        _check(rc, "isoloco_beam_select")
    return BeamSelection(s, b, t, f)


def _fold_state(shape, step, size: int, batch: int, width: int, two: bool, what: str, any_order: bool):
    """(strides in bytes of batch, beam and piece, pieces, bytes of a piece) of a state."""
    if two and len(shape) > 1 and shape[0] == batch and shape[1] == width:
        s_batch, s_beam, at = step[0], step[1], 2
    elif len(shape) > 0 and shape[0] == batch * width:
        s_batch, s_beam, at = width * step[0], step[0], 1
    else:
        raise ValueError(f"{what}: states of {batch} x {width} (or {batch * width}) beams expected")
    if 0 in shape:
        return 0, 0, 0, 0, 0
    run, outer, s_outer = 1, 1, 0
    dims = zip(step[:at - 1:-1], shape[:at - 1:-1])
    for s, n in sorted(dims) if any_order else dims:
        if n == 1:
            continue
        if outer == 1:
            if s == run:
                run *= n
            else:
                outer, s_outer = n, s
        elif s == outer * s_outer:
            outer *= n
        else:
            raise ValueError(f"{what}: a state's dimensions behind the beams' do not fold into pieces of one pitch")
    return s_batch * size, s_beam * size, s_outer * size, outer, run * size


def _fold_pair(shape, step, to_step, size: int, batch: int, width: int, two: bool):
    """The strides of a state and of its result, and the pieces of both."""
    same = step == to_step  # (the order of the dimensions is then free)
    sb, sw, so, n, run = _fold_state(shape, step, size, batch, width, two, "states", same)
    if same:
        return sb, sw, so, sb, sw, so, n, run
    db, dw, do, nd, rund = _fold_state(shape, to_step, size, batch, width, two, "out", False)
    if run != rund:
        # one of the two is in one piece where the other is in several: both in the shorter pieces
        short = min(run, rund)
        if (n > 1 and run != short) or (nd > 1 and rund != short):
            raise ValueError("out: the pieces of a state and of its result do not match")
        so, do = (so if run == short else short), (do if rund == short else short)
        n, run = n * run // short, short
    return sb, sw, so, db, dw, do, n, run


def beam_reorder(states: Iterable[torch.Tensor], beams: torch.Tensor, out: Optional[Iterable[torch.Tensor]] = None,
                 stream=None) -> List[torch.Tensor]:
    """state[b, w] = state[b, beams[b, w]] for what is kept for beams (caches, histories of tokens; any types), in place or
    into `out`; returns the list of results.  beams: batch x width (or width) of int32 or int64, an entry outside [0, width) stands for
    the beam itself.  States are batch x width x ... or (batch * width) x ...; the used part of a longer cache is given as a slice (of which the
    rest stays as it is).  Results may not share memory with one another or with states that they are not made in place of, and are lazily conjugated or
    negated views where the states are."""
    states, out = list(states), None if out is None else list(out)
    if stream is not None:
        return _on(stream, beam_reorder, states, beams, out)
    size = _tokens(beams, "beams")
    if beams.dim() not in (1, 2):
        raise ValueError("beams: batch x width (or width) entries expected")
    batch, width = (1, beams.shape[0]) if beams.dim() == 1 else beams.shape
    if not 1 <= width <= MAX_BEAMS:
        raise ValueError(f"beams: 1 .. {MAX_BEAMS} of a batch entry")
    if out is not None and len(out) != len(states):
        raise ValueError("out: one tensor per state")
    to, dev, two = states if out is None else out, _current_device(), beams.dim() == 2
    if set(map(_get_device, states)) - {dev} or set(map(_get_device, to)) - {dev}:
        raise ValueError("states, out: tensors on the current CUDA device are needed")
    types, shapes, steps = [t.dtype for t in states], [t.shape for t in states], list(map(_stride, states))
    to_steps = steps
    if out is not None:
        to_steps = list(map(_stride, out))
        if [t.dtype for t in out] != types or [t.shape for t in out] != shapes:
            raise ValueError("out: tensors of the states' shapes and types expected")
    # isoloco_state_t entries; a call's states are mostly alike, one after the other
    words, n, i = array.array("q"), len(states), 0
    while i < n:
        typ, shape, step, to_step = types[i], shapes[i], steps[i], to_steps[i]
        k = i + 1
        while k < n and types[k] is typ and steps[k] == step and shapes[k] == shape and to_steps[k] == to_step:
            k += 1
        words.extend(array.array("q", (0, 0, *_fold_pair(shape, step, to_step, typ.itemsize, batch, width, two))) * (k - i))
        # Bytes are moved: what torch conjugates or negates when it is read has to be so on both sides.  (Real tensors that are
        # negated so are imaginary parts, whose strides are even; asking each tensor costs 0.1 us.)
        if out is not None and (typ.is_complex or not step[-1] & to_step[-1] & 1) and \
                any(s.is_conj() != t.is_conj() or s.is_neg() != t.is_neg() for s, t in zip(states[i:k], out[i:k])):
            raise ValueError("out: conjugated or negated lazily where the states are not, or the other way round")
        i = k
    words[0::10] = array.array("q", map(_data_ptr, states))
    words[1::10] = array.array("q", map(_data_ptr, to))
    rc = lib().isoloco_beam_reorder(words.buffer_info()[0], len(states), batch, width, beams.data_ptr(), size, _raw_stream(dev))
    if rc:
        _check(rc, "isoloco_beam_reorder")
    return to


def _tensor_list(tensors: List[torch.Tensor], what: str):
    """isoloco_tensor_t entries (address, length, type) as 64-bit words."""
    codes = [_DTYPE.get(t.dtype, -1) for t in tensors]
    if -1 in codes or not all(map(_is_contiguous, tensors)) or set(map(_get_device, tensors)) - {_current_device()}:
        raise ValueError(f"{what}: contiguous tensors of fp32, bf16 or fp16 on the current CUDA device are needed")
    n = len(codes)
    words = array.array("q", bytes(24 * max(n, 1)))
    words[0:3 * n:3] = array.array("q", map(_data_ptr, tensors))
    words[1:3 * n:3] = array.array("q", map(_numel, tensors))
    words[2:3 * n:3] = array.array("q", codes)
    return words


def grad_norm(grads: Iterable[torch.Tensor], stream=None) -> torch.Tensor:
    """The norm over all entries of all tensors, a 0-d fp32 tensor on the device."""
    grads = list(grads)
    if stream is not None:
        return _on(stream, grad_norm, grads)
    words = _tensor_list(grads, "grads")
    L, n, dev, arr = lib(), len(grads), _current_device(), words.buffer_info()[0]
    need = L.isoloco_grad_norm_workspace(arr, n)
    ws = _buffer(need, "isoloco_grad_norm_workspace", dev)
    norm = _empty((), dtype=torch.float32, device=dev)
    rc = L.isoloco_grad_norm(arr, n, norm.data_ptr(), _ptr(ws), need, _raw_stream(dev))
    if rc:
        _check(rc, "isoloco_grad_norm")
    return norm


def clip_grads(grads: Iterable[torch.Tensor], max_norm: float, out: Optional[Iterable[torch.Tensor]] = None,
               stream=None) -> torch.Tensor:
    """Scales the gradient by min(1, max_norm / norm), in place or into `out`, and returns the norm
    (0-d, fp32).  A NaN or infinite norm scales nothing."""
    grads, out = list(grads), None if out is None else list(out)
    if stream is not None:
        return _on(stream, clip_grads, grads, max_norm, out)
    words, outs = _tensor_list(grads, "grads"), None
    if out is not None:
        if len(out) != len(grads):
            raise ValueError("out: one tensor per gradient")
        outs = _tensor_list(out, "out")
    L, n, dev, arr = lib(), len(grads), _current_device(), words.buffer_info()[0]
    need = L.isoloco_grad_norm_workspace(arr, n)
    ws = _buffer(need, "isoloco_grad_norm_workspace", dev)
    norm = _empty((), dtype=torch.float32, device=dev)
    rc = L.isoloco_clip_grads(arr, outs and outs.buffer_info()[0], n, max_norm, norm.data_ptr(), _ptr(ws), need,
                              _raw_stream(dev))
    if rc:
        _check(rc, "isoloco_clip_grads")
    return norm


def status(stream=None) -> int:
    """Waits for `stream`; 0, or isoloco.ERR_TIMEOUT if a kernel of these operators gave up a wait on
    the current device since the last call."""
    return lib().isoloco_inner_status(isoloco._stream(stream))
