"""Operators of a worker's inner step, over the C ABI of libisoloco (include/isoloco.h).

Between two outer steps a worker looks tokens up in its embedding (`embed`), runs gated feed-forward
blocks (`gated_ffn`), scores the next tokens from the head's logits (`token_logprobs`) and clips the
global norm of its gradient (`clip_grads`); the `*_grad` functions are the backward passes.

Argument marshalling only, as in `isoloco`: tensors are torch CUDA tensors on the current device, in
fp32, bf16 or fp16 (the gated block: bf16 or fp16), whose last dimension is contiguous; other strides
are free as long as the leading dimensions fold into one.  Work is enqueued on `stream` (default: the
current stream); outputs and workspaces are allocated there.  Inputs made on another stream have to be
ordered before the call by the caller.  Bad arguments raise ValueError (shapes and types) or
IsolocoError (what the library refuses) before anything is launched.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional, Sequence

import torch

from . import isoloco
from .isoloco import IsolocoError, Tensor, _check, lib  # noqa: F401  (IsolocoError: what these functions raise)

_DTYPE = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_ACT = {"silu": 0, "gelu_tanh": 1}
MAX_TOP = 32


class _On:
    """The call's stream: its handle, and the place where its outputs are allocated."""

    def __init__(self, stream):
        if stream is None:
            self.ctx, self.handle = None, torch.cuda.current_stream().cuda_stream
        else:
            if not hasattr(stream, "cuda_stream"):
                stream = torch.cuda.ExternalStream(int(stream))
            self.ctx, self.handle = torch.cuda.stream(stream), stream.cuda_stream

    def empty(self, shape, dtype, device):
        if self.ctx is None:
            return torch.empty(shape, dtype=dtype, device=device)
        with self.ctx:
            return torch.empty(shape, dtype=dtype, device=device)


def _rows(t: torch.Tensor, what: str, like: Optional[torch.Tensor] = None):
    """(t as rows x columns, pitch): leading dimensions folded, without a copy."""
    if not t.is_cuda or t.dtype not in _DTYPE:
        raise ValueError(f"{what}: a CUDA tensor of fp32, bf16 or fp16 is needed")
    if like is not None and (t.dtype != like.dtype or t.device != like.device):
        raise ValueError(f"{what}: type or device differs from the other operands'")
    if t.dim() < 1 or t.shape[-1] == 0:
        raise ValueError(f"{what}: at least one column is needed")
    if t.dim() != 2:
        n = t.shape[-1]
        try:
            t = t.view(t.numel() // n, n)
        except RuntimeError:
            raise ValueError(f"{what}: the leading dimensions do not fold into rows of one pitch") from None
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{what}: the last dimension must be contiguous")
    ld = t.stride(0) if t.shape[0] > 1 else t.shape[1]
    if ld < t.shape[1]:
        raise ValueError(f"{what}: rows overlap")
    return t, ld


def _tokens(ids: torch.Tensor, what: str, count: Optional[int] = None) -> torch.Tensor:
    if not ids.is_cuda or ids.dtype not in (torch.int32, torch.int64):
        raise ValueError(f"{what}: a CUDA tensor of int32 or int64 is needed")
    if not ids.is_contiguous():
        raise ValueError(f"{what}: must be contiguous")
    if count is not None and ids.numel() != count:
        raise ValueError(f"{what}: {count} entries expected, got {ids.numel()}")
    return ids


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def embed(weight: torch.Tensor, ids: torch.Tensor, scale: float = 1.0, stream=None) -> torch.Tensor:
    """scale * weight[ids] (vocab x width by ids of any shape); zeros where an id is outside
    [0, vocab)."""
    w, ld = _rows(weight, "weight")
    ids = _tokens(ids, "ids")
    on = _On(stream)
    vocab, width = w.shape
    y = on.empty(ids.shape + (width,), w.dtype, w.device)
    _check(lib().isoloco_embed(w.data_ptr(), ld, _DTYPE[w.dtype], vocab, width, ids.data_ptr(), ids.element_size(),
                               ids.numel(), scale, y.data_ptr(), width, on.handle), "isoloco_embed")
    return y


def embed_grad(grad: torch.Tensor, ids: torch.Tensor, vocab: int, scale: float = 1.0, dtype=None,
               stream=None) -> torch.Tensor:
    """The lookup's gradient by the whole table (vocab x width, of `dtype`: grad's or fp32), from
    grad = d loss / d embed(weight, ids, scale)."""
    dy, ld = _rows(grad, "grad")
    ids = _tokens(ids, "ids", dy.shape[0])
    dtype = dtype or dy.dtype
    if dtype not in (dy.dtype, torch.float32):
        raise ValueError("dtype: grad's type or fp32")
    on = _On(stream)
    L, width, n = lib(), dy.shape[1], dy.shape[0]
    dw = on.empty((vocab, width), dtype, dy.device)
    need = L.isoloco_embed_grad_workspace(vocab, width, n)
    if need < 0:
        raise ValueError("vocab must be in 1 .. 2^31 - 1")
    ws = on.empty(need, torch.uint8, dy.device)
    _check(L.isoloco_embed_grad(dy.data_ptr(), ld, _DTYPE[dy.dtype], vocab, width, ids.data_ptr(), ids.element_size(), n,
                                scale, dw.data_ptr(), width, _DTYPE[dtype], ws.data_ptr(), need, on.handle),
           "isoloco_embed_grad")
    return dw


def _rows16(t: torch.Tensor, ld: int) -> bool:
    return t.data_ptr() % 16 == 0 and ld % 8 == 0


def _ffn_operands(x, w_gate, w_up, act):
    x2, ldx = _rows(x, "x")
    wg, ldg = _rows(w_gate, "w_gate", x2)
    wu, ldu = _rows(w_up, "w_up", x2)
    if x2.dtype == torch.float32:
        raise ValueError("x: the gated block takes bf16 or fp16")
    if wg.shape != wu.shape or wg.shape[0] != x2.shape[1]:
        raise ValueError(f"w_gate, w_up: width x ff matrices expected for width {x2.shape[1]}")
    if ldg != ldu:
        raise ValueError("w_gate and w_up must have the same pitch")
    if act not in _ACT:
        raise ValueError(f"act: one of {sorted(_ACT)}")
    aligned = _rows16(x2, ldx) and _rows16(wg, ldg) and _rows16(wu, ldg) and (x2.shape[1] | wg.shape[1]) % 8 == 0
    return x2, ldx, wg, wu, ldg, _ACT[act], aligned


def gated_ffn(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, act: str = "silu", save: bool = False,
              stream=None):
    """h = act(x w_gate) * (x w_up); w_gate and w_up are width x ff.  With save=True returns
    (h, saved), where `saved` is what gated_ffn_grad needs besides the operands."""
    x2, ldx, wg, wu, ldw, code, aligned = _ffn_operands(x, w_gate, w_up, act)
    on = _On(stream)
    L, (n, width), ff = lib(), x2.shape, wg.shape[1]
    h = on.empty(x.shape[:-1] + (ff,), x.dtype, x.device)
    saved = on.empty(L.isoloco_gated_ffn_saved_bytes(n, ff, _DTYPE[x.dtype]), torch.uint8, x.device) if save else None
    need = L.isoloco_gated_ffn_workspace(n, width, ff, aligned)
    ws = on.empty(need, torch.uint8, x.device)
    _check(L.isoloco_gated_ffn(x2.data_ptr(), ldx, wg.data_ptr(), wu.data_ptr(), ldw, _DTYPE[x.dtype], n, width, ff, code,
                               h.data_ptr(), ff, _ptr(saved), ws.data_ptr(), need, on.handle), "isoloco_gated_ffn")
    return (h, saved) if save else h


def gated_ffn_grad(grad: torch.Tensor, x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, saved: torch.Tensor,
                   act: str = "silu", need_x: bool = True, need_w: bool = True, stream=None):
    """(dx, dw_gate, dw_up) for grad = d loss / d h; None for what is not needed."""
    x2, ldx, wg, wu, ldw, code, aligned = _ffn_operands(x, w_gate, w_up, act)
    dh, ldh = _rows(grad, "grad", x2)
    L, (n, width), ff = lib(), x2.shape, wg.shape[1]
    if dh.shape != (n, ff):
        raise ValueError(f"grad: {n} rows of {ff} expected")
    if saved.dtype != torch.uint8 or not saved.is_contiguous() or saved.device != x.device or \
            saved.numel() != L.isoloco_gated_ffn_saved_bytes(n, ff, _DTYPE[x.dtype]):
        raise ValueError("saved: not what gated_ffn(save=True) returned for these sizes")
    on = _On(stream)
    dx = on.empty(x.shape, x.dtype, x.device) if need_x else None
    dwg = on.empty((width, ff), x.dtype, x.device) if need_w else None
    dwu = on.empty((width, ff), x.dtype, x.device) if need_w else None
    need = L.isoloco_gated_ffn_grad_workspace(n, width, ff, aligned)
    ws = on.empty(need, torch.uint8, x.device)
    _check(L.isoloco_gated_ffn_grad(dh.data_ptr(), ldh, x2.data_ptr(), ldx, wg.data_ptr(), wu.data_ptr(), ldw,
                                    _DTYPE[x.dtype], n, width, ff, code, saved.data_ptr(), _ptr(dx), width, _ptr(dwg),
                                    _ptr(dwu), ff, ws.data_ptr(), need, on.handle), "isoloco_gated_ffn_grad")
    return dx, dwg, dwu


class TokenLogprobs(NamedTuple):
    logp: torch.Tensor                     # fp32, one per row; 0 where the target is no token
    entropy: torch.Tensor                  # fp32, one per row
    lse: torch.Tensor                      # fp32, one per row
    top_logp: Optional[torch.Tensor]       # fp32, rows x top
    top_index: Optional[torch.Tensor]      # int64, rows x top
    grad_logits: Optional[torch.Tensor]    # of the logits' type and shape


def _per_row(t: Optional[torch.Tensor], n: int, what: str):
    if t is None:
        return None
    if not t.is_cuda or t.dtype != torch.float32 or not t.is_contiguous() or t.numel() != n:
        raise ValueError(f"{what}: {n} contiguous fp32 CUDA entries expected")
    return t.data_ptr()


def token_logprobs(logits: torch.Tensor, targets: torch.Tensor, scale: float = 1.0, top: int = 0,
                   grad_logp: Optional[torch.Tensor] = None, grad_entropy: Optional[torch.Tensor] = None,
                   stream=None) -> TokenLogprobs:
    """Log probability of each row's target under softmax(scale * logits), the rows' entropies and
    logarithms of the sum of exponentials, and the `top` likeliest tokens (ties: the lowest index).
    With grad_logp or grad_entropy (a gradient per row, known in advance as for a weighted sum of log
    probabilities) the same call returns the gradient by the logits."""
    z, ld = _rows(logits, "logits")
    n, vocab = z.shape
    targets = _tokens(targets, "targets", n)
    if not 0 <= top <= min(vocab, MAX_TOP):
        raise ValueError(f"top: 0 .. {min(vocab, MAX_TOP)}")
    gl, ge = _per_row(grad_logp, n, "grad_logp"), _per_row(grad_entropy, n, "grad_entropy")
    on = _On(stream)
    L, lead, dev = lib(), logits.shape[:-1], z.device
    stats = on.empty((3,) + lead, torch.float32, dev)
    logp, ent, lse = stats.unbind(0)
    tl = on.empty(lead + (top,), torch.float32, dev) if top else None
    ti = on.empty(lead + (top,), torch.int64, dev) if top else None
    want = grad_logp is not None or grad_entropy is not None
    gz = on.empty(logits.shape, z.dtype, dev) if want else None
    need = L.isoloco_token_logprobs_workspace(n, vocab, top)
    ws = on.empty(need, torch.uint8, dev)
    _check(L.isoloco_token_logprobs(z.data_ptr(), ld, _DTYPE[z.dtype], n, vocab, targets.data_ptr(), targets.element_size(),
                                    scale, logp.data_ptr(), ent.data_ptr(), lse.data_ptr(), top, _ptr(tl), _ptr(ti), gl, ge,
                                    _ptr(gz), vocab, ws.data_ptr(), need, on.handle), "isoloco_token_logprobs")
    return TokenLogprobs(logp, ent, lse, tl, ti, gz)


def token_logprobs_grad(logits: torch.Tensor, targets: torch.Tensor, lse: torch.Tensor, entropy: Optional[torch.Tensor],
                        grad_logp: Optional[torch.Tensor], grad_entropy: Optional[torch.Tensor], scale: float = 1.0,
                        stream=None) -> torch.Tensor:
    """The gradient by the logits alone, from the lse and entropy of token_logprobs (backward pass of
    an autograd step, where the rows' gradients come later)."""
    z, ld = _rows(logits, "logits")
    n, vocab = z.shape
    targets = _tokens(targets, "targets", n)
    on = _On(stream)
    gz = on.empty(logits.shape, z.dtype, z.device)
    _check(lib().isoloco_token_logprobs_grad(z.data_ptr(), ld, _DTYPE[z.dtype], n, vocab, targets.data_ptr(),
                                             targets.element_size(), scale, _per_row(lse, n, "lse"),
                                             _per_row(entropy, n, "entropy"), _per_row(grad_logp, n, "grad_logp"),
                                             _per_row(grad_entropy, n, "grad_entropy"), gz.data_ptr(), vocab, on.handle),
           "isoloco_token_logprobs_grad")
    return gz


def _tensor_list(tensors: Sequence[torch.Tensor], what: str):
    arr = (Tensor * max(1, len(tensors)))()
    for e, t in zip(arr, tensors):
        if not t.is_cuda or t.dtype not in _DTYPE or not t.is_contiguous():
            raise ValueError(f"{what}: contiguous CUDA tensors of fp32, bf16 or fp16 are needed")
        e.data, e.n, e.dtype = t.data_ptr(), t.numel(), _DTYPE[t.dtype]
    return arr


def grad_norm(grads: Sequence[torch.Tensor], stream=None) -> torch.Tensor:
    """The norm over all entries of all tensors, a 0-d fp32 tensor on the device."""
    grads = list(grads)
    arr = _tensor_list(grads, "grads")
    on = _On(stream)
    L, dev = lib(), grads[0].device if grads else torch.device("cuda")
    norm = on.empty((), torch.float32, dev)
    need = L.isoloco_grad_norm_workspace(len(grads))
    ws = on.empty(need, torch.uint8, dev)
    _check(L.isoloco_grad_norm(arr, len(grads), norm.data_ptr(), ws.data_ptr(), need, on.handle), "isoloco_grad_norm")
    return norm


def clip_grads(grads: Sequence[torch.Tensor], max_norm: float, out: Optional[Sequence[torch.Tensor]] = None,
               stream=None) -> torch.Tensor:
    """Scales the gradient by min(1, max_norm / norm), in place or into `out`, and returns the norm
    (0-d, fp32).  A NaN or infinite norm scales nothing."""
    grads = list(grads)
    arr = _tensor_list(grads, "grads")
    outs = None
    if out is not None:
        out = list(out)
        if len(out) != len(grads):
            raise ValueError("out: one tensor per gradient")
        outs = _tensor_list(out, "out")
    on = _On(stream)
    L, dev = lib(), grads[0].device if grads else torch.device("cuda")
    norm = on.empty((), torch.float32, dev)
    need = L.isoloco_grad_norm_workspace(len(grads))
    ws = on.empty(need, torch.uint8, dev)
    _check(L.isoloco_clip_grads(arr, outs, len(grads), max_norm, norm.data_ptr(), ws.data_ptr(), need, on.handle),
           "isoloco_clip_grads")
    return norm


def status(stream=None) -> int:
    """Waits for `stream`; 0, or isoloco.ERR_TIMEOUT if a kernel of these operators gave up a wait on
    the current device since the last call."""
    return lib().isoloco_inner_status(isoloco._stream(stream))
