"""Cross entropy of a linear head over a large vocabulary, with its gradients, over torch tensors.

A thin layer over ``ssgd_xent_forward`` and ``ssgd_xent_backward`` (``include/signsgd.h``) that allocates outputs and workspaces:
the logits are never in memory.  All work is enqueued on the current stream of the operands' device, whichever device is
current.
"""
from __future__ import annotations

import functools
import math
from typing import NamedTuple, Optional, Tuple

import torch

from . import binding as B
from .waits import check, status_of  # noqa: F401  (check: part of this module)

_DTYPES = B._Codes({torch.bfloat16: 1, torch.float16: 2}, TypeError, "h and w must be of dtype bfloat16 or float16")
_SMALL = 1 << 20
_stream_of, _current_device = B._stream_of, B._current_device
_pack_align, _pack_forward, _pack_backward = B.XENT_ALIGN_ARGS.pack, B.XENT_FORWARD_ARGS.pack, B.XENT_BACKWARD_ARGS.pack


@functools.lru_cache(maxsize=256)
def _sizes(index: int, tokens: int, vocab: int, width: int) -> Tuple[int, int]:
    """Workspace bytes of the two passes on a device; the caller has made it current."""
    return B.xent_sizes(tokens, vocab, width)


def _stride_as_it_is(t: torch.Tensor, width: int) -> int:
    """The row stride of a matrix whose rows asynchronous copies can read as they lie, starting at multiples of 16 bytes; else 0."""
    ld, step = t.stride()
    if (step == 1 or width == 1) and t.data_ptr() % 16 == 0:
        if t.shape[0] == 1:
            return (width + 7) // 8 * 8
        if ld % 8 == 0 and ld >= width:
            return ld
    return 0


def _align(h: torch.Tensor, ldh: int, w: torch.Tensor, ldw: int, index: int):
    """h and w, copied where their stride is given as 0, and their strides."""
    tokens, width = h.shape
    vocab = w.shape[0]
    padded = (width + 7) // 8 * 8
    rows = 0 if ldh else tokens
    copy = torch.empty(rows + (0 if ldw else vocab), padded, dtype=h.dtype, device=h.device)
    at = copy.data_ptr()
    status = B.lib().ssgd_xent_align_block(_pack_align(
        h.data_ptr(), *h.stride(), rows, at, w.data_ptr(), *w.stride(), 0 if ldw else vocab, at + 2 * rows * padded, width, padded, _stream_of(index)))
    if status:
        B._check(status, "ssgd_xent_align")
    return h if ldh else copy[:tokens], ldh or padded, w if ldw else copy[rows:], ldw or padded


class Kept(NamedTuple):
    """What the backward pass needs of the forward pass."""
    h: torch.Tensor             # [tokens][..], as the kernels read it
    w: torch.Tensor
    targets: torch.Tensor
    state: torch.Tensor         # log sum exp, loss and kind of each token
    ld: Tuple[int, int]         # row strides of h and w
    sides: Tuple[int, int, int]


def cross_entropy_forward(h: torch.Tensor, w: torch.Tensor, targets: torch.Tensor, ignore_index: int = -100) -> Tuple[torch.Tensor, Kept]:
    """losses[t] = log sum_v exp (h_t . w_v) - h_t . w_target (float32; 0 where the target is ignore_index, NaN where it is another number
    outside the vocabulary), with what `cross_entropy_backward` needs.  h [tokens][width] and w [vocabulary][width] of one type,
    bfloat16 or float16, rows at any stride (rows that do not start at multiples of 16 bytes are copied); targets int64 [tokens].  Autograd does not see
    this pass: `cross_entropy` is the one that it differentiates."""
    code = _DTYPES[h.dtype]
    if w.dtype != h.dtype:
        raise TypeError("h and w must be of one dtype, got %s and %s" % (h.dtype, w.dtype))
    if targets.dtype != torch.int64:
        raise TypeError("targets must be of dtype int64")
    if h.dim() != 2 or w.dim() != 2 or targets.dim() != 1 or h.shape[1] != w.shape[1] or h.shape[0] != targets.shape[0]:
        raise ValueError("h must be tokens x width, w vocabulary x width, targets one a token: got %s, %s and %s" % (tuple(h.shape), tuple(w.shape), tuple(targets.shape)))
    device = h.device
    index = device.index
    if index is None or not h.is_cuda:
        raise ValueError("h must live in device memory")
    if w.device != device or targets.device != device:
        raise ValueError("h, w and targets must live in the memory of one device")
    (tokens, width), vocab = h.shape, w.shape[0]
    if vocab < 1 or width < 1:
        raise ValueError("an empty vocabulary or width has no loss")
    if index != _current_device():
        with B._on(index):
            return cross_entropy_forward(h, w, targets, ignore_index)
    ldh, ldw = _stride_as_it_is(h, width), _stride_as_it_is(w, width)
    if tokens and not (ldh and ldw):
        h, ldh, w, ldw = _align(h, ldh, w, ldw, index)
    if not targets.is_contiguous():
        targets = targets.contiguous()
    losses = torch.empty(tokens, dtype=torch.float32, device=device)
    need = _sizes(index, tokens, vocab, width)[0] if tokens else 0
    kept = (9 * tokens + 15) // 16 * 16
    if need <= _SMALL:                      # one allocation for what is kept and what is not: 2 us less
        state = torch.empty(kept + need, dtype=torch.uint8, device=device)
        at = state.data_ptr()
        work_at = at + kept
    else:
        state = torch.empty(kept, dtype=torch.uint8, device=device)
        work = torch.empty(need, dtype=torch.uint8, device=device)
        at, work_at = state.data_ptr(), work.data_ptr()
    if tokens:
        status = B.lib().ssgd_xent_forward_block(_pack_forward(
            h.data_ptr(), ldh, w.data_ptr(), ldw, code, tokens, vocab, width, targets.data_ptr(), ignore_index, losses.data_ptr(), at,
            at + 8 * tokens, work_at, status_of(device)[1], _stream_of(index)))
        if status:
            B._check(status, "ssgd_xent_forward")
    return losses, Kept(h, w, targets, state, (ldh, ldw), (tokens, vocab, width))


def cross_entropy_backward(kept: Kept, g: torch.Tensor, dw: Optional[torch.Tensor] = None, dw_dtype: Optional[torch.dtype] = None,
                           want_h: bool = True, want_w: bool = True) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor]]:
    """dh (of h's type) and dw for the gradient g (float32, one a token, at any stride) of the losses; dw of dw_dtype (None: w's type) or
    into `dw` where given (float32, bfloat16 or float16, rows at any stride).  One that is not wanted is None."""
    tokens, vocab, width = kept.sides
    device = kept.h.device
    index = device.index
    if g.dtype != torch.float32:
        raise TypeError("g must be of dtype float32")
    if g.shape != (tokens,) or g.device != device:
        raise ValueError("g must hold one gradient for each of the %d tokens, on the operands' device" % tokens)
    if dw is None:
        code = B.DTYPE_CODE[dw_dtype or kept.w.dtype]
    else:
        code = B.DTYPE_CODE[dw.dtype]
        if dw.shape != (vocab, width) or dw.device != device or (width > 1 and dw.stride(1) != 1) or (vocab > 1 and dw.stride(0) < width):
            raise ValueError("dw must be %d x %d with unit column stride, on the operands' device" % (vocab, width))
    if index != _current_device():
        with B._on(index):
            return cross_entropy_backward(kept, g, dw, dw_dtype, want_h, want_w)
    dh = torch.empty(tokens, width, dtype=kept.h.dtype, device=device) if want_h else None
    if not want_w:
        dw = None
    elif dw is None:
        dw = torch.empty(vocab, width, dtype=dw_dtype or kept.w.dtype, device=device)
    if tokens == 0:
        return dh, dw.zero_() if want_w else None
    if want_h or want_w:
        work = torch.empty(_sizes(index, tokens, vocab, width)[1], dtype=torch.uint8, device=device)
        at = kept.state.data_ptr()
        status = B.lib().ssgd_xent_backward_block(_pack_backward(
            kept.h.data_ptr(), kept.ld[0], kept.w.data_ptr(), kept.ld[1], _DTYPES[kept.h.dtype], tokens, vocab, width, kept.targets.data_ptr(), at,
            at + 8 * tokens, g.data_ptr(), g.stride(0), dh.data_ptr() if want_h else 0, width, dw.data_ptr() if want_w else 0, code,
            (dw.stride(0) if vocab > 1 else width) if want_w else width, work.data_ptr(), status_of(device)[1], _stream_of(index)))
        if status:
            B._check(status, "ssgd_xent_backward")
    return dh, dw


class _Once(torch.autograd.Function):
    """Passes a gradient on; an error where somebody differentiates it."""

    @staticmethod
    def forward(ctx, gradient, g):
        return gradient.view_as(gradient)

    @staticmethod
    def backward(ctx, _):
        raise RuntimeError("loss.cross_entropy can be differentiated once only: its gradients have none of their own")


class _CrossEntropy(torch.autograd.Function):
    @staticmethod
    def forward(ctx, h, w, targets, ignore_index, grad):
        losses, kept = cross_entropy_forward(h.reshape(math.prod(h.shape[:-1]), h.shape[-1]), w, targets.reshape(-1), ignore_index)
        if grad and any(ctx.needs_input_grad[:2]):
            ctx.save_for_backward(*kept[:4])
            ctx.rest, ctx.h_shape = kept[4:], h.shape
        return losses.view(targets.shape)

    @staticmethod
    def backward(ctx, g):
        with torch.no_grad():
            dh, dw = cross_entropy_backward(Kept(*ctx.saved_tensors, *ctx.rest), g.reshape(-1), want_h=ctx.needs_input_grad[0], want_w=ctx.needs_input_grad[1])
            dh = dh if dh is None else dh.view(ctx.h_shape)
        if torch.is_grad_enabled():            # create_graph=True
            dh, dw = [None if d is None else _Once.apply(d.requires_grad_(), g) for d in (dh, dw)]
        return dh, dw, None, None, None


def cross_entropy(h: torch.Tensor, w: torch.Tensor, targets: torch.Tensor, ignore_index: int = -100, reduction: str = "mean") -> torch.Tensor:
    """The losses of `cross_entropy_forward` for torch's autograd, h [..., width] and targets [...]: "none" as they are, "sum", or "mean"
    over the tokens that are not ignored (0 where all are).  First derivatives only.  To capture gradients into a CUDA graph while an eager
    graph of the same leaves lives, take leaves of the capture's own (`x.detach().requires_grad_()`): torch ties a leaf to the
    stream of its living graph."""
    if reduction not in ("none", "sum", "mean"):
        raise ValueError("reduction must be 'none', 'sum' or 'mean', got %r" % (reduction,))
    if h.dim() < 1 or h.shape[:-1] != targets.shape:
        raise ValueError("targets must have h's shape without its last side: got %s and %s" % (tuple(targets.shape), tuple(h.shape)))
    losses = _CrossEntropy.apply(h, w, targets, ignore_index, torch.is_grad_enabled())
    if reduction == "none":
        return losses
    total = losses.sum()
    return total if reduction == "sum" else total / (targets != ignore_index).sum().clamp(min=1)
