"""Orthogonalised updates over torch tensors: a matrix with its singular values brought near one, and the momentum step with it.

A thin layer over ``ssgd_orthogonalise`` and ``ssgd_orthogonal_step`` (``include/signsgd.h``) that allocates outputs and workspaces.
Tensors are matrices, or batches of matrices of one shape [..., rows, cols], such as one layer's weights of every block; parameters
and momenta may be views of flat vectors.  All work is enqueued on the current stream of the operands' device, whichever
device is current.
"""
from __future__ import annotations

import functools
import math
from typing import Optional, Tuple

import torch

from . import binding as B
from .waits import check, status_of  # noqa: F401  (check: part of this module)

# Five steps with these bring singular values from 0.003 of the norm on to 0.68 .. 1.14: steep at 0 rather than exact at 1.
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
# Smaller side from which a bfloat16 result is computed with operands of 11 bits: the error stays below the rounding of
# the result there, and below it the time is that of the launches.
ONE_PRODUCT_SIDE = 256

_stream_of, _current_device = B._stream_of, B._current_device
_pack_orthogonalise, _pack_step = B.ORTHOGONALISE_ARGS.pack, B.ORTHOGONAL_STEP_ARGS.pack
_DTYPES = B.DTYPE_CODE


@functools.lru_cache(maxsize=256)
def _ws_bytes(n: int, rows: int, cols: int) -> int:
    return B.orthogonal_ws_bytes(n, rows, cols)


def _batch(t: torch.Tensor, name: str, written: bool) -> Tuple[torch.Tensor, int, int, int]:
    """t as a batch of matrices with side by side columns: the tensor, their number, row and matrix stride."""
    shape = t.shape
    if len(shape) < 2:
        raise ValueError("%s must be a matrix or a batch of them, got %d dimensions" % (name, len(shape)))
    if len(shape) > 3:
        lead = math.prod(shape[:-2])
        try:
            t = t.view(lead, *shape[-2:])
        except RuntimeError:
            if written:
                raise ValueError("the leading sides of %s must be one in memory" % name) from None
            t = t.reshape(lead, *shape[-2:])
        shape = t.shape
    rows, cols = shape[-2:]
    stride = t.stride()
    n = shape[0] if len(shape) == 3 else 1
    # matrices behind one another, or their rows in turn
    shared = written and n > 1 and rows and cols and stride[0] < (rows - 1) * stride[-2] + cols and (stride[0] < cols or stride[-2] < (n - 1) * stride[0] + cols)
    if (cols > 1 and stride[-1] != 1) or (rows > 1 and stride[-2] < cols) or shared:
        if written:
            raise ValueError("the matrices of %s must have unit column stride and share no elements" % name)
        t = t.contiguous()
        stride = t.stride()
    return t, n, stride[-2] if rows > 1 else cols, stride[0] if n > 1 else rows * cols


def _options(steps, coefficients, products) -> Tuple[float, float, float]:
    """The coefficients as floats; the options have been looked at."""
    if not 1 <= steps <= 100:
        raise ValueError("steps must be 1 to 100, got %r" % (steps,))
    if products not in (1, 3):
        raise ValueError("products must be 1 or 3, got %r" % (products,))
    a, b, c = coefficients
    return float(a), float(b), float(c)


class _NoDerivative(torch.autograd.Function):
    """Passes a result on; an error where somebody differentiates it."""

    @staticmethod
    def forward(ctx, result, u):
        ctx.mark_dirty(result)                  # the tensor itself: a view of it could not be changed in place
        return result

    @staticmethod
    def backward(ctx, _):
        raise RuntimeError("orthogonal.orthogonalise has no derivative; detach() u where none is meant")


def orthogonalise(u: torch.Tensor, steps: int = 5, coefficients=COEFFICIENTS, dtype: Optional[torch.dtype] = None,
                  out: Optional[torch.Tensor] = None, products: Optional[int] = None) -> torch.Tensor:
    """X = u / |u|, then `steps` times X <- a X + (b A + c A^2) X with A = X X^T, for each matrix of u (float32, bfloat16 or float16);
    of `dtype` (None: u's), or into `out`, which may be u.  products: 3, as exact as products in float32, or 1, off by about 1e-3 of
    the result's norm; None: 1 for a bfloat16 result whose smaller side is 256 or more, else 3.  There is no derivative: where autograd
    would want one of a result (`out` is written as it is), its backward pass is an error."""
    code = _DTYPES[u.dtype]
    device = u.device
    index = device.index
    if index is None or not u.is_cuda:
        raise ValueError("u must live in device memory")
    if out is not None and (out.shape != u.shape or out.device != device):
        raise ValueError("out must be of u's shape, on its device")
    out_code = _DTYPES[(dtype or u.dtype) if out is None else out.dtype]
    if index != _current_device():
        with B._on(index):
            return orthogonalise(u, steps, coefficients, dtype, out, products)
    us, n, ldu, su = _batch(u, "u", False)
    wanted = out is None and torch.is_grad_enabled() and getattr(u, "requires_grad", False)
    if out is None:
        out = torch.empty(u.shape, dtype=dtype or u.dtype, device=device)
    os, _, ldo, so = _batch(out, "out", True)
    rows, cols = us.shape[-2:]
    if products is None:
        products = 1 if out_code == 1 and min(rows, cols) >= ONE_PRODUCT_SIDE else 3
    abc = _options(steps, coefficients, products)
    if n and rows and cols:
        work = torch.empty(_ws_bytes(n, rows, cols), dtype=torch.uint8, device=device)
        status = B.lib().ssgd_orthogonalise_block(_pack_orthogonalise(
            us.data_ptr(), code, n, rows, cols, ldu, su, *abc, steps, products, os.data_ptr(), out_code, ldo, so,
            work.data_ptr(), status_of(device)[1], _stream_of(index)))
        if status:
            B._check(status, "ssgd_orthogonalise")
    return _NoDerivative.apply(out, u) if wanted else out


def momentum_step(x: torch.Tensor, g: torch.Tensor, m: torch.Tensor, beta: float, delta: float, steps: int = 5,
                  coefficients=COEFFICIENTS, nesterov: bool = False, products: int = 3) -> None:
    """In place, unseen by autograd: m <- beta m + (1 - beta) g, then x <- x - delta orthogonalise(m), or with nesterov of
    beta m + (1 - beta) g.  x and m float32, g float32, bfloat16 or float16; matrices, or batches of one shape, no two of them in
    the same memory.  A factor for the shape (such as max(1, rows / cols) ** 0.5) goes into delta."""
    if x.dtype != torch.float32 or m.dtype != torch.float32:
        raise TypeError("x and m must be of dtype float32")
    code = _DTYPES[g.dtype]
    device = x.device
    index = device.index
    if index is None or not x.is_cuda:
        raise ValueError("x must live in device memory")
    if g.shape != x.shape or m.shape != x.shape or g.device != device or m.device != device:
        raise ValueError("x, g and m must be of one shape, on one device")
    if index != _current_device():
        with B._on(index):
            return momentum_step(x, g, m, beta, delta, steps, coefficients, nesterov, products)
    xs, n, ldx, sx = _batch(x, "x", True)
    ms, _, ldm, sm = _batch(m, "m", True)
    gs, _, ldg, sg = _batch(g, "g", False)
    rows, cols = xs.shape[-2:]
    abc = _options(steps, coefficients, products)
    if n and rows and cols:
        if len({xs.data_ptr(), ms.data_ptr(), gs.data_ptr()}) < 3:
            raise ValueError("x, g and m must not share memory")
        work = torch.empty(_ws_bytes(n, rows, cols), dtype=torch.uint8, device=device)
        status = B.lib().ssgd_orthogonal_step_block(_pack_step(
            xs.data_ptr(), ldx, sx, gs.data_ptr(), code, ldg, sg, ms.data_ptr(), ldm, sm, n, rows, cols, beta, delta, 1 if nesterov else 0,
            *abc, steps, products, work.data_ptr(), status_of(device)[1], _stream_of(index)))
        if status:
            B._check(status, "ssgd_orthogonal_step")
