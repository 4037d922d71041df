"""Operands in microscaled 4-bit floating point over torch tensors: packing, unpacking, products, a linear layer.

A thin layer over ``binding.fp4_*`` that allocates the outputs; the formats ("mx": blocks of 32 with a power of two,
"nv": blocks of 16 with an E4M3 number and a tensor scale) and the arithmetic are those of ``include/signsgd.h``.  All
work is enqueued on the current stream of the operands' device.
"""
from __future__ import annotations

from typing import NamedTuple, Optional, Tuple

import torch

from . import binding as B


class Packed(NamedTuple):
    """A matrix in 4 bits, blocks along its columns."""
    codes: torch.Tensor                     # uint8 [rows][row bytes]
    scales: torch.Tensor                    # uint8, tiles of 128 rows x 4 blocks
    tensor_scale: Optional[torch.Tensor]    # float32, its first element (None: 1)
    rows: int
    cols: int
    fmt: str


_status = {}


def _status_of(device: torch.device) -> torch.Tensor:
    s = _status.get(device)
    if s is None:
        s = _status[device] = torch.zeros(1, dtype=torch.int32, device=device)
    return s


def check(device="cuda") -> None:
    """Waits for the device and raises if a product since the last check had to give up a bounded wait."""
    device = torch.device("cuda", torch.cuda.current_device()) if torch.device(device).index is None else torch.device(device)
    s = _status_of(device)
    if int(s.item()):
        s.zero_()
        raise RuntimeError("a 4-bit product did not receive its operands in time; its output is not valid")


def _matrix(x: torch.Tensor) -> torch.Tensor:
    if x.dim() != 2:
        raise ValueError("a matrix is wanted, got %d dimensions" % x.dim())
    # rows at any stride; a single column, or a single row, has no stride of its own to look at
    return x if (x.stride(1) == 1 or x.shape[1] <= 1) and x.stride(0) >= x.shape[1] else x.contiguous()


def _empty(rows: int, cols: int, fmt: str, device) -> Tuple[torch.Tensor, torch.Tensor]:
    return (torch.empty(rows, (cols + 31) // 32 * 16, dtype=torch.uint8, device=device),
            torch.empty(B.fp4_scale_bytes(fmt, rows, cols), dtype=torch.uint8, device=device))


def _quantise(x, fmt, amax, by_rows, by_columns):
    if fmt not in B.FP4_FORMAT:
        raise ValueError("fmt must be 'mx' or 'nv'")
    x = _matrix(x)
    rows, cols = x.shape
    codes = scales = codes_t = scales_t = ts = None
    if by_rows:
        codes, scales = _empty(rows, cols, fmt, x.device)
    if by_columns:
        codes_t, scales_t = _empty(cols, rows, fmt, x.device)
    if fmt == "nv":
        ts = torch.empty(2, device=x.device) if rows and cols else torch.ones(2, device=x.device)
    if rows and cols:
        B.fp4_quantise(x, rows, cols, max(x.stride(0), cols), fmt, amax, ts, codes, scales, codes_t, scales_t)
    return (Packed(codes, scales, ts, rows, cols, fmt) if by_rows else None,
            Packed(codes_t, scales_t, ts, cols, rows, fmt) if by_columns else None)


def quantise(x: torch.Tensor, fmt: str = "mx", amax: Optional[torch.Tensor] = None) -> Packed:
    """x (float32, bfloat16 or float16, rows at any stride) packed with blocks along its columns.  `amax`: a device
    float32 with max |x|, "nv" only, where the caller has it already (`binding.tensors_norm(kind="max")`)."""
    return _quantise(x, fmt, amax, True, False)[0]


def quantise_columns(x: torch.Tensor, fmt: str = "mx", amax: Optional[torch.Tensor] = None) -> Packed:
    """The transpose of x packed: blocks along x's rows."""
    return _quantise(x, fmt, amax, False, True)[1]


def quantise_both(x: torch.Tensor, fmt: str = "mx", amax: Optional[torch.Tensor] = None) -> Tuple[Packed, Packed]:
    """x and its transpose packed, as a layer's forward and backward products want them."""
    return _quantise(x, fmt, amax, True, True)


def dequantise(p: Packed, dtype: torch.dtype = torch.float32) -> torch.Tensor:
    """The values of a packed matrix."""
    out = torch.empty(p.rows, p.cols, dtype=dtype, device=p.codes.device)
    if p.rows and p.cols:
        B.fp4_dequantise(p.codes, p.scales, p.tensor_scale, p.fmt, p.rows, p.cols, out, max(1, p.cols))
    return out


def matmul(a: Packed, b: Packed, dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """a b^T of two packed matrices of one format, fp32 accumulation; into `out` (rows at any stride) where given."""
    if a.fmt != b.fmt or a.cols != b.cols:
        raise ValueError("a product needs operands of one format and one length: got %s x %d and %s x %d" % (a.fmt, a.cols, b.fmt, b.cols))
    if out is None:
        out = torch.empty(a.rows, b.rows, dtype=dtype, device=a.codes.device)
    elif out.shape != (a.rows, b.rows) or (b.rows > 1 and out.stride(1) != 1) or (a.rows > 1 and out.stride(0) < b.rows):
        raise ValueError("out must be %d x %d with unit column stride" % (a.rows, b.rows))
    if a.cols == 0:
        return out.zero_()
    if a.rows and b.rows:
        B.fp4_matmul(a.codes, a.scales, a.tensor_scale, b.codes, b.scales, b.tensor_scale, a.rows, b.rows, a.cols, a.fmt, out,
                     out.stride(0) if a.rows > 1 else max(1, b.rows), _status_of(a.codes.device))
    return out


class Kept(NamedTuple):
    """What a linear layer's backward products need of its forward pass."""
    x_columns: Packed
    w_columns: Packed
    dtype: torch.dtype


def linear_forward(x: torch.Tensor, w: torch.Tensor, fmt: str = "mx") -> Tuple[torch.Tensor, Kept]:
    """y = x w^T in x's type (x [tokens][in], w [out][in]), with what `linear_backward` needs."""
    xr, xc = quantise_both(x, fmt)
    wr, wc = quantise_both(w, fmt)
    return matmul(xr, wr, x.dtype), Kept(xc, wc, x.dtype)


def linear_backward(kept: Kept, dy: torch.Tensor, dw: Optional[torch.Tensor] = None,
                    dw_dtype: torch.dtype = torch.float32) -> Tuple[torch.Tensor, torch.Tensor]:
    """dx = dy w in the forward's type and dw = dy^T x, into `dw` where given: the gradient passes straight through the
    rounding, each product taking its operands quantised along its own k."""
    dr, dc = quantise_both(dy, kept.x_columns.fmt)
    return matmul(dr, kept.w_columns, kept.dtype), matmul(dc, kept.x_columns, dw_dtype, dw)


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, fmt):
        y, ctx.kept = linear_forward(x.detach(), w.detach(), fmt)
        ctx.w_dtype = w.dtype
        return y

    @staticmethod
    def backward(ctx, dy):
        dx, dw = linear_backward(ctx.kept, dy, dw_dtype=ctx.w_dtype)
        return dx, dw, None


def linear(x: torch.Tensor, w: torch.Tensor, fmt: str = "mx") -> torch.Tensor:
    """x w^T with all three products in 4 bits, for torch's autograd."""
    return _Linear.apply(x, w, fmt)
