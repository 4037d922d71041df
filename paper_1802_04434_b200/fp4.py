"""Operands in microscaled 4-bit floating point over torch tensors: packing, unpacking, products, a linear layer.

A thin layer over ``binding.fp4_*`` that allocates the outputs; the formats ("mx": blocks of 32 with a power of two,
"nv": blocks of 16 with an E4M3 number and a tensor scale) and the arithmetic are those of ``include/signsgd.h``.  All
work is enqueued on the current stream of the operands' device, whichever device is current.
"""
from __future__ import annotations

import math
from typing import NamedTuple, Optional, Tuple

import torch

from . import binding as B
from .waits import _status, check, status_of  # noqa: F401  (check: part of this module)

_BLOCK = {"mx": 32, "nv": 16}
_U8 = torch.uint8


def _sizes(rows: int, cols: int, fmt: str) -> Tuple[int, int]:
    """Bytes of the codes and of the scales of a packed operand."""
    return rows * ((cols + 31) // 32 * 16), (rows + 127) // 128 * (((cols + _BLOCK[fmt] - 1) // _BLOCK[fmt] + 3) // 4) * 512


class Packed:
    """A matrix in 4 bits, blocks along its columns.

    codes          uint8 [rows][row bytes], contiguous
    scales         uint8, tiles of 128 rows x 4 blocks, contiguous
    tensor_scale   float32, its first element (None: 1); "nv" only

    Its three parts may lie in one buffer, as `quantise` makes them; they are cut out of it when they are asked for."""
    __slots__ = ("rows", "cols", "fmt", "device", "pointers", "_parts", "_buffer")      # _buffer: (buffer, byte offsets of the parts)

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, tensor_scale: Optional[torch.Tensor], rows: int, cols: int, fmt: str):
        if fmt not in _BLOCK:
            raise ValueError("fmt must be 'mx' or 'nv'")
        if fmt == "mx" and tensor_scale is not None:
            raise ValueError("the mx format has no tensor scale")
        if codes.dtype != _U8 or scales.dtype != _U8 or (tensor_scale is not None and tensor_scale.dtype != torch.float32):
            raise TypeError("codes and scales must be uint8 tensors, tensor_scale a float32 one")
        device = codes.device
        if not codes.is_cuda or scales.device != device or (tensor_scale is not None and tensor_scale.device != device):
            raise ValueError("codes, scales and tensor_scale must live in the memory of one device")
        B._need_first(tensor_scale, "tensor_scale")
        if not (codes.is_contiguous() and scales.is_contiguous()):
            raise ValueError("codes and scales must be contiguous")
        n, m = _sizes(rows, cols, fmt)
        if codes.numel() < n or scales.numel() < m:
            raise ValueError("codes hold %d bytes, scales %d; %d x %d %s needs %d and %d" % (codes.numel(), scales.numel(), rows, cols, fmt, n, m))
        self.pointers = (codes.data_ptr(), scales.data_ptr(), 0 if tensor_scale is None else tensor_scale.data_ptr())
        self.rows, self.cols, self.fmt, self.device = rows, cols, fmt, device
        self._parts, self._buffer = (codes, scales, tensor_scale), None

    def _cut(self):
        if self._parts is None:
            buffer, (c, s, t) = self._buffer
            n, m = _sizes(self.rows, self.cols, self.fmt)
            self._parts = (buffer[c:c + n].view(self.rows, -1) if n else buffer[:0].view(self.rows, (self.cols + 31) // 32 * 16), buffer[s:s + m],
                           None if t is None else buffer[t:t + 8].view(torch.float32))
        return self._parts

    codes = property(lambda self: self._cut()[0])
    scales = property(lambda self: self._cut()[1])
    tensor_scale = property(lambda self: self._cut()[2])

    def _replace(self, **parts) -> "Packed":
        """A copy with some of codes, scales, tensor_scale, rows, cols, fmt replaced."""
        names = ("codes", "scales", "tensor_scale", "rows", "cols", "fmt")
        return Packed(*[parts.get(n, getattr(self, n)) for n in names])


# These calls are a few microseconds of Python each, next to kernels of a few microseconds: what is below avoids calls,
# temporary objects and look-ups on the way to the library.
_new = object.__new__
_stream_of, _current_device = B._stream_of, B._current_device
_pack_quantise, _pack_dequantise, _pack_matmul = B.FP4_QUANTISE_ARGS.pack, B.FP4_DEQUANTISE_ARGS.pack, B.FP4_MATMUL_ARGS.pack
_DTYPES, _FORMATS = B.DTYPE_CODE, B.FP4_FORMAT


def _packed_in(buffer, base, codes, scales, ts, rows, cols, fmt, device):
    """A packed matrix whose parts lie at the given byte offsets of one buffer, whose address is `base`."""
    p = _new(Packed)
    p.rows = rows
    p.cols = cols
    p.fmt = fmt
    p.device = device
    p.pointers = (base + codes, base + scales, 0 if ts is None else base + ts)
    p._parts = None
    p._buffer = (buffer, (codes, scales, ts))
    return p


def _quantise(x, fmt, amax, by_rows, by_columns):
    block = _BLOCK.get(fmt)
    if block is None:
        raise ValueError("fmt must be 'mx' or 'nv'")
    dtype = _DTYPES.get(x.dtype)
    if dtype is None:
        raise TypeError("the matrix must be of dtype float32, bfloat16 or float16")
    strides = x.stride()
    if len(strides) != 2:
        raise ValueError("a matrix is wanted, got %d dimensions" % len(strides))
    device = x.device
    index = device.index
    if index is None or not x.is_cuda:
        raise ValueError("the matrix must live in device memory")
    if amax is not None:
        B._need_first(amax, "amax")
        B._need_device(index, amax=amax)
    if index != _current_device():
        with B._on(index):
            return _quantise(x, fmt, amax, by_rows, by_columns)
    rows, cols = x.shape
    ldx, step = strides
    # rows at any stride; a single column, or a single row, has no stride of its own to look at
    if (step != 1 and cols > 1) or (ldx < cols and rows > 1):
        x = x.contiguous()
        ldx = cols
    at = 0                                    # the parts one after another: all are multiples of 16 bytes
    if by_rows:
        s = rows * ((cols + 31) // 32 * 16)
        at = s + (rows + 127) // 128 * ((cols + 4 * block - 1) // (4 * block)) * 512
    if by_columns:
        ct = at
        st = ct + cols * ((rows + 31) // 32 * 16)
        at = st + (cols + 127) // 128 * ((rows + 4 * block - 1) // (4 * block)) * 512
    if block == 32:
        ts, size = None, at
    else:
        ts, size = at, at + (4 * B.FP4_SCALE_FLOATS if amax is None and rows * cols > B.FP4_SMALL else 8)
    buffer = torch.empty(size, dtype=_U8, device=device)
    base = buffer.data_ptr()
    if rows and cols:
        status = B.lib().ssgd_fp4_quantise_block(_pack_quantise(
            x.data_ptr(), dtype, rows, cols, ldx if ldx > cols else cols, 0 if ts is None else 1,
            0 if amax is None else B._ptr(amax, torch.float32, "amax"), 0 if ts is None else base + ts, base if by_rows else 0,
            base + s if by_rows else 0, base + ct if by_columns else 0, base + st if by_columns else 0, _stream_of(index)))
        if status:
            B._check(status, "ssgd_fp4_quantise")
    elif ts is not None:
        buffer[ts:ts + 8].view(torch.float32).fill_(1.0)
    if not by_columns:
        return _packed_in(buffer, base, 0, s, ts, rows, cols, fmt, device)
    transposed = _packed_in(buffer, base, ct, st, ts, cols, rows, fmt, device)
    return (_packed_in(buffer, base, 0, s, ts, rows, cols, fmt, device), transposed) if by_rows else transposed


def quantise(x: torch.Tensor, fmt: str = "mx", amax: Optional[torch.Tensor] = None) -> Packed:
    """x (float32, bfloat16 or float16, rows at any stride) packed with blocks along its columns.  `amax`: a device
    float32 with max |x|, "nv" only, where the caller has it already (`binding.tensors_norm(kind="max")`)."""
    return _quantise(x, fmt, amax, True, False)


def quantise_columns(x: torch.Tensor, fmt: str = "mx", amax: Optional[torch.Tensor] = None) -> Packed:
    """The transpose of x packed: blocks along x's rows."""
    return _quantise(x, fmt, amax, False, True)


def quantise_both(x: torch.Tensor, fmt: str = "mx", amax: Optional[torch.Tensor] = None) -> Tuple[Packed, Packed]:
    """x and its transpose packed, as a layer's forward and backward products want them."""
    return _quantise(x, fmt, amax, True, True)


def dequantise(p: Packed, dtype: torch.dtype = torch.float32) -> torch.Tensor:
    """The values of a packed matrix."""
    code = _DTYPES[dtype]
    rows, cols, device = p.rows, p.cols, p.device
    index = device.index
    if index != _current_device():
        with B._on(index):
            return dequantise(p, dtype)
    out = torch.empty(rows, cols, dtype=dtype, device=device)
    if rows and cols:
        status = B.lib().ssgd_fp4_dequantise_block(_pack_dequantise(
            *p.pointers, _FORMATS[p.fmt], rows, cols, out.data_ptr(), code, cols, _stream_of(index)))
        if status:
            B._check(status, "ssgd_fp4_dequantise")
    return out


def matmul(a: Packed, b: Packed, dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """a b^T of two packed matrices of one format, fp32 accumulation; into `out` (rows at any stride) where given."""
    fmt, k, device = a.fmt, a.cols, a.device
    if fmt != b.fmt or k != b.cols or device != b.device:
        raise ValueError("a product needs operands of one format, one length and one device: got %s x %d and %s x %d" % (fmt, k, b.fmt, b.cols))
    index = device.index
    if index != _current_device():
        with B._on(index):
            return matmul(a, b, dtype, out)
    rows, cols = a.rows, b.rows
    ldo = cols or 1
    code = _DTYPES[dtype if out is None else out.dtype]
    if out is None:
        out = torch.empty(rows, cols, dtype=dtype, device=device)
    else:
        if out.shape != (rows, cols) or out.device != device or (cols > 1 and out.stride(1) != 1) or (rows > 1 and out.stride(0) < cols):
            raise ValueError("out must be %d x %d with unit column stride, on the operands' device" % (rows, cols))
        ldo = out.stride(0) if rows > 1 else ldo
    if k == 0:
        return out.zero_()
    if rows and cols:
        status = _status.get(device) or status_of(device)
        failed = B.lib().ssgd_fp4_matmul_block(_pack_matmul(
            *a.pointers, *b.pointers, rows, cols, k, _FORMATS[fmt], out.data_ptr(), code, ldo, status[1], _stream_of(index)))
        if failed:
            B._check(failed, "ssgd_fp4_matmul")
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


def _rows_of(x: torch.Tensor) -> torch.Tensor:
    """x [..., n] as a matrix; its sides may be 0, where reshape(-1, n) would not know how many rows there are."""
    return x.reshape(math.prod(x.shape[:-1]), x.shape[-1])


class _Once(torch.autograd.Function):
    """Passes a gradient on; an error where somebody differentiates it.  (torch's once_differentiable does so only where the gradient
    that comes in can be differentiated, but dx depends on w, and dw on x, whatever comes in.)"""

    @staticmethod
    def forward(ctx, gradient, dy):
        return gradient.view_as(gradient)

    @staticmethod
    def backward(ctx, _):
        raise RuntimeError("fp4.linear can be differentiated once only: its products' gradients have none of their own")


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, fmt, grad):
        rows = _rows_of(x)
        # needs_input_grad says what the inputs want, in whatever mode the call is made
        need_x, need_w = [grad and need for need in ctx.needs_input_grad[:2]]
        # only what the backward products will want is packed by columns
        xr, xc = quantise_both(rows, fmt) if need_w else (quantise(rows, fmt), None)
        wr, wc = quantise_both(w, fmt) if need_x else (quantise(w, fmt), None)
        ctx.save_for_backward(*[None if p is None else p._buffer[0] for p in (xc, wc)])
        ctx.places = [None if p is None else (*p._buffer[1], p.rows, p.cols) for p in (xc, wc)]      # in their buffers, and sides
        ctx.fmt, ctx.x_dtype, ctx.w_dtype, ctx.x_shape = fmt, x.dtype, w.dtype, x.shape
        return matmul(xr, wr, x.dtype).view(*x.shape[:-1], w.shape[0])

    @staticmethod
    def backward(ctx, dy):
        with torch.no_grad():
            dx, dw = _Linear._gradients(ctx, dy)
        if torch.is_grad_enabled():            # create_graph=True
            dx, dw = [None if g is None else _Once.apply(g.requires_grad_(), dy) for g in (dx, dw)]
        return dx, dw, None, None

    @staticmethod
    def _gradients(ctx, dy):
        fmt = ctx.fmt
        xc, wc = [None if b is None else _packed_in(b, b.data_ptr(), *at, fmt, b.device) for b, at in zip(ctx.saved_tensors, ctx.places)]
        rows = _rows_of(dy)
        if xc is None:
            dr, dc = quantise(rows, fmt), None
        elif wc is None:
            dr, dc = None, quantise_columns(rows, fmt)
        else:
            dr, dc = quantise_both(rows, fmt)
        dx = matmul(dr, wc, ctx.x_dtype).view(ctx.x_shape) if dr is not None else None
        return dx, matmul(dc, xc, ctx.w_dtype) if dc is not None else None


def linear(x: torch.Tensor, w: torch.Tensor, fmt: str = "mx") -> torch.Tensor:
    """x w^T with all three products in 4 bits, for torch's autograd; x [..., in], w [out][in].  First derivatives only."""
    if w.dim() != 2 or x.dim() < 1 or x.shape[-1] != w.shape[1]:
        raise ValueError("x's last side must be w's second: got %s and %s" % (tuple(x.shape), tuple(w.shape)))
    return _Linear.apply(x, w, fmt, torch.is_grad_enabled())
