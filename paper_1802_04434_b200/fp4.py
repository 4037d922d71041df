"""Operands in microscaled 4-bit floating point over torch tensors: packing, unpacking, products, a linear layer.

A thin layer over ``binding.fp4_*`` that allocates the outputs; the formats ("mx": blocks of 32 with a power of two,
"nv": blocks of 16 with an E4M3 number and a tensor scale) and the arithmetic are those of ``include/signsgd.h``.  All
work is enqueued on the current stream of the operands' device.
"""
from __future__ import annotations

from typing import NamedTuple, Optional, Tuple

import torch

from . import binding as B

_BLOCK = {"mx": 32, "nv": 16}
_U8 = torch.uint8


def _sizes(rows: int, cols: int, fmt: str) -> Tuple[int, int]:
    """Bytes of the codes and of the scales of a packed operand."""
    return rows * ((cols + 31) // 32 * 16), (rows + 127) // 128 * (((cols + _BLOCK[fmt] - 1) // _BLOCK[fmt] + 3) // 4) * 512


class Packed:
    """A matrix in 4 bits, blocks along its columns.

    codes          uint8 [rows][row bytes], contiguous
    scales         uint8, tiles of 128 rows x 4 blocks, contiguous
    tensor_scale   float32, its first element (None: 1)

    Its three parts may lie in one buffer, as `quantise` makes them; they are cut out of it when they are asked for."""
    __slots__ = ("rows", "cols", "fmt", "device", "pointers", "_parts", "_buffer")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, tensor_scale: Optional[torch.Tensor], rows: int, cols: int, fmt: str):
        if fmt not in _BLOCK:
            raise ValueError("fmt must be 'mx' or 'nv'")
        if codes.dtype != _U8 or scales.dtype != _U8 or (tensor_scale is not None and tensor_scale.dtype != torch.float32):
            raise TypeError("codes and scales must be uint8 tensors, tensor_scale a float32 one")
        device = codes.device
        if not codes.is_cuda or scales.device != device or (tensor_scale is not None and tensor_scale.device != device):
            raise ValueError("codes, scales and tensor_scale must live in the memory of one device")
        if not (codes.is_contiguous() and scales.is_contiguous()):
            raise ValueError("codes and scales must be contiguous")
        n, m = _sizes(rows, cols, fmt)
        if codes.numel() < n or scales.numel() < m:
            raise ValueError("codes hold %d bytes, scales %d; %d x %d %s needs %d and %d" % (codes.numel(), scales.numel(), rows, cols, fmt, n, m))
        self.pointers = (codes.data_ptr(), scales.data_ptr(), 0 if tensor_scale is None else tensor_scale.data_ptr())
        self.rows, self.cols, self.fmt, self.device = rows, cols, fmt, device
        self._parts, self._buffer = (codes, scales, tensor_scale), None

    @classmethod
    def _in(cls, buffer: torch.Tensor, base: int, at: Tuple[int, int, Optional[int]], rows: int, cols: int, fmt: str,
            device: torch.device) -> "Packed":
        """Parts at the given byte offsets of one buffer whose address is `base`."""
        p = cls.__new__(cls)
        p.rows, p.cols, p.fmt, p.device = rows, cols, fmt, device
        p.pointers = (base + at[0], base + at[1], 0 if at[2] is None else base + at[2])
        p._parts, p._buffer = None, (buffer, at)
        return p

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


_status = {}


def _status_of(device: torch.device) -> Tuple[torch.Tensor, int]:
    """The word of a device in which a product reports a wait that ran out."""
    s = _status.get(device)
    if s is None:
        if torch.cuda.is_current_stream_capturing():
            raise RuntimeError("the first 4-bit product on a device must come before any stream capture")
        t = torch.zeros(1, dtype=torch.int32, device=device)
        torch.cuda.synchronize(device)      # zero before a product on any stream may use it
        s = _status[device] = (t, t.data_ptr())
    return s


def check(device="cuda") -> None:
    """Waits for the device and raises if a product since the last check had to give up a bounded wait."""
    device = torch.device("cuda", torch.cuda.current_device()) if torch.device(device).index is None else torch.device(device)
    s = _status_of(device)[0]
    torch.cuda.synchronize(device)
    if int(s.item()):
        s.zero_()
        raise RuntimeError("a 4-bit product did not receive its operands in time; its output is not valid")


def _quantise(x, fmt, amax, by_rows, by_columns):
    block = _BLOCK.get(fmt)
    if block is None:
        raise ValueError("fmt must be 'mx' or 'nv'")
    dtype = B.DTYPE_CODE.get(x.dtype)
    if dtype is None:
        raise TypeError("the matrix must be of dtype float32, bfloat16 or float16")
    shape = x.shape
    if len(shape) != 2:
        raise ValueError("a matrix is wanted, got %d dimensions" % len(shape))
    rows, cols = shape
    index = x.get_device()
    if index < 0:
        raise ValueError("the matrix must live in device memory")
    ldx, step = x.stride()
    # rows at any stride; a single column, or a single row, has no stride of its own to look at
    if (step != 1 and cols > 1) or (ldx < cols and rows > 1):
        x = x.contiguous()
        ldx = cols
    n = m = nt = mt = 0
    if by_rows:
        n, m = _sizes(rows, cols, fmt)
    if by_columns:
        nt, mt = _sizes(cols, rows, fmt)
    nv = block == 16
    ts = n + m + nt + mt                      # all parts are multiples of 16 bytes
    device = x.device
    tail = 0 if not nv else 4 * B.FP4_SCALE_FLOATS if amax is None and rows * cols > B.FP4_SMALL else 8
    buffer = torch.empty(ts + tail, dtype=_U8, device=device)
    base = buffer.data_ptr()
    if rows and cols:
        status = B.lib().ssgd_fp4_quantise_block(B.FP4_QUANTISE_ARGS.pack(
            x.data_ptr(), dtype, rows, cols, ldx if ldx > cols else cols, 1 if nv else 0,
            0 if amax is None else B._ptr(amax, torch.float32, "amax"), base + ts if nv else 0, base if by_rows else 0, base + n,
            base + n + m if by_columns else 0, base + n + m + nt, B._stream_of(index)))
        if status:
            B._check(status, "ssgd_fp4_quantise")
    elif nv:
        buffer[ts:ts + 8].view(torch.float32).fill_(1.0)
    at = ts if nv else None
    return (Packed._in(buffer, base, (0, n, at), rows, cols, fmt, device) if by_rows else None,
            Packed._in(buffer, base, (n + m, n + m + nt, at), cols, rows, fmt, device) if by_columns else None)


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
    out = torch.empty(p.rows, p.cols, dtype=dtype, device=p.device)
    if p.rows and p.cols:
        codes, scales, ts = p.pointers
        status = B.lib().ssgd_fp4_dequantise_block(B.FP4_DEQUANTISE_ARGS.pack(
            codes, scales, ts, B.FP4_FORMAT[p.fmt], p.rows, p.cols, out.data_ptr(), B.DTYPE_CODE[dtype], p.cols, B._stream_of(p.device.index)))
        if status:
            B._check(status, "ssgd_fp4_dequantise")
    return out


def matmul(a: Packed, b: Packed, dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """a b^T of two packed matrices of one format, fp32 accumulation; into `out` (rows at any stride) where given."""
    if a.fmt != b.fmt or a.cols != b.cols or a.device != b.device:
        raise ValueError("a product needs operands of one format, one length and one device: got %s x %d and %s x %d" % (a.fmt, a.cols, b.fmt, b.cols))
    rows, cols = a.rows, b.rows
    ldo = max(1, cols)
    if out is None:
        out = torch.empty(rows, cols, dtype=dtype, device=a.device)
    else:
        if out.shape != (rows, cols) or out.device != a.device or (cols > 1 and out.stride(1) != 1) or (rows > 1 and out.stride(0) < cols):
            raise ValueError("out must be %d x %d with unit column stride, on the operands' device" % (rows, cols))
        ldo = out.stride(0) if rows > 1 else ldo
    if a.cols == 0:
        return out.zero_()
    if rows and cols:
        status = B.lib().ssgd_fp4_matmul_block(B.FP4_MATMUL_ARGS.pack(
            *a.pointers, *b.pointers, rows, cols, a.cols, B.FP4_FORMAT[a.fmt], out.data_ptr(), B.DTYPE_CODE[out.dtype], ldo,
            _status_of(a.device)[1], B._stream_of(a.device.index)))
        if status:
            B._check(status, "ssgd_fp4_matmul")
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
