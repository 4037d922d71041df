"""Host-side checks of the calls around the step (tables of tensors, 4-bit operands): refusals and sizes, no GPU."""
import ctypes
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import fp4_reference as ref  # noqa: E402

A = 0x10000          # a fake, aligned address: these calls must fail before touching it
OK, NULL, ALIGN, SIZE, ARG = 0, 1, 2, 3, 4


@pytest.fixture(scope="module")
def B():
    from paper_1802_04434_b200 import _build, binding
    _build.build()
    binding.lib()
    return binding


def table_size(B, entries, groups):
    arr = (B._Tensor * max(1, len(entries)))(*[B._Tensor(*e) for e in entries])
    out = [ctypes.c_size_t() for _ in range(3)]
    st = B.lib().ssgd_table_size(arr, len(entries), groups, *[ctypes.byref(o) for o in out])
    return st, [o.value for o in out], arr


def test_table_sizes_and_refusals(B):
    # (src, dst, n, src_type, dst_type, group, reserved)
    assert table_size(B, [(A, A, 8192, 0, 0, 0, 0), (A, None, 8193, 1, 0, 1, 0), (None, None, 0, 0, 0, 1, 0)], 2)[:2] == (OK, [3, 32 + 3 * 32, 32])
    assert table_size(B, [], 1)[:2] == (OK, [0, 32, 16])
    assert table_size(B, [(None, None, 1, 0, 0, 0, 0)], 1)[0] == NULL
    assert table_size(B, [(A + 2, A, 1, 0, 0, 0, 0)], 1)[0] == ALIGN
    assert table_size(B, [(A + 2, A + 2, 1, 1, 0, 0, 0)], 1)[0] == ALIGN
    assert table_size(B, [(A + 2, A + 2, 1, 1, 2, 0, 0)], 1)[0] == OK
    assert table_size(B, [(A, A, 1, 3, 0, 0, 0)], 1)[0] == ARG
    assert table_size(B, [(A, A, 1, 0, 0, 1, 0)], 1)[0] == ARG              # group out of range
    assert table_size(B, [(A, A, 1, 0, 0, 1, 0), (A, A, 1, 0, 0, 0, 0)], 2)[0] == ARG   # groups out of order
    assert table_size(B, [], 0)[0] == SIZE and table_size(B, [], 1025)[0] == SIZE
    assert table_size(B, [(A, A, 1 << 49, 0, 0, 0, 0)], 1)[0] == SIZE
    assert B.lib().ssgd_table_size(None, 1, 1, None, None, None) == NULL


def test_table_contents(B):
    st, (tiles, nbytes, _), arr = table_size(B, [(A, A, 8193, 0, 1, 0, 0), (A + 64, None, 5, 2, 0, 2, 0)], 4)
    assert st == OK and tiles == 3
    buf = np.zeros(nbytes + 8, dtype=np.uint8)
    buf[nbytes:] = 0xA5
    assert B.lib().ssgd_table_build(arr, 2, 4, buf.ctypes.data, nbytes) == OK
    assert (buf[nbytes:] == 0xA5).all()
    first = buf[:40].view(np.uint64)
    assert first.tolist() == [0, 2, 2, 3, 3]
    e = buf[64:64 + 96].reshape(3, 32)
    src, dst = e[:, :8].copy().view(np.uint64).ravel(), e[:, 8:16].copy().view(np.uint64).ravel()
    n, group = e[:, 16:20].copy().view(np.uint32).ravel(), e[:, 20:24].copy().view(np.uint32).ravel()
    assert src.tolist() == [A, A + 4 * 8192, A + 64] and dst.tolist() == [A, A + 2 * 8192, 0]
    assert n.tolist() == [8192, 1, 5] and group.tolist() == [0, 0, 2]
    assert B.lib().ssgd_table_build(arr, 2, 4, buf.ctypes.data, nbytes - 1) == SIZE
    assert B.lib().ssgd_table_build(arr, 2, 4, None, nbytes) == NULL


def test_norm_and_clip_refusals(B):
    f, g = B.lib().ssgd_tensors_norm, B.lib().ssgd_tensors_clip
    assert f(None, 1, 1, 0, A, A, None) == NULL and f(A, 1, 1, 0, None, A, None) == NULL and f(A, 1, 1, 0, A, None, None) == NULL
    assert f(A + 8, 1, 1, 0, A, A, None) == ALIGN and f(A, 1, 1, 0, A + 4, A, None) == ALIGN and f(A, 1, 1, 0, A, A + 2, None) == ALIGN
    assert f(A, 1, 0, 0, A, A, None) == SIZE and f(A, 1, 1025, 0, A, A, None) == SIZE and f(A, 1 << 40, 1, 0, A, A, None) == SIZE
    assert f(A, 1, 1, 2, A, A, None) == ARG
    for bad in (-1.0, float("nan"), -float("inf")):
        assert g(A, 1, 1, 0, bad, 0, A, A, None) == ARG
    assert g(None, 1, 1, 0, 1.0, 0, A, A, None) == NULL


def test_fp4_sizes(B):
    L = B.lib()
    for cols in (0, 1, 31, 32, 33, 1024, 4103):
        assert L.ssgd_fp4_row_bytes(cols) == -(-cols // 32) * 16
        for fmt, b in ((0, 32), (1, 16)):
            for rows in (0, 1, 128, 129):
                assert L.ssgd_fp4_scale_bytes(fmt, rows, cols) == -(-rows // 128) * -(-(-(-cols // b)) // 4) * 512
    assert L.ssgd_fp4_scale_bytes(2, 1, 1) == 0 and L.ssgd_fp4_scale_bytes(0, 1 << 31, 1) == 0


def test_quantise_refusals(B):
    f = B.lib().ssgd_fp4_quantise
    good = dict(x=A, dtype=0, rows=3, cols=40, ldx=40, fmt=1, amax=None, ts=A, codes=A, scales=A, codes_t=A, scales_t=A)

    def call(**k):
        a = {**good, **k}
        return f(a["x"], a["dtype"], a["rows"], a["cols"], a["ldx"], a["fmt"], a["amax"], a["ts"], a["codes"], a["scales"], a["codes_t"], a["scales_t"], None)

    assert call(x=None) == NULL and call(ts=None) == NULL and call(scales=None) == NULL and call(scales_t=None) == NULL
    assert call(codes=None, codes_t=None) == NULL
    assert call(dtype=3) == ARG and call(fmt=2) == ARG
    assert call(ldx=39) == SIZE and call(rows=1 << 31) == SIZE and call(cols=1 << 31, ldx=1 << 31) == SIZE
    assert call(rows=1 << 30, ldx=1 << 40) == SIZE
    assert call(x=A + 2) == ALIGN and call(codes=A + 8) == ALIGN and call(scales=A + 1) == ALIGN and call(codes_t=A + 4) == ALIGN
    assert call(scales_t=A + 8) == ALIGN and call(ts=A + 2) == ALIGN and call(amax=A + 1) == ALIGN
    assert call(rows=0) == OK and call(cols=0) == OK


def test_dequantise_and_product_refusals(B):
    f = B.lib().ssgd_fp4_dequantise
    assert f(None, A, None, 0, 1, 32, A, 0, 32, None) == NULL and f(A, None, None, 0, 1, 32, A, 0, 32, None) == NULL
    assert f(A, A, None, 0, 1, 32, None, 0, 32, None) == NULL
    assert f(A + 1, A, None, 0, 1, 32, A, 0, 32, None) == ALIGN and f(A, A, A + 1, 0, 1, 32, A, 0, 32, None) == ALIGN
    assert f(A, A, None, 0, 1, 32, A + 2, 0, 32, None) == ALIGN
    assert f(A, A, None, 0, 2, 32, A, 0, 31, None) == SIZE and f(A, A, None, 7, 1, 32, A, 0, 32, None) == ARG
    assert f(A, A, None, 0, 0, 32, A, 0, 32, None) == OK
    g = B.lib().ssgd_fp4_matmul
    good = dict(a=A, sa=A, ta=None, b=A, sb=A, tb=None, M=4, N=8, K=64, fmt=0, out=A, dtype=1, ldo=8, status=A)

    def call(**k):
        v = {**good, **k}
        return g(v["a"], v["sa"], v["ta"], v["b"], v["sb"], v["tb"], v["M"], v["N"], v["K"], v["fmt"], v["out"], v["dtype"], v["ldo"], v["status"], None)

    for k in ("a", "sa", "b", "sb", "out", "status"):
        assert call(**{k: None}) == NULL, k
    for k in ("a", "sa", "b", "sb"):
        assert call(**{k: A + 8}) == ALIGN, k
    assert call(out=A + 1) == ALIGN and call(ta=A + 2) == ALIGN and call(tb=A + 2) == ALIGN and call(status=A + 2) == ALIGN
    assert call(fmt=3) == ARG and call(dtype=9) == ARG
    assert call(ldo=7) == SIZE and call(M=1 << 31) == SIZE and call(N=1 << 31, ldo=1 << 31) == SIZE and call(K=1 << 31) == SIZE
    assert call(M=0) == OK and call(N=0) == OK


def test_reference_formats():
    """The restatement that the GPU tests lean on, against values written out by hand."""
    assert ref.E4M3[[0, 1, 8, 56, 126]].tolist() == [0.0, 2.0 ** -9, 2.0 ** -6, 1.0, 448.0]
    x = np.zeros((1, 32), dtype=np.float32)
    x[0, :10] = [6.0, 5.0, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, -0.3, 7.9]
    code, byte, _ = ref.quantise(x, "mx")                       # largest 7.9: exponent 2, scale 1
    assert byte.tolist() == [[127]] and code[0, :10].tolist() == [7, 6, 6, 4, 4, 2, 2, 0, 9, 7]
    x[0, 9] = 0
    code, byte, ts = ref.quantise(x, "nv")                      # 6 = 1.5 * 2^2 > 1.3125 * 2^2: 2^-8; 6 / 2^-8 / 6 = 256
    assert ts == 2.0 ** -8 and byte.tolist() == [[0x78, 1]]
    assert code[0, :9].tolist() == [7, 6, 6, 4, 4, 2, 2, 0, 9]
    assert ref.tensor_scale(2688.0) == 1.0 and ref.tensor_scale(2688.1) == 2.0 and ref.tensor_scale(0.0) == 1.0
    assert ref.pack_codes(np.array([[1, 2, 3]], dtype=np.uint8))[0, :3].tolist() == [0x21, 3, 0]
    s = ref.pack_scales(np.arange(129 * 5, dtype=np.int64).reshape(129, 5).astype(np.uint8))
    assert s.size == 2 * 2 * 512 and s[33 % 32 * 16 + 4 + 2] == (33 * 5 + 2) % 256 and s[2 * 512] == (128 * 5) % 256


def test_block_calls(B):
    """The calls with their arguments in one block refuse what the others refuse."""
    import struct
    L = B.lib()
    for f in (L.ssgd_tensors_clip_block, L.ssgd_fp4_quantise_block, L.ssgd_fp4_dequantise_block, L.ssgd_fp4_matmul_block):
        assert f(None) == NULL
    clip = lambda *a: L.ssgd_tensors_clip_block(B._CLIP_ARGS.pack(*a))  # noqa: E731
    assert clip(A, 1, 1, 0, -1.0, 0, A, A, 0) == ARG and clip(0, 1, 1, 0, 1.0, 0, A, A, 0) == NULL and clip(A, 1, 1025, 0, 1.0, 0, A, A, 0) == SIZE
    assert clip(A, 1, 1, 0, float("nan"), 0, A, A, 0) == ARG and clip(A, 1, 1, 0, 1.0, 0, A, A + 2, 0) == ALIGN
    q = lambda *a: L.ssgd_fp4_quantise_block(B.FP4_QUANTISE_ARGS.pack(*a))  # noqa: E731
    assert q(A, 0, 3, 40, 39, 1, 0, A, A, A, A, A, 0) == SIZE and q(A, 0, 0, 40, 40, 1, 0, A, A, A, A, A, 0) == OK
    assert q(A, 0, 3, 40, 40, 2, 0, A, A, A, A, A, 0) == ARG and q(A, 0, 3, 40, 40, 1, 0, A, A + 8, A, A, A, 0) == ALIGN
    d = lambda *a: L.ssgd_fp4_dequantise_block(B.FP4_DEQUANTISE_ARGS.pack(*a))  # noqa: E731
    assert d(A, A, 0, 0, 2, 32, A, 0, 31, 0) == SIZE and d(A, A, 0, 0, 0, 32, A, 0, 32, 0) == OK and d(0, A, 0, 0, 2, 32, A, 0, 32, 0) == NULL
    m = lambda *a: L.ssgd_fp4_matmul_block(B.FP4_MATMUL_ARGS.pack(*a))  # noqa: E731
    assert m(A, A, 0, A, A, 0, 4, 8, 64, 0, A, 1, 7, A, 0) == SIZE and m(A, A, 0, A, A, 0, 0, 8, 64, 0, A, 1, 8, A, 0) == OK
    assert m(A, A, 0, A, A, 0, 4, 8, 64, 0, A, 1, 8, 0, 0) == NULL and struct.calcsize(B.FP4_MATMUL_ARGS.format) == 15 * 8
