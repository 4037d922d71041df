"""Norm and clipping over many tensors, 4-bit quantisation and products: parity on a B200 against plain forms in 64 bits."""
import math
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import fp4_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
HALF_ULP = {t: torch.finfo(t).eps / 2 for t in (F32, BF16, F16)}     # unit roundoff of each type


@pytest.fixture(scope="module")
def B():
    from paper_1802_04434_b200 import binding
    binding.lib()
    return binding


@pytest.fixture(scope="module")
def fp4(B):
    from paper_1802_04434_b200 import fp4
    return fp4


def randn(*shape, seed=0, dtype=F32, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def f64(t):
    return t.detach().double().cpu().numpy()


# ---------------------------------------------------------------------------------------------------------------------
# norm and clipping


def clip_reference(groups, max_norm, kind):
    """Norms and clipped tensors in 64 bits; groups: list of lists of float64 arrays."""
    norms, out = [], []
    for g in groups:
        flat = np.concatenate([t.reshape(-1) for t in g]) if g else np.zeros(0)
        with np.errstate(all="ignore"):
            n = math.sqrt(float((flat ** 2).sum())) if kind == "two" else float(np.abs(flat).max()) if flat.size else 0.0
        norms.append(n)
        c = max_norm / n if n > max_norm else 1.0
        out.append([t * c for t in g])
    return norms, out


def check_clip(B, sizes_by_group, src_type, dst_type, max_norm, kind="two", offset=0, scale=1e-2, seed=0):
    """Tensors end to end (from `offset` elements past an aligned start), rows with canaries between the tensors."""
    src, dst, groups, holders = [], [], [], []
    for w, sizes in enumerate(sizes_by_group):
        flat = randn(sum(sizes) + offset, seed=seed + w, dtype=src_type, scale=scale * (1 + w))
        row = torch.full((sum(sizes) + 3 * len(sizes) + offset,), 7.0, dtype=dst_type, device="cuda")
        holders.append((flat, row, sizes))
        o = p = offset
        for n in sizes:
            src.append(flat[o:o + n]); dst.append(row[p:p + n]); groups.append(w)
            o += n; p += n + 3
    W = len(sizes_by_group)
    table = B.TensorTable(src, dst, groups, workers=W)
    norms = torch.full((W,), -1.0, device="cuda")
    B.tensors_clip(table, max_norm, norms, kind)
    torch.cuda.synchronize()
    expect, rows = clip_reference([[f64(t) for t, g in zip(src, groups) if g == w] for w in range(W)], max_norm, kind)
    got = norms.tolist()
    for w in range(W):
        # fp64 sums of exact squares, one rounding to fp32
        assert abs(got[w] - expect[w]) <= 2.0 ** -23 * expect[w] + 1e-45, (w, got[w], expect[w])
    it = iter(dst)
    for w, (flat, row, sizes) in enumerate(holders):
        for k, n in enumerate(sizes):
            t = f64(next(it))
            want = rows[w][k]
            # the norm's, the quotient's and the product's roundings (four half ulps of fp32 at most), then the type's
            tol = (4 * 2.0 ** -24 + HALF_ULP[dst_type]) * np.abs(want) + (2.0 ** -25 if dst_type == F16 else 0.0)
            assert (np.abs(t - want) <= tol).all()
        gap, p = row.clone(), offset
        for n in sizes:
            gap[p:p + n] = 7.0
            p += n + 3
        assert bool((gap == 7.0).all()), "an element between the tensors was written"
    again = torch.zeros(W, device="cuda")
    B.tensors_norm(table, again, kind)
    assert torch.equal(again, norms)     # no atomics: equal inputs give equal bits


@pytest.mark.parametrize("src", [F32, BF16, F16])
@pytest.mark.parametrize("dst", [F32, BF16, F16])
@pytest.mark.parametrize("kind", ["two", "max"])
def test_clip_types(B, src, dst, kind):
    check_clip(B, [[5, 1, 8192, 8193, 100], [4096, 3]], src, dst, 0.05, kind)


@pytest.mark.parametrize("offset", [0, 1, 2, 3, 4, 5, 7])
@pytest.mark.parametrize("src", [F32, BF16])
def test_clip_alignments(B, src, offset):
    check_clip(B, [[1, 2, 3, 4, 5, 1000, 8191, 8192, 20000]], src, F32, 1.0, offset=offset)


@pytest.mark.parametrize("sizes", [[[]], [[0]], [[1]], [[0, 0, 3], [], [2, 0]], [[1] * 1500], [[7, 300_001], [65_536], [1], [123_457]],
                                   [[3_000_017, 11, 2_000_003]]])
@pytest.mark.parametrize("max_norm", [0.0, 0.5, math.inf])
def test_clip_sizes(B, sizes, max_norm):
    check_clip(B, sizes, F32, F32, max_norm)


def test_clip_many_workers(B):
    check_clip(B, [[i % 5 * 100 + 1, 33] for i in range(1024)], BF16, F32, 0.3)


def test_norm_beyond_fp32_squares(B):
    x = torch.tensor([1e30, 2e30, -2e30], device="cuda")
    y = torch.full((1000,), 1e-30, device="cuda")
    out = torch.empty_like(x)
    norms = torch.zeros(2, device="cuda")
    B.tensors_clip(B.TensorTable([x, y], [out, None], [0, 1]), 3.0, norms)
    assert abs(norms[0].item() - 3e30) <= 3e30 * 2.0 ** -22
    assert abs(norms[1].item() - 1e-30 * math.sqrt(1000)) <= 4e-29 * 2.0 ** -22
    assert torch.allclose(out, torch.tensor([1.0, 2.0, -2.0], device="cuda"), rtol=1e-6)


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("kind", ["two", "max"])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_clip_nonfinite(B, bad, kind, dtype):
    x = randn(3, 20_000, seed=1, dtype=dtype)
    x[1, 12_345] = bad
    before = x.clone()
    norms = torch.zeros(3, device="cuda")
    out = torch.full((3, 20_000), 5.0, device="cuda")
    table = B.TensorTable(list(x), list(out), [0, 1, 2])
    B.tensors_clip(table, 1.0, norms, kind, zero_nonfinite=True)
    n = norms.tolist()
    assert math.isfinite(n[0]) and math.isfinite(n[2])
    assert math.isnan(n[1]) if math.isnan(bad) else n[1] == math.inf
    assert bool((out[1] == 0).all()) and bool((out[0] != 0).any()) and bool((out[2] != 5.0).all())
    B.tensors_clip(table, 1.0, norms, kind)
    if math.isnan(bad):
        assert bool(out[1].isnan().all())
    else:
        assert bool(out[1, 12_345].isnan()) and bool((out[1, :12_345] == 0).all())
    assert torch.equal(before.view(torch.int16 if dtype != F32 else torch.int32), x.view(torch.int16 if dtype != F32 else torch.int32))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_clip_in_place(B, dtype):
    x = randn(50_001, seed=3, dtype=dtype)
    want = x.double()
    n = float(want.norm())
    norms = torch.zeros(1, device="cuda")
    table = B.TensorTable([x[:17], x[17:]], [x[:17], x[17:]])
    B.tensors_clip(table, 2 * n, norms)                       # nothing to clip: not a bit changes
    assert torch.equal(x.double(), want)
    B.tensors_clip(table, n / 8, norms)
    assert float((x.double() - want / 8).abs().max()) <= float(want.abs().max()) / 8 * 2 * HALF_ULP[dtype] + 1e-12
    B.tensors_norm(table, norms)
    assert abs(norms.item() - n / 8) < n / 8 * 2.0 ** -8


def test_clip_on_a_stream_of_its_own(B):
    s = torch.cuda.Stream()
    x = randn(1_000_003, seed=4)
    out, norms = torch.zeros_like(x), torch.zeros(1, device="cuda")
    table = B.TensorTable([x], [out])
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        x.mul_(2.0)
        B.tensors_clip(table, 1.0, norms)
        y = out.clone()
    s.synchronize()
    assert abs(float(y.double().norm()) - 1.0) < 1e-6


def test_clip_in_a_graph(B):
    x = randn(300_000, seed=5)
    out, norms = torch.zeros_like(x), torch.zeros(1, device="cuda")
    table = B.TensorTable([x[:100], x[100:]], [out[:100], out[100:]])
    B.tensors_clip(table, 1.0, norms)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.tensors_clip(table, 1.0, norms)
    for k in (2.0, 5.0):
        x.mul_(k)
        g.replay()
        torch.cuda.synchronize()
        assert abs(norms.item() - float(x.double().norm())) <= norms.item() * 2.0 ** -23
        assert abs(float(out.double().norm()) - 1.0) < 1e-6


# ---------------------------------------------------------------------------------------------------------------------
# quantisation


def check_packed(p, x64, fmt, amax=None):
    code, byte, ts = ref.quantise(x64.astype(np.float32), fmt, amax)
    assert np.array_equal(p.codes.cpu().numpy(), ref.pack_codes(code))
    assert np.array_equal(p.scales.cpu().numpy(), ref.pack_scales(byte))
    if fmt == "nv":
        assert p.tensor_scale[0].item() == ts
    return ref.values(code, byte, ts, fmt)


SIDES = [(1, 1), (1, 16), (1, 31), (3, 33), (8, 1024), (16, 64), (31, 257), (127, 128), (128, 127), (129, 130), (200, 513), (1024, 96),
         (1000, 1), (257, 4100), (384, 640)]


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows,cols", SIDES)
def test_quantise(fp4, rows, cols, dtype, fmt):
    x = randn(rows, cols, seed=rows * 7 + cols, dtype=dtype) * torch.exp(randn(rows, 1, seed=2)).to(dtype)
    p, pt = fp4.quantise_both(x, fmt)
    v = check_packed(p, f64(x), fmt)
    vt = check_packed(pt, f64(x).T, fmt)
    for out in (F32, BF16, F16):
        for q, w in ((p, v), (pt, vt)):
            got, want = fp4.dequantise(q, out), torch.from_numpy(w).to(F32).to(out)
            assert torch.equal(got.cpu(), want)
    one, other = fp4.quantise(x, fmt), fp4.quantise_columns(x, fmt)
    for a, b in ((one, p), (other, pt)):
        assert torch.equal(a.codes, b.codes) and torch.equal(a.scales, b.scales)


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("scale", [1e-38, 1e-20, 1e-4, 1.0, 1e10, 1e37])
def test_quantise_ranges(fp4, fmt, scale):
    x = randn(130, 200, seed=9).clamp(-3, 3) * torch.exp(2 * randn(130, 200, seed=10).clamp(-3, 3)) * 1e-3 * scale
    x[5] = 0
    x[7, :40] = 0
    x[9, 3] = -0.0
    p, pt = fp4.quantise_both(x, fmt)
    check_packed(p, f64(x), fmt)
    check_packed(pt, f64(x).T, fmt)


@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_quantise_ties(fp4, fmt):
    # every multiple of 1/8 up to 6 in blocks whose scale is a power of two, then blocks of every E4M3 fraction
    v = torch.arange(-48, 49, device="cuda") / 8.0
    x = torch.zeros(64, 16 * 97 * 2, device="cuda")
    x[:, 0::16] = 6.0
    x[:, 1::16] = v.repeat(2)
    x[:, 2::16] = v.roll(7).repeat(2)
    x *= (1 + torch.arange(64, device="cuda") % 8 / 8.0)[:, None] * 2.0 ** (torch.arange(64, device="cuda") // 8)[:, None]
    for dtype in (F32, BF16, F16):
        p, pt = fp4.quantise_both(x.to(dtype), fmt)
        check_packed(p, f64(x.to(dtype)), fmt)
        check_packed(pt, f64(x.to(dtype)).T, fmt)


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_quantise_nonfinite(fp4, fmt, bad):
    x = randn(200, 300, seed=11, dtype=BF16)
    x[3, 250] = bad
    x[150, 299] = bad
    p, pt = fp4.quantise_both(x, fmt)
    check_packed(p, f64(x), fmt)
    check_packed(pt, f64(x).T, fmt)
    b = ref.BLOCK[fmt]
    back = fp4.dequantise(p).isnan().cpu().numpy()
    want = np.zeros((200, 300), dtype=bool)
    want[3, 250 // b * b:250 // b * b + b] = True
    want[150, 299 // b * b:] = True
    assert np.array_equal(back, want)


def test_quantise_with_a_given_amax(fp4, B):
    x = randn(100, 200, seed=12, dtype=BF16)
    norms = torch.zeros(1, device="cuda")
    B.tensors_norm(B.TensorTable([x]), norms, "max")
    a, b = fp4.quantise(x, "nv"), fp4.quantise(x, "nv", norms)
    assert torch.equal(a.codes, b.codes) and torch.equal(a.scales, b.scales) and a.tensor_scale[0] == b.tensor_scale[0]
    for amax in (1e-3, 1e-30, 100.0, 1e30):       # too small saturates, too large loses small blocks, neither breaks
        p = fp4.quantise(x, "nv", torch.tensor([amax], device="cuda"))
        check_packed(p, f64(x), "nv", np.float32(amax))


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_quantise_strided_rows(fp4, fmt, dtype):
    base = randn(70, 333, seed=13, dtype=dtype)
    for x in (base[:, 1:300], base[::2, 5:], base[3:4], base.t(), base[:, :1], base[:, 128:256]):
        p, pt = fp4.quantise_both(x, fmt)
        check_packed(p, f64(x), fmt)
        check_packed(pt, f64(x).T, fmt)


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("rows,cols", [(0, 5), (5, 0), (0, 0)])
def test_quantise_empty(fp4, fmt, rows, cols):
    x = torch.zeros(rows, cols, device="cuda")
    p, pt = fp4.quantise_both(x, fmt)
    assert fp4.dequantise(p).shape == (rows, cols) and fp4.dequantise(pt).shape == (cols, rows)


def test_quantise_leaves_its_surroundings_alone(B):
    for fmt in ("mx", "nv"):
        rows, cols = 131, 77
        x = randn(rows, cols, seed=14)
        n = [rows * B.fp4_row_bytes(cols), B.fp4_scale_bytes(fmt, rows, cols), cols * B.fp4_row_bytes(rows), B.fp4_scale_bytes(fmt, cols, rows)]
        bufs = [torch.full((k + 64,), 0xA5, dtype=torch.uint8, device="cuda") for k in n]
        ts = torch.full((4,), 9.0, device="cuda")
        B.fp4_quantise(x, rows, cols, cols, fmt, None, ts, *bufs)
        for k, b in zip(n, bufs):
            assert bool((b[k:] == 0xA5).all())
        assert ts[2:].tolist() == [9.0, 9.0]
        out = torch.full((rows * 80 + 16,), 3.0, device="cuda")
        B.fp4_dequantise(bufs[0], bufs[1], ts, fmt, rows, cols, out, 80)
        o = out[:rows * 80].view(rows, 80)
        assert bool((o[:, cols:] == 3.0).all()) and bool((out[rows * 80:] == 3.0).all())


# ---------------------------------------------------------------------------------------------------------------------
# product


def values_of(p):
    """float64 values of a packed operand, from its bytes."""
    code = p.codes.cpu().numpy()
    code = np.stack((code & 15, code >> 4), 2).reshape(p.rows, -1)[:, :p.cols]
    nb = -(-p.cols // ref.BLOCK[p.fmt])
    tk = -(-nb // 4)
    r, k = np.meshgrid(np.arange(p.rows), np.arange(nb), indexing="ij")
    byte = p.scales.cpu().numpy()[((r // 128) * tk + k // 4) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + k % 4]
    return ref.values(code, byte, p.tensor_scale[0].item() if p.tensor_scale is not None else 1.0, p.fmt)


def check_product(a, b, got, dtype):
    va, vb = values_of(a), values_of(b)
    want, total = va @ vb.T, np.abs(va) @ np.abs(vb).T
    # any order of K additions with one ulp (2^-23) of a partial sum lost in each, then the type's rounding
    tol = a.cols * 2.0 ** -23 * total + HALF_ULP[dtype] * np.abs(want) + (2.0 ** -25 if dtype == F16 else 0.0)
    off = np.abs(f64(got) - want)
    assert (off <= tol).all(), (off / np.maximum(tol, 1e-300)).max()


PRODUCTS = [(1, 1, 1), (1, 1, 32), (1, 128, 64), (1, 129, 256), (2, 8, 96), (3, 1000, 4096), (7, 65, 100), (8, 128, 128), (9, 300, 1024), (16, 16, 16),
            (17, 257, 2600), (33, 5, 513), (64, 512, 320), (100, 100, 1000), (128, 128, 64), (128, 256, 256), (129, 255, 257), (200, 300, 4097),
            (256, 128, 512), (257, 129, 1056), (300, 1, 700), (1, 5003, 777), (512, 640, 768), (777, 1111, 1500), (2500, 70, 190)]


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("M,N,K", PRODUCTS)
def test_product(fp4, M, N, K, fmt):
    a = fp4.quantise(randn(M, K, seed=M + K) * torch.exp(randn(M, 1, seed=1)), fmt)
    b = fp4.quantise(randn(N, K, seed=N * 3 + K, scale=0.02, dtype=BF16), fmt)
    for dtype in (F32, BF16, F16):
        check_product(a, b, fp4.matmul(a, b, dtype), dtype)
    fp4.check()


@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_product_of_every_code_and_scale(fp4, fmt):
    """Operands set byte by byte: each row its own code pattern, each block its own scale."""
    g = np.random.default_rng(5)
    M, N, K = 140, 150, 512
    nb = K // ref.BLOCK[fmt]

    def operand(rows):
        code = g.integers(0, 16, (rows, K)).astype(np.uint8)
        byte = (g.integers(100, 150, (rows, nb)) if fmt == "mx" else g.integers(0, 127, (rows, nb))).astype(np.uint8)
        ts = torch.tensor([2.0 ** -5], device="cuda") if fmt == "nv" else None
        return fp4.Packed(torch.from_numpy(ref.pack_codes(code)).cuda(), torch.from_numpy(ref.pack_scales(byte)).cuda(), ts, rows, K, fmt)

    a, b = operand(M), operand(N)
    check_product(a, b, fp4.matmul(a, b, F32), F32)
    one = fp4.Packed(a.codes[:1].contiguous(), a.scales, a.tensor_scale, 1, K, fmt)
    check_product(one, b, fp4.matmul(one, b, F32), F32)
    fp4.check()


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("M", [1, 5, 40, 150])
def test_product_rows_do_not_touch_one_another(fp4, fmt, M):
    """A row of NaN scales spoils its own outputs only; what lies behind the operands' last row does not matter."""
    x, w = randn(M + 3, 640, seed=21), randn(300, 640, seed=22)
    x[M // 2, 77] = math.nan
    w[123, 600] = math.inf
    a, b = fp4.quantise(x[:M], fmt), fp4.quantise(w, fmt)
    rows = -(-M // 128) * 128
    scales = a.scales.view(-1, a.scales.numel() // (rows // 128) // 512, 32, 4, 4).clone()      # [row tile][k tile][row % 32][row / 32][block]
    for r in range(M, rows):
        scales[r // 128, :, r % 32, r % 128 // 32, :] = 255 if fmt == "mx" else 0x7F
    a = a._replace(scales=scales.view(-1))
    bad = fp4.matmul(a, b, F32).isnan()
    want = torch.zeros_like(bad)
    want[M // 2] = True
    want[:, 123] = True
    assert torch.equal(bad, want)
    fp4.check()


def test_product_into_a_view_and_with_k_zero(fp4):
    a, b = fp4.quantise(randn(20, 100, seed=31)), fp4.quantise(randn(30, 100, seed=32))
    base = torch.full((20, 50), 4.0, device="cuda")
    fp4.matmul(a, b, F32, out=base[:, 7:37])
    check_product(a, b, base[:, 7:37], F32)
    assert bool((base[:, :7] == 4).all()) and bool((base[:, 37:] == 4).all())
    z = fp4.matmul(fp4.quantise(torch.zeros(3, 0, device="cuda")), fp4.quantise(torch.zeros(5, 0, device="cuda")), BF16)
    assert z.shape == (3, 5) and bool((z == 0).all())
    assert fp4.matmul(fp4.quantise(torch.zeros(0, 64, device="cuda")), b._replace(cols=64, codes=b.codes[:, :32].contiguous())).shape == (0, 30)


def test_product_twice_and_on_a_stream(fp4):
    a, b = fp4.quantise(randn(300, 2000, seed=41), "nv"), fp4.quantise(randn(500, 2000, seed=42), "nv")
    first = fp4.matmul(a, b, F32)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        second = fp4.matmul(a, b, F32)
    s.synchronize()
    assert torch.equal(first, second)
    fp4.check()


# ---------------------------------------------------------------------------------------------------------------------
# linear layer


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("tokens,n_in,n_out", [(1, 64, 32), (50, 100, 70), (256, 384, 512), (333, 500, 257)])
def test_linear_gradient_is_the_formulas(fp4, tokens, n_in, n_out, fmt):
    x, w, dy = randn(tokens, n_in, seed=51, dtype=BF16), randn(n_out, n_in, seed=52, scale=0.05), randn(tokens, n_out, seed=53, dtype=BF16, scale=1e-3)
    y, kept = fp4.linear_forward(x, w, fmt)
    dw_out = torch.empty(n_out, n_in, device="cuda")
    dx, dw = fp4.linear_backward(kept, dy, dw_out)
    assert dw is dw_out and y.dtype == BF16 and dx.dtype == BF16
    check_product(fp4.quantise(x, fmt), fp4.quantise(w, fmt), y, BF16)
    check_product(fp4.quantise(dy, fmt), fp4.quantise(w.t().contiguous(), fmt), dx, BF16)
    check_product(fp4.quantise(dy.t().contiguous(), fmt), fp4.quantise(x.t().contiguous(), fmt), dw, F32)
    xa, wa = x.clone().requires_grad_(), w.clone().requires_grad_()
    ya = fp4.linear(xa, wa, fmt)
    ya.backward(dy)
    assert torch.equal(ya, y) and torch.equal(xa.grad, dx) and torch.equal(wa.grad, dw)


@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_linear_gradient_against_differences(fp4, fmt):
    """On values that 4 bits hold exactly the layer is linear, so a difference over one step of a value is the derivative."""
    g = torch.Generator(device="cuda")
    g.manual_seed(6)
    T, I, O = 64, 64, 32
    pick = lambda *s: torch.tensor([-4.0, -2.0, -1.0, 1.0, 2.0, 4.0], device="cuda")[torch.randint(0, 6, s, generator=g, device="cuda")]  # noqa: E731
    x, w, dy = pick(T, I), pick(O, I), pick(T, O)
    for t in (x, w, dy):                # every block of either direction holds a 6, at places left alone below: all scales are 1
        t[::16] = 6.0
        t[:, ::16] = 6.0
    y, kept = fp4.linear_forward(x, w, fmt)
    dx, dw = fp4.linear_backward(kept, dy)
    for i, j in ((1, 1), (5, 40), (63, 63), (17, 2)):
        for t, grad in ((x, dx), (w, dw)):
            i2 = i % t.shape[0]
            moved = t.clone()
            moved[i2, j] = 3.0 if t[i2, j] != 3.0 else 2.0
            out = fp4.linear_forward(moved if t is x else x, moved if t is w else w, fmt)[0]
            change = ((out - y).double() * dy.double()).sum().item()
            assert change == (moved[i2, j] - t[i2, j]).item() * grad[i2, j].item()


# ---------------------------------------------------------------------------------------------------------------------
# together


@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_training_example(fmt):
    """Products in 4 bits, clipping into the workers' rows and the vote, as the example runs them: the loss falls."""
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import train_fp4_signum as example
    losses, norms, net, task = example.train(steps=150, workers=3, fmt=fmt)
    assert all(math.isfinite(v) for v in losses + norms) and all(n > 0 for n in norms)
    assert sum(losses[-10:]) < 0.5 * sum(losses[:10])
    assert math.isfinite(example.serve(net, task))


def test_clipped_rows_feed_the_step(B):
    """bf16 tensors through tensors_clip and signsgd_step against the step on rows clipped in 64 bits."""
    sizes, M = [100, 33, 4096, 7], 5
    d = sum(-(-n // 32) * 32 for n in sizes)
    src = [randn(n, seed=100 * w + n, dtype=BF16, scale=3.0 ** w) for w in range(M) for n in sizes]
    rows = torch.zeros(M, d, device="cuda")
    dst = [p[:n] for row in rows for p, n in zip(row.split([-(-n // 32) * 32 for n in sizes]), sizes)]
    norms = torch.zeros(M, device="cuda")
    B.tensors_clip(B.TensorTable(src, dst, [w for w in range(M) for _ in sizes]), 10.0, norms)
    for w in range(M):
        flat = torch.cat([t.double() for t in src[w * len(sizes):(w + 1) * len(sizes)]])
        c = min(1.0, 10.0 / float(flat.norm()))
        got = torch.cat([t for t in dst[w * len(sizes):(w + 1) * len(sizes)]])
        assert torch.equal(got > 0, flat > 0) and float((got.double() - flat * c).abs().max()) <= 4 * 2.0 ** -24 * float((flat * c).abs().max())
    words = -(-d // 128) * 4
    x, m = torch.zeros(d, device="cuda"), torch.zeros(M, d, device="cuda")
    bits, vote = torch.zeros(M, words, dtype=torch.int32, device="cuda"), torch.zeros(-(-d // 32), dtype=torch.int32, device="cuda")
    B.signsgd_step(x, rows, m, M, d, d, 0.9, 1.0, bits, words, vote)
    votes = torch.where(rows < 0, -1, 1).sum(0)
    assert torch.equal(x, torch.where(votes >= 0, -1.0, 1.0))


def test_product_in_a_graph(fp4):
    x, w = randn(150, 700, seed=61, dtype=BF16), fp4.quantise(randn(300, 700, seed=62), "nv")
    out = torch.zeros(150, 300, device="cuda")
    fp4.matmul(fp4.quantise(x, "nv"), w, out=out)             # first call: attributes, the status word
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        fp4.matmul(fp4.quantise(x, "nv"), w, out=out)
    for seed in (63, 64):
        x.copy_(randn(150, 700, seed=seed, dtype=BF16))
        g.replay()
        torch.cuda.synchronize()
        check_product(fp4.quantise(x, "nv"), w, out, F32)


def test_linear_layers_share_nothing_over_streams(fp4):
    """Products on two streams at the same time."""
    a = [fp4.quantise(randn(m, 1000, seed=m), "mx") for m in (1, 40, 200, 600)]
    w = fp4.quantise(randn(500, 1000, seed=9), "mx")
    want = [fp4.matmul(p, w, F32) for p in a]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for k in range(40):
        with torch.cuda.stream(streams[k % 2]):
            got.append(fp4.matmul(a[k % 4], w, F32))
    torch.cuda.synchronize()
    assert all(torch.equal(got[k], want[k % 4]) for k in range(40))
    fp4.check()


def test_refusals_of_the_torch_layer(fp4, B):
    x = randn(4, 64)
    with pytest.raises(ValueError):
        fp4.quantise(x, "e4")
    with pytest.raises(ValueError):
        fp4.quantise(x[0], "mx")
    with pytest.raises(ValueError):
        fp4.quantise(x.cpu(), "mx")
    with pytest.raises(TypeError):
        fp4.quantise(x.double(), "mx")
    a = fp4.quantise(x, "mx")
    with pytest.raises(ValueError):
        fp4.matmul(a, fp4.quantise(x, "nv"))
    with pytest.raises(ValueError):
        fp4.matmul(a, fp4.quantise(randn(4, 32), "mx"))
    with pytest.raises(ValueError):
        fp4.matmul(a, a, out=torch.empty(4, 5, device="cuda"))
    with pytest.raises(ValueError):
        fp4.Packed(a.codes[:2].contiguous(), a.scales, None, 4, 64, "mx")
    with pytest.raises(ValueError):
        B.TensorTable([x], [x[:2].contiguous()])
    with pytest.raises(ValueError):
        B.TensorTable([x[:, ::2]])
    with pytest.raises(TypeError):
        B.TensorTable([x.to(torch.int32)])
    with pytest.raises(B.SignSGDError):
        B.tensors_clip(B.TensorTable([x]), -1.0, torch.zeros(1, device="cuda"))
    with pytest.raises(ValueError):
        B.tensors_norm(B.TensorTable([x, x], None, [0, 1]), torch.zeros(1, device="cuda"))


@pytest.mark.parametrize("M,N", [(5, 100), (128, 128), (200, 250), (250, 256)])
@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_waits_of_the_product_run_out(fp4, B, M, N, fmt):
    """Stages that wait for bytes nobody sends: the kernel gives up, says so, writes nothing, and the next product is right."""
    a, b = fp4.quantise(randn(M, 500, seed=71), fmt), fp4.quantise(randn(N, 500, seed=72), fmt)
    out, status = torch.full((M, N), 7.0, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    st = B.lib().ssgd_fp4_matmul_wait_selftest(a.pointers[0], a.pointers[1], b.pointers[0], b.pointers[1], M, N, 500, B.FP4_FORMAT[fmt],
                                               out.data_ptr(), 0, N, status.data_ptr(), torch.cuda.current_stream().cuda_stream)
    assert st == 0
    torch.cuda.synchronize()
    assert status.item() == 1 and bool((out == 7.0).all())
    check_product(a, b, fp4.matmul(a, b, F32), F32)
    fp4.check()


@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_linear_in_autograd(fp4, fmt):
    """Leading sides, a broadcast gradient, inputs that want no gradient."""
    x, w = randn(3, 5, 96, seed=81, dtype=BF16), randn(40, 96, seed=82, scale=0.1)
    xa, wa = x.clone().requires_grad_(), w.clone().requires_grad_()
    y = fp4.linear(xa, wa, fmt)
    assert y.shape == (3, 5, 40)
    y.sum().backward()                                        # dy is one number, expanded
    flat, kept = fp4.linear_forward(x.view(15, 96), w, fmt)
    dx, dw = fp4.linear_backward(kept, torch.ones(15, 40, dtype=BF16, device="cuda"))
    assert torch.equal(y.view(15, 40), flat) and torch.equal(xa.grad.view(15, 96), dx) and torch.equal(wa.grad, dw)
    xb, wb = x.clone().requires_grad_(), w.clone().requires_grad_()
    fp4.linear(xb, w, fmt).sum().backward()
    fp4.linear(x, wb, fmt).sum().backward()
    assert torch.equal(xb.grad, xa.grad) and torch.equal(wb.grad, wa.grad)
    with torch.no_grad():
        assert torch.equal(fp4.linear(x, w, fmt), y)
    z = fp4.linear(torch.zeros(0, 96, device="cuda", requires_grad=True), w.requires_grad_(), fmt)
    z.sum().backward()
    assert z.shape == (0, 40) and bool((w.grad == 0).all())
    with pytest.raises(ValueError):
        fp4.linear(x, w.t(), fmt)


@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_rows_beyond_32_bits(fp4, B, fmt):
    """Rows so far apart that their places pass 2^32 elements and bytes."""
    stride = (1 << 31) + 64
    base = torch.empty(2 * stride + 1024, dtype=BF16, device="cuda")
    x = base.as_strided((3, 200), (stride, 1), 8)
    x.copy_(randn(3, 200, seed=91))
    p, pt = fp4.quantise_both(x, fmt)
    check_packed(p, f64(x), fmt)
    check_packed(pt, f64(x).T, fmt)
    B.fp4_dequantise(p.codes, p.scales, p.tensor_scale, fmt, 3, 200, x, stride)
    assert torch.equal(x, fp4.dequantise(p, BF16))
    del base, x
    a, b = fp4.quantise(randn(150, 320, seed=92), fmt), fp4.quantise(randn(60, 320, seed=93), fmt)
    for rows, ldo in ((150, 1 << 25), (150, (1 << 25) + 1), (100, (1 << 25) + (1 << 24))):
        q = fp4.quantise(randn(rows, 320, seed=92), fmt)
        out = torch.empty(rows * ldo, device="cuda").as_strided((rows, 60), (ldo, 1))
        fp4.matmul(q, b, out=out)
        assert torch.equal(out, fp4.matmul(q, b, F32))
        del out
    fp4.check()


def test_norm_of_more_than_32_bits_of_elements(B):
    n = (1 << 32) + 5
    x = torch.empty(n, dtype=BF16, device="cuda").fill_(0.5)
    norms = torch.zeros(1, device="cuda")
    B.tensors_clip(B.TensorTable([x], [x]), 1.0, norms)
    want = 0.5 * math.sqrt(n)
    assert abs(norms.item() - want) <= want * 2.0 ** -23
    c = torch.tensor(0.5, device="cuda") * (torch.tensor(1.0, device="cuda") / norms[0])
    assert bool((x[-9:] == c.to(BF16)).all()) and bool((x[(1 << 31) - 4:(1 << 31) + 4] == c.to(BF16)).all()) and x[0] == c.to(BF16)
