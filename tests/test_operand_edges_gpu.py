"""Operands, products and clipping where they went wrong once: slices, extreme scales, sums of 16-bit squares; on a B200
against plain forms in 64 bits."""
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


# ---------------------------------------------------------------------------------------------------------------------
# the tensor scale of a slice


@pytest.mark.parametrize("rows,cols,width,dtype", [
    (64, 1111, 1112, BF16), (512, 100, 104, F16), (512, 101, 104, F32), (300, 129, 136, BF16), (33, 2049, 2056, F16), (40, 1000, 1008, BF16),
    (16, 4103, 4104, F32), (9, 8205, 8208, BF16), (2100, 1501, 1504, BF16), (1999, 515, 516, F32), (3000, 33, 40, F16)])
def test_largest_value_in_the_last_columns_of_a_slice(fp4, rows, cols, width, dtype):
    """Rows at multiples of 16 bytes whose last 16-byte piece is not whole: each of its columns holds the largest value once."""
    piece = 128 // torch.finfo(dtype).bits
    base = randn(rows, width, seed=rows + cols, dtype=dtype)
    base[:, cols:] = math.inf                                  # not part of the matrix
    x = base[:, :cols]
    for back in range(1, cols % piece + 1):
        y = x.clone()
        x[(back * 37) % rows, cols - back] = 1000.0
        want = ref.quantise(x.float().cpu().numpy(), "nv")
        for p, t in ((fp4.quantise(x, "nv"), False), (fp4.quantise_columns(x, "nv"), True), (fp4.quantise_both(x, "nv")[0], False)):
            assert p.tensor_scale.tolist() == [want[2], 1000.0]
            if not t:
                assert np.array_equal(p.codes.cpu().numpy(), ref.pack_codes(want[0]))
                assert np.array_equal(p.scales.cpu().numpy(), ref.pack_scales(want[1]))
        x.copy_(y)


# ---------------------------------------------------------------------------------------------------------------------
# tensor scales at the ends of their range


def constant(fp4, rows, K, code, byte, scale, zero_row=None):
    """An nv operand of one code and one scale byte, one row of it zeros."""
    c = np.full((rows, K), code, dtype=np.uint8)
    if zero_row is not None:
        c[zero_row] = 0
    b = np.full((rows, K // 16), byte, dtype=np.uint8)
    return fp4.Packed(torch.from_numpy(ref.pack_codes(c)).cuda(), torch.from_numpy(ref.pack_scales(b)).cuda(),
                      torch.tensor([scale], device="cuda"), rows, K, "nv")


@pytest.mark.parametrize("M,N,K,ldo", [(3, 40, 512, 40), (3, 40, 4096, 40), (200, 300, 512, 301), (200, 300, 512, 304), (150, 300, 8192, 300)])
@pytest.mark.parametrize("ta,tb", [(100, 60), (60, 117), (-80, -70), (-100, -60), (117, -100), (-100, 117), (-90, 117), (64, 64), (-63, -64)])
@pytest.mark.parametrize("code", [2, 7])
def test_product_of_extreme_tensor_scales(fp4, M, N, K, ldo, ta, tb, code):
    """Sums that are exact in fp32, so the result is the formula's, rounded once: infinity or a subnormal where it has to be, and
    zeros stay zeros."""
    for byte in (0x38, 0x7E):                                  # 1 and 448
        a, b = constant(fp4, M, K, code, byte, 2.0 ** ta, zero_row=1), constant(fp4, N, K, code, byte, 2.0 ** tb)
        value = ref.LEVELS[code] * ref.E4M3[byte]
        exact = value * value * K                              # an integer of at most 24 bits times a power of two
        with np.errstate(over="ignore"):
            want = np.float32(exact * 2.0 ** (ta + tb))        # exact in 64 bits before
        for dtype in (F32, BF16):
            out = torch.empty(M, ldo, dtype=dtype, device="cuda")[:, :N]
            fp4.matmul(a, b, out=out)
            expected = torch.full((M, N), float(want), device="cuda").to(dtype)
            expected[1] = 0
            assert torch.equal(out, expected), (byte, dtype, out[0, 0].item(), float(want))
    fp4.check()


# ---------------------------------------------------------------------------------------------------------------------
# waits that run out where k is split over a cluster


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("M,N", [(5, 100), (40, 250), (128, 256)])
def test_waits_of_a_split_product_run_out(fp4, B, fmt, M, N):
    """k is split over a cluster of eight: nobody adds up what its neighbours did not finish, `out` stays as it was."""
    K = 4096
    a, b = fp4.quantise(randn(M, K, seed=1), fmt), fp4.quantise(randn(N, K, seed=2), fmt)
    want = fp4.matmul(a, b, F32)
    out, status = torch.full((M, N), 7.0, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    st = B.lib().ssgd_fp4_matmul_wait_selftest(a.pointers[0], a.pointers[1], b.pointers[0], b.pointers[1], M, N, K, B.FP4_FORMAT[fmt],
                                               out.data_ptr(), 0, N, status.data_ptr(), torch.cuda.current_stream().cuda_stream)
    assert st == 0
    torch.cuda.synchronize()
    assert status.item() == 1 and bool((out == 7.0).all())
    assert torch.equal(fp4.matmul(a, b, F32), want)
    fp4.check()


def test_waits_selftest_refuses_large_products(B):
    A, SIZE = 0x10000, 3
    f = B.lib().ssgd_fp4_matmul_wait_selftest
    for M, N, K in ((257, 8, 64), (8, 257, 64), (8, 8, 4097), (129, 8, 513)):
        assert f(A, A, A, A, M, N, K, 0, A, 0, N, A, None) == SIZE


# ---------------------------------------------------------------------------------------------------------------------
# norms


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("repeats", [1, 1000, 200_000])
@pytest.mark.parametrize("pattern", [[1.0] + [2.0 ** -12] * 7, [2.0 ** -12] * 7 + [1.0], [1.0, 2.0 ** -12, 2.0 ** -12, 2.0 ** -12] * 2,
                                     [1.0, 0.0, 2.0 ** -12, 0.0, 2.0 ** -12, 0.0, 2.0 ** -12, 0.0], [0.0, 1.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0]])
def test_norm_of_16_bit_squares_that_differ_in_size(B, dtype, repeats, pattern):
    """Squares of 2^-24 next to squares of 1: an fp32 sum of many drops them, always to the same side."""
    x = torch.tensor(pattern, dtype=dtype, device="cuda").repeat(repeats)
    norms = torch.zeros(1, device="cuda")
    B.tensors_norm(B.TensorTable([x]), norms)
    want = math.sqrt(repeats * sum(v * v for v in pattern))
    # sums in fp64, one rounding to fp32
    assert abs(norms.item() - want) <= 2.0 ** -23 * want


@pytest.mark.parametrize("n", [1000, 600_000])
@pytest.mark.parametrize("bad", [math.inf, math.nan])
@pytest.mark.parametrize("kind", ["two", "max"])
def test_no_clipping_is_a_copy_whatever_the_norm(B, n, bad, kind):
    x = randn(n, seed=7)
    x[n // 3] = bad
    out, same, norms = torch.zeros_like(x), x.clone(), torch.zeros(1, device="cuda")
    B.tensors_clip(B.TensorTable([x], [out]), math.inf, norms, kind)
    # 1 * NaN is a NaN, of which payload is not said
    assert torch.equal(out.isnan(), x.isnan()) and torch.equal(out.nan_to_num(0.0), x.nan_to_num(0.0)) and not math.isfinite(norms.item())
    B.tensors_clip(B.TensorTable([same], [same]), math.inf, norms, kind)
    assert torch.equal(same.view(torch.int32), x.view(torch.int32))
    B.tensors_clip(B.TensorTable([x], [out]), math.inf, norms, kind, zero_nonfinite=True)
    assert bool((out == 0).all())


@pytest.mark.parametrize("groups", [1, 2, 15, 16])
@pytest.mark.parametrize("elements", [8192, 8 * 8192, 8 * 8192 + 1, 16 * 8192])
@pytest.mark.parametrize("even", [True, False])
def test_norms_around_the_one_launch_form(B, groups, elements, even):
    """Groups of 1, 8, 9 and 16 tiles, each of them or only the last."""
    src = [randn(elements if even or g == groups - 1 else 1, seed=g, dtype=BF16) for g in range(groups)]
    dst, norms = [torch.zeros(t.numel(), device="cuda") for t in src], torch.zeros(groups, device="cuda")
    B.tensors_clip(B.TensorTable(src, dst, list(range(groups))), 0.5, norms)
    for t, d, n in zip(src, dst, norms.tolist()):
        want = float(t.double().norm())
        assert abs(n - want) <= 2.0 ** -23 * want
        c = 0.5 / want if want > 0.5 else 1.0
        assert bool(((d.double() - t.double() * c).abs() <= 4 * 2.0 ** -24 * (t.double() * c).abs()).all())


# ---------------------------------------------------------------------------------------------------------------------
# linear layer


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("lead,n_in,n_out", [((2, 5), 0, 3), ((2, 5), 8, 0), ((5,), 0, 0), ((0, 4), 0, 3), ((2, 0), 8, 0)])
def test_layers_without_inputs_outputs_or_tokens(fp4, fmt, lead, n_in, n_out):
    x, w = randn(*lead, n_in, dtype=BF16).requires_grad_(), randn(n_out, n_in).requires_grad_()
    y = fp4.linear(x, w, fmt)
    assert y.shape == (*lead, n_out) and bool((y == 0).all())
    y.sum().backward()
    assert x.grad.shape == x.shape and w.grad.shape == w.shape and bool((x.grad == 0).all()) and bool((w.grad == 0).all())
    with torch.no_grad():
        assert torch.equal(fp4.linear(x, w, fmt), y)
    fp4.check()


# ---------------------------------------------------------------------------------------------------------------------
# products into slices


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("M,N,K", [(200, 1, 64), (200, 3, 300), (257, 5, 64), (300, 9, 100), (129, 33, 64), (300, 257, 300), (500, 509, 64), (2050, 2057, 300),
                                   (4100, 4101, 300), (20000, 129, 64)])
def test_product_into_a_slice_of_odd_width(fp4, M, N, K, dtype):
    """Rows of out at multiples of 16 bytes, but not its last columns: what lies behind them belongs to somebody else."""
    a, b = fp4.quantise(randn(M, K, seed=1)), fp4.quantise(randn(N, K, seed=2))
    apart = torch.empty(M, N + 1 - N % 2, dtype=dtype, device="cuda")[:, :N]    # rows that start anywhere: stores of one element
    fp4.matmul(a, b, out=apart)
    base = torch.full((M + 1, -(-N // 8) * 8 + 8), 7.0, dtype=dtype, device="cuda")
    fp4.matmul(a, b, out=base[:M, :N])
    assert torch.equal(base[:M, :N], apart)
    assert bool((base[:M, N:] == 7.0).all()) and bool((base[M] == 7.0).all())


# every form of the product: tile widths, several tiles of a pair one after the other, splits of k


def values_of(p):
    """float64 values of a packed operand on its device, from its bytes."""
    code = p.codes.view(p.rows, -1)
    code = torch.stack((code & 15, code >> 4), 2).reshape(p.rows, -1)[:, :p.cols].long()
    value = torch.from_numpy(np.concatenate([ref.LEVELS, -ref.LEVELS])).cuda()[code]
    block = ref.BLOCK[p.fmt]
    nb = -(-p.cols // block)
    tk = -(-nb // 4)
    r, k = torch.arange(p.rows, device="cuda")[:, None], torch.arange(nb, device="cuda")[None]
    byte = p.scales[((r // 128) * tk + k // 4) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + k % 4].long()
    table = 2.0 ** (np.arange(256.0) - 127) if p.fmt == "mx" else np.concatenate([ref.E4M3, np.full(129, np.nan)])
    scale = torch.from_numpy(table).cuda()[byte]
    if p.fmt == "nv":
        scale = scale * p.tensor_scale[0].double()
    return value * scale.repeat_interleave(block, 1)[:, :p.cols]


# M, N, K, row stride of out; CTAs of a tile, rows, splits, by asynchronous copies, rounds (at least)
FORMS = [(2048, 2056, 700, 2056, 2, 128, 1, True, 2), (2050, 2064, 700, 2072, 2, 128, 1, True, 3), (2050, 2057, 700, 2064, 2, 128, 1, False, 3), (2050, 2057, 700, 2057, 2, 128, 1, False, 3),
         (129, 15000, 2600, 15000, 2, 128, 1, True, 2), (20000, 40, 2600, 41, 2, 128, 1, False, 3),
         (4100, 4104, 300, 4104, 2, 256, 1, True, 4), (4100, 4104, 300, 4112, 2, 256, 1, True, 4), (4100, 4101, 300, 4104, 2, 256, 1, False, 4), (4100, 4101, 300, 4101, 2, 256, 1, False, 4),
         (4096, 4096, 520, 4096, 2, 256, 1, True, 4), (129, 30000, 5000, 30000, 2, 256, 1, True, 2), (193, 30000, 5000, 30001, 2, 256, 1, False, 2),
         (20000, 136, 64, 144, 2, 64, 1, True, 4), (20000, 40, 2600, 40, 2, 64, 1, True, 2), (129, 20000, 2600, 20001, 2, 64, 1, False, 4),
         (16, 5003, 4096, 5003, 1, 16, 2, False, 1), (16, 2000, 3200, 2000, 1, 16, 4, False, 1), (3, 1000, 4096, 1000, 1, 16, 8, False, 1),
         (30, 5003, 4096, 5003, 1, 32, 2, False, 1), (60, 2000, 3200, 2003, 1, 64, 4, False, 1), (120, 1400, 5000, 1400, 1, 128, 8, False, 1),
         (128, 3000, 3300, 3000, 1, 128, 4, False, 1), (150, 300, 8192, 300, 1, 128, 8, False, 1), (300, 600, 8192, 601, 1, 128, 4, False, 1),
         (64, 5003, 700, 5003, 1, 64, 1, False, 1)]


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("M,N,K,ldo,ctas,rows,splits,wide,rounds", FORMS)
def test_product_of_every_form(fp4, B, M, N, K, ldo, ctas, rows, splits, wide, rounds, fmt):
    a = fp4.quantise(randn(M, K, seed=M + K) * torch.exp(randn(M, 1, seed=1)), fmt)
    b = fp4.quantise(randn(N, K, seed=N * 3 + K, scale=0.02, dtype=BF16), fmt)
    va, vb = values_of(a), values_of(b)
    want, total = va @ vb.t(), va.abs() @ vb.abs().t()
    for dtype in (F32, BF16, F16):
        form = B.fp4_matmul_form(M, N, K, dtype, ldo, torch.cuda.get_device_properties(0).multi_processor_count)
        # 4-byte elements keep rows of 16 bytes at strides where 2-byte ones do not: the sizes are chosen for both alike
        assert form[:4] == (ctas, rows, splits, wide) and form.rounds >= rounds, form
        base = torch.full((M, ldo), 7.0, dtype=dtype, device="cuda")
        out = base[:, :N]
        fp4.matmul(a, b, out=out)
        # any order of K additions with one ulp (2^-23) of a partial sum lost in each, then the type's rounding
        tol = K * 2.0 ** -23 * total + torch.finfo(dtype).eps / 2 * want.abs() + (2.0 ** -25 if dtype == F16 else 0.0)
        assert bool(((out.double() - want).abs() <= tol).all())
        assert bool((base[:, N:] == 7.0).all())
        again = torch.empty_like(base)[:, :N]
        fp4.matmul(a, b, out=again)
        assert torch.equal(out, again)
    fp4.check()
