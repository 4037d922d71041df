"""The loss over a large vocabulary and orthogonalised updates on a GPU: long sums, gradients of any size, boxes that are used again, other layouts."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import loss_orthogonal_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def device():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    yield torch.device("cuda", torch.cuda.current_device())
    from paper_1802_04434_b200 import waits
    waits.check()


@pytest.fixture(scope="module")
def loss():
    from paper_1802_04434_b200 import loss
    return loss


@pytest.fixture(scope="module")
def orthogonal():
    from paper_1802_04434_b200 import orthogonal
    return orthogonal


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


# ---------------------------------------------------------------------------------------------------------------------
# orthogonalised updates


@pytest.mark.parametrize("n,rows,cols", [(1, 2500, 1100), (1, 1100, 2500), (6, 1030, 1024), (3, 700, 700), (4, 300, 200)])
def test_boxes_that_are_used_again(orthogonal, n, rows, cols):
    # Behind the last step a warp writes its box as fp32 and the next elements of X are then copied into it: in products of one and of three
    # terms (two boxes in turn, and one), in tiles of every width and in clusters, to each type and into the parameters.  The error of a result is
    # below 2^-18 of its norm (three terms) or 4e-3, that is 2^-13 or 2^-3 for norms up to 34, were all of it in one element; it is spread over
    # all of them, and each is held to 2^-10 and 2^-4.  Bytes of one use read as the other's are off by any number up to 2^13.
    u = torch.randn(n, rows, cols, generator=gen(rows), device="cuda")
    want = ref.orthogonal(u)
    for products, most in ((3, 2.0 ** -10), (1, 2.0 ** -4)):
        for dtype in (F32, BF16, F16):
            first = orthogonal.orthogonalise(u, dtype=dtype, products=products)
            assert float((first.double() - want).abs().max()) <= most + 1.2 * ref.HALF_STEP[dtype]
            for _ in range(3):
                assert torch.equal(orthogonal.orthogonalise(u, dtype=dtype, products=products), first)
        moved = []
        for _ in range(2):
            x, m = torch.zeros_like(u), torch.zeros_like(u)
            orthogonal.momentum_step(x, u, m, 0.0, -1.0, products=products)
            moved.append(x)
        assert torch.equal(*moved) and float((moved[0].double() - want).abs().max()) <= most


def test_batches_of_empty_matrices(orthogonal):
    for shape in ((2, 3, 0, 5), (2, 3, 4, 0), (2, 0, 4, 5), (2, 3, 1, 0, 5)):
        x = torch.zeros(shape, device="cuda")
        assert orthogonal.orthogonalise(x).shape == shape and orthogonal.orthogonalise(x, out=torch.zeros_like(x)).shape == shape
        orthogonal.momentum_step(x, x.clone(), x.clone(), 0.9, 0.1)


@pytest.mark.parametrize("n,rows,cols,gap", [(3, 40, 33, 0), (2, 100, 128, 3), (3, 200, 140, 1), (2, 700, 500, 4)])
def test_matrices_whose_rows_lie_in_turn(orthogonal, n, rows, cols, gap):
    # one row of each matrix behind the other, as where several weights are one: in place, and as the parameters and momenta of a step
    def in_turn(t):
        big = torch.full((rows, n * (cols + gap)), 7.0, device="cuda")
        view = big.as_strided((n, rows, cols), (cols + gap, n * (cols + gap), 1))
        view.copy_(t)
        return big, view
    u, x0 = (torch.randn(n, rows, cols, generator=gen(rows + i), device="cuda") for i in (0, 1))
    want = orthogonal.orthogonalise(u)
    big, view = in_turn(u)
    assert orthogonal.orthogonalise(view, out=view).data_ptr() == view.data_ptr() and torch.equal(view, want)
    (_, x), (_, m) = in_turn(x0), in_turn(u)
    xs, ms = x0.clone(), u.clone()
    for a, b in ((x, m), (xs, ms)):
        orthogonal.momentum_step(a, u, b, 0.9, 0.1)
    assert torch.equal(x, xs) and torch.equal(m, ms)
    for b, v in ((big, view), (x._base, x), (m._base, m)):
        v.fill_(7.0)
        assert bool((b == 7.0).all())


def test_results_that_autograd_would_differentiate(orthogonal):
    for shape in ((20, 30), (2, 3, 200, 140), (4, 0, 5)):
        u = torch.randn(shape, generator=gen(1), device="cuda").requires_grad_()
        got = orthogonal.orthogonalise(u)
        assert torch.equal(got, orthogonal.orthogonalise(u.detach()))
        got.mul_(0.1)
        with pytest.raises(RuntimeError, match="no derivative"):
            (got.sum() + u.sum()).backward()
        x, m = u.detach().clone().requires_grad_(), torch.zeros(shape, device="cuda")
        orthogonal.momentum_step(x, torch.ones(shape, device="cuda"), m, 0.9, 0.1)
        assert x.is_leaf


# ---------------------------------------------------------------------------------------------------------------------
# the loss's gradients


def gradients(h, w, y, g, part=16384):
    """dh and dw (as if in fp32) of sum_t g_t losses_t without ignored tokens, and bounds that take sums as sums of parts, all in float64.

    A logit is off by (32 + D / 256) 2^-23 S, S = sum |h_d w_d|, a loss by 2^-19 (1 + lse) beside, forward and backward: dz by the two, and
    by 2^-38 of the largest g where fp16 ends.  Entries of dz are rounded to 16 bits, each to either side: sums of those errors are held to six standard
    deviations, half a step / sqrt(3) each.  Targets' entries lie close to the largest, which is kept, and are off by no more than they
    differ from it.  A sum's parts are 2048 long: 128 steps of 2 * 2^-23 of a part each, and 2^-23 of the sum for each of the parts."""
    T, D = h.shape
    V = w.shape[0]
    hd, half = h.double(), ref.HALF_STEP[h.dtype]
    z = torch.cat([hd @ p.double().t() for p in w.split(part)], 1)
    S = torch.stack([(hd.abs() @ p.double().abs().t()).amax(1) for p in w.split(part)]).amax(0)
    lse = torch.logsumexp(z, 1)
    gd, at = g.double()[:, None], (torch.arange(T, device=h.device), y)
    dz = z.sub_(lse[:, None]).exp_()
    z_tol = (2 * (32 + D / 256) * 2.0 ** -23 * S + 2.0 ** -19 * (1 + lse.abs()))[:, None]
    tol = gd.abs() * dz * z_tol + gd.abs().max() * 2.0 ** -38
    dz[at] -= 1
    dz *= gd
    target = dz[at].abs() / dz[at].abs().max()
    tol[at] += torch.minimum(half * target, 1 - target) * dz[at].abs().max() + 2.0 ** -22 * dz[at].abs()
    spread = (half * dz).square_() / 3
    spread[at] = 0

    def product(rows, k):
        """f(dz or what is like it, by columns of the vocabulary): rows that it is multiplied by."""
        value, loose, chance, size = (rows(t, f) for t, f in ((dz, lambda b: b), (tol, torch.abs), (spread, torch.square), (dz.abs(), torch.abs)))
        return value, loose + 6 * chance.sqrt() + (2 * 128 + k / 2048 + 2) * 2.0 ** -23 * size
    dh, dh_tol = product(lambda t, f: sum(t[:, i:i + part] @ f(w[i:i + part].double()) for i in range(0, V, part)), V)
    dw, dw_tol = product(lambda t, f: t.t() @ f(hd), T)
    return dh, dh_tol + half * dh.abs() + ref.SMALLEST[h.dtype], dw, dw_tol + 2.0 ** -24 * dw.abs()


def long_problem(T, V, D, dtype, deviation, mean, words):
    """Rows with a part that all of them share, several times their own, so that sums grow with every term: logits of `mean` and their `deviation`."""
    r = gen(T + V + D)
    def randn(*s):
        return torch.randn(*s, generator=r, device="cuda")
    shared = randn(D)
    w = randn(V, D).add_(4 * shared)
    h = randn(T, D)
    if mean:
        h += shared
        w -= w.mean(0) - 4 * shared
        h *= mean / (h @ w.mean(0))[:, None]
        w -= 4 * shared
        w *= deviation / float((h[:8] @ w.t()).std(1).mean())
        w += 4 * shared
    else:
        h -= h @ shared[:, None] * shared / shared.square().sum()
        h *= deviation / float((h[:8] @ w.t()).std(1).mean())
    y = torch.randint(0, words, (T,), generator=r, device="cuda")
    return h.to(dtype), w.to(dtype), y


def within(got, want, tol, what):
    got = got.double()
    assert torch.isfinite(got).all(), what
    off = (got - want).abs()
    assert bool((off <= tol).all()), "%s: %g of its bound, off by %g of %g" % (what, (off / tol).nan_to_num().max(), off.max(), want.abs().max())


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("T,V,D", [(700, 131072, 6000), (64, 200000, 256)])
def test_gradients_over_a_long_vocabulary(loss, T, V, D, dtype):
    # dh's sum is V long, in one accumulator where there are enough tiles (the first), with planes of their own where not
    h, w, y = long_problem(T, V, D, dtype, 0.05, 0, V)
    _, kept = loss.cross_entropy_forward(h, w, y)
    g = torch.ones(T, device="cuda")
    dh, dw = loss.cross_entropy_backward(kept, g, dw_dtype=F32)
    want, tol, dw_want, dw_tol = gradients(h, w, y, g)
    within(dh, want, tol, "dh")
    within(dw, dw_want, dw_tol, "dw")


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_weight_gradient_of_many_tokens(loss, dtype):
    # dw's sum is T long: words that are no token's target have terms of one sign
    w, h, _ = long_problem(2304, 65536, 2048, dtype, 0.1, 0, 10)
    y = torch.randint(0, 10, (65536,), generator=gen(3), device="cuda")
    _, kept = loss.cross_entropy_forward(h, w, y)
    g = torch.ones(65536, device="cuda")
    dh, dw = loss.cross_entropy_backward(kept, g, dw_dtype=F32)
    want, tol, dw_want, dw_tol = gradients(h, w, y, g)
    within(dw, dw_want, dw_tol, "dw")
    within(dh, want, tol, "dh")


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("T", [3, 300])
def test_large_logits_over_a_long_width(loss, T, dtype):
    # The backward pass makes its logits once more: what they are off from the forward pass's is a factor of the probabilities, and a row of dz
    # does not sum to zero.  That sum is dh where w has a column of ones (and h of zeros); one token counts, whose target's entry is the scale of dz
    # and is kept.  In it: the logits', twice, as in `gradients`; roundings of dz; the product's parts; the target's p, 2^-22.
    V, D = 2000, 16384
    h, w, y = long_problem(T, V, D, dtype, 0.3, 40.0, V)
    h[:, -1], w[:, -1] = 0, 1
    t = T // 2
    y[torch.arange(T, device="cuda") != t] = -100
    _, kept = loss.cross_entropy_forward(h, w, y)
    g = torch.ones(T, device="cuda")
    dh, dw = loss.cross_entropy_backward(kept, g, dw_dtype=F32)
    z = h[t].double() @ w.double().t()
    S = float((h[t].double().abs() @ w.double().abs().t()).max())
    p = torch.softmax(z, 0)
    tol = 2 * (32 + D / 256) * 2.0 ** -23 * S + 2.0 ** -19 * (1 + float(torch.logsumexp(z, 0))) + 6 * ref.HALF_STEP[dtype] * float(p.square().sum().sqrt()) / 3 ** 0.5 \
        + 2 * (2 * 128 + 3) * 2.0 ** -23 + 2.0 ** -22
    assert abs(float(dh[t, -1])) <= tol, (float(dh[t, -1]), tol)
    want, dh_tol, dw_want, dw_tol = gradients(h[t:t + 1], w, y[t:t + 1], g[:1])
    within(dw, dw_want, dw_tol, "dw")
    within(dh[t:t + 1], want, dh_tol, "dh")
    others = torch.arange(T, device="cuda") != t
    assert not dh[others].any()


def problem(T, V, D, dtype, seed=0):
    r = gen(seed * 7919 + T + 31 * V + 1009 * D)
    w = torch.randn(V, D, generator=r, device="cuda").mul_(1.5 / D ** 0.5)
    y = torch.randint(0, V, (T,), generator=r, device="cuda")
    h = torch.randn(T, D, generator=r, device="cuda")
    g = (torch.rand(T, generator=r, device="cuda") - 0.3) / T
    return h.to(dtype), w.to(dtype), y, g


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("scale", [3e-30, 1e-29, 1.5e38, 3e38])
def test_gradients_at_the_ends_of_fp32(loss, dtype, scale):
    # dz is scaled by a power of two there, 2^114 or 2^-114: fp16 keeps it to 2^-25 of what that is the inverse of
    h, w, y, g = problem(50, 60, 64, dtype)
    _, kept = loss.cross_entropy_forward(h, w, y)
    _, dw = loss.cross_entropy_backward(kept, g * scale, dw_dtype=F32)
    want, tol = ref.loss_and_gradients(h, w, y, g)
    kept_to = 2.0 ** -25 * (2.0 ** -114 if scale < 1 else 2.0 ** 114) / scale
    within(dw.double() / scale, want[2], tol[2] + 2.0 ** -23 * want[2].abs() + kept_to * h.double().abs().sum(0), "dw")


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_a_gradient_that_is_not_finite_leaves_the_other_rows(loss, dtype, value):
    # gradients of a mean over many tokens: in fp16 what is not scaled vanishes
    h, w, y, _ = problem(40, 5000, 64, dtype)
    g = torch.full((40,), 1.0 / 8192, device="cuda")
    want, tol = ref.loss_and_gradients(h, w, y, g)
    g[7] = value
    _, kept = loss.cross_entropy_forward(h, w, y)
    dh, dw = loss.cross_entropy_backward(kept, g)
    rest = torch.arange(40, device="cuda") != 7
    within(dh[rest], want[1][rest], tol[1][rest], "dh")
    assert not torch.isfinite(dh[7]).all() and not torch.isfinite(dw).all()
    # nothing but such gradients
    dh, dw = loss.cross_entropy_backward(kept, torch.full_like(g, value))
    assert not torch.isfinite(dh).any()


@pytest.mark.parametrize("T", [3, 300])
def test_every_row_of_a_weight_beyond_32_bits(loss, T):
    # 4.3e9 bytes of w and 8.6e9 of dw, each block of rows another one, targets all over the vocabulary: a share of it that is lost, repeated or
    # another's shows in dh and in that block of dw.  In norm: roundings to bf16 of dz and of dh, 2^-8 each at most; logits as in `gradients`, that is
    # 1e-3 for sums of magnitudes near 55.
    V, D, part = 262_657, 8192, 16384
    h = torch.randn(T, D, generator=gen(T), device="cuda").to(BF16)
    w = torch.empty(V, D, dtype=BF16, device="cuda")
    for i, block in enumerate(w.split(part)):
        block.copy_(torch.randn(block.shape, generator=gen(1000 + i), device="cuda").mul_(0.01))
    y = torch.randint(0, V, (T,), generator=gen(5), device="cuda")
    y[0], y[1], y[2] = V - 1, 0, V // 2
    losses, kept = loss.cross_entropy_forward(h, w, y)
    dh, dw = loss.cross_entropy_backward(kept, torch.ones(T, device="cuda"), dw_dtype=F32)
    z = torch.cat([h.double() @ block.double().t() for block in w.split(part)], 1)
    lse = torch.logsumexp(z, 1)
    at = torch.arange(T, device="cuda"), y
    want = lse - z[at]
    assert float((losses.double() - want).abs().max()) < 1e-3
    dz = z.sub_(lse[:, None]).exp_()
    dz[at] -= 1
    assert ref.off(dh, sum(dz[:, i:i + part] @ w[i:i + part].double() for i in range(0, V, part))) < 2.0 ** -7 + 1e-3
    for i in range(0, V, part):
        assert ref.off(dw[i:i + part], dz[:, i:i + part].t() @ h.double()) < 2.0 ** -8 + 1e-3, i
