"""The loss over a large vocabulary and orthogonalised updates on a GPU, against plain forms in 64 bits."""
import ctypes
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


def problem(T, V, D, dtype, ignored=0.2, seed=0):
    r = gen(seed * 7919 + T + 31 * V + 1009 * D)
    w = torch.randn(V, D, generator=r, device="cuda").mul_(1.5 / D ** 0.5)
    y = torch.randint(0, V, (T,), generator=r, device="cuda")
    h = torch.randn(T, D, generator=r, device="cuda")
    h += 5 * torch.rand(T, 1, generator=r, device="cuda") * w[y]          # some tokens sure of their target
    y = torch.where(torch.rand(T, generator=r, device="cuda") < ignored, -100, y)
    g = (torch.rand(T, generator=r, device="cuda") - 0.3) / T
    return h.to(dtype), w.to(dtype), y, g


def within(got, want, tol, what):
    got = got.double()
    assert torch.isfinite(got).all(), what
    worst = ((got - want).abs() - tol).max()
    assert worst <= 0, "%s: %g beyond its bound, off by %g of %g" % (what, worst, (got - want).abs().max(), want.abs().max())


def check_loss(loss, h, w, y, g, ignore=-100, **how):
    losses, kept = loss.cross_entropy_forward(h, w, y, ignore_index=ignore)
    dh, dw = loss.cross_entropy_backward(kept, g, **how)
    assert losses.dtype == F32 and dh.dtype == h.dtype and dh.shape == h.shape and dw.shape == w.shape
    want, tol = ref.loss_and_gradients(h, w, y, g, ignore)
    for name, a, b, t in zip(("losses", "dh", "dw"), (losses, dh, dw), want, tol):
        within(a, b, t, name)
    return losses, dh, dw


# one token and few (a kernel of their own), one word, one column; sides about the tiles' (64, 128, 256) and stages' (16, 64, 256); few tiles and a long
# width, or a long vocabulary (k split by a cluster, or into planes); many tiles
SIZES = [(1, 1, 1), (1, 2, 8), (2, 33, 7), (3, 5, 300), (1, 300, 264), (2, 1000, 1031), (4, 100, 17), (5, 64, 64), (17, 65, 72), (63, 127, 15), (64, 128, 16),
         (65, 129, 80), (127, 257, 63), (129, 255, 129), (200, 513, 1032), (256, 256, 256), (300, 700, 2056), (8, 5000, 520), (40, 9001, 96), (777, 1111, 333),
         (1000, 3001, 128), (2049, 2100, 64), (1500, 4099, 1111)]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("T,V,D", SIZES)
def test_loss_and_gradients(loss, T, V, D, dtype):
    check_loss(loss, *problem(T, V, D, dtype))


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_vocabulary_in_pieces(loss, dtype):
    # dz of a piece holds at most 2^27 numbers: two pieces, the second of 20 columns; dh is added up in fp32
    h, w, y, g = problem(70_000, 1812, 24, dtype, ignored=0.1)
    check_loss(loss, h, w, y, g)


def test_rows_beyond_32_bits(loss):
    # 4.4e9 bytes of w, more than 2^31 elements
    V, D = 262_657, 8192
    h, _, y, g = problem(3, 1000, D, BF16, ignored=0.0)
    w = torch.empty(V, D, dtype=BF16, device="cuda")
    for part in w.split(16384):
        part.copy_(torch.randn(part.shape, generator=gen(part.shape[0]), device="cuda").mul_(0.01))
    y = torch.tensor([V - 1, 0, V // 2], device="cuda")
    losses, kept = loss.cross_entropy_forward(h, w, y)
    dh, dw = loss.cross_entropy_backward(kept, g)
    z = torch.cat([h.double() @ part.double().t() for part in w.split(16384)], 1)
    lse = torch.logsumexp(z, 1)
    want = lse - z.gather(1, y[:, None])[:, 0]
    S = 0.05 * h.double().abs().sum(1)                       # |w| is below that
    assert ((losses.double() - want).abs() <= 2 * 64 * 2.0 ** -23 * S + 2.0 ** -19 * (1 + lse)).all()
    dz = (z - lse[:, None]).exp()
    dz[torch.arange(3), y] -= 1
    dz *= g.double()[:, None]
    tail = dz[:, -5000:].t() @ h.double()
    assert ref.off(dw[-5000:], tail) < 2.0 ** -7             # a rounding of dz and one of dw, 2^-8 each at most
    within(dh, sum(dz[:, i:i + 16384] @ w[i:i + 16384].double() for i in range(0, V, 16384)), 2.0 ** -7 * (dz.abs().amax(1, keepdim=True) * 0.05) +
           2.0 ** -6 * g.double().abs()[:, None] * 0.05, "dh")


@pytest.mark.parametrize("T", [1, 2, 3, 100])
def test_strides_and_places(loss, T):
    h, w, y, g = problem(T, 300, 96, BF16)
    plain = check_loss(loss, h, w, y, g)

    def wide(t, off_, pad, rows=1):                          # t inside a larger matrix, NaN all around
        big = torch.full((t.shape[0] * rows, off_ + t.shape[1] + pad), float("nan"), dtype=t.dtype, device="cuda")
        view = big[::rows, off_:off_ + t.shape[1]]
        view.copy_(t)
        return view
    for off_, pad, rows in ((0, 8, 1), (8, 16, 1), (1, 3, 1), (0, 1, 1), (4, 4, 1), (0, 0, 2), (3, 8, 3)):
        for got, want in zip(check_loss(loss, wide(h, off_, pad, rows), wide(w, off_, pad, rows), y, g), plain):
            assert torch.equal(got, want)                    # the same numbers in the same order
    yy = torch.stack([y, y + 1], 1)[:, 0]                    # every second one
    gg = torch.stack([g, g], 1)[:, 1]
    for got, want in zip(check_loss(loss, h.t().contiguous().t(), w.t().contiguous().t(), yy, gg), plain):
        assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("out", [F32, BF16, F16])
def test_weight_gradient_into_place(loss, dtype, out):
    for V, D, ld, at in ((300, 72, 80, 0), (129, 33, 47, 1), (64, 128, 128, 0)):
        h, w, y, g = problem(150, V, D, dtype)
        losses, kept = loss.cross_entropy_forward(h, w, y)
        big = torch.full((V + 1, ld), 7.0, dtype=out, device="cuda")
        dw = big[:V, at:at + D]
        dh, got = loss.cross_entropy_backward(kept, g, dw=dw)
        assert got.data_ptr() == dw.data_ptr()
        want, tol = ref.loss_and_gradients(h, w, y, g)
        extra = ref.HALF_STEP[out] * want[2].abs() + ref.SMALLEST[out]
        within(dw, want[2], tol[2] + extra, "dw")
        big[:V, at:at + D] = 7.0
        assert bool((big == 7.0).all())                      # what lies around is as it was
        _, alone = loss.cross_entropy_backward(kept, g, dw_dtype=out, want_h=False)
        assert alone.dtype == out and _ is None
        within(alone, want[2], tol[2] + extra, "dw alone")
        only_h, none = loss.cross_entropy_backward(kept, g, want_w=False)
        assert none is None and torch.equal(only_h, dh)


def test_no_tokens(loss):
    h, w = torch.zeros(0, 16, dtype=BF16, device="cuda"), torch.zeros(10, 16, dtype=BF16, device="cuda")
    losses, kept = loss.cross_entropy_forward(h, w, torch.zeros(0, dtype=torch.int64, device="cuda"))
    dw = torch.ones(10, 16, device="cuda")
    dh, got = loss.cross_entropy_backward(kept, torch.zeros(0, device="cuda"), dw=dw)
    assert losses.shape == (0,) and dh.shape == (0, 16) and bool((dw == 0).all())


@pytest.mark.parametrize("T", [1, 2, 70, 600])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_ignored_tokens_have_no_part(loss, T, dtype):
    h, w, y, g = problem(T, 200, 80, dtype, ignored=0.4, seed=3)
    y[0] = -100
    losses, dh, dw = check_loss(loss, h, w, y, g)
    gone = y == -100
    assert bool((losses[gone] == 0).all()) and bool((dh[gone] == 0).all())
    broken, gb = h.clone(), g.clone()
    for i, value in enumerate((float("nan"), float("inf"), -float("inf"), torch.finfo(dtype).max, torch.finfo(dtype).min)):
        broken[gone, i::5] = value
    gb[gone] = float("nan")
    if T > 1:                                                # one row alone that is not finite, the others ignored and finite
        for rows in (gone, torch.arange(T, device="cuda") == 0):
            some = torch.where(rows[:, None], broken, h)
            for got, want in zip(check_loss(loss, some, w, y, gb), (losses, dh, dw)):
                assert torch.equal(got, want)
    # all of them ignored
    l, d, e = check_loss(loss, broken, w, torch.full_like(y, -100), gb)
    assert not l.any() and not d.any() and not e.any()
    # a number of the vocabulary may be the one that is ignored
    y7 = torch.where(gone, 7, torch.where(y == 7, 8, y))
    for got, want in zip(check_loss(loss, broken, w, y7, gb, ignore=7), check_loss(loss, h, w, torch.where(gone, -100, y7), g)):
        assert torch.equal(got, want)


def test_targets_outside_the_vocabulary(loss):
    h, w, y, g = problem(40, 100, 64, BF16, ignored=0.0)
    good, kept = loss.cross_entropy_forward(h, w, y)
    for bad in (100, -1, -99, 1 << 40, -(1 << 40)):
        y2 = y.clone()
        y2[3] = bad
        losses, kept = loss.cross_entropy_forward(h, w, y2)
        assert bool(losses[3].isnan()) and torch.equal(torch.cat([losses[:3], losses[4:]]), torch.cat([good[:3], good[4:]]))
        dh, dw = loss.cross_entropy_backward(kept, g)
        assert bool(dh[3].isnan().all()) and bool(torch.isfinite(dh[:3]).all()) and bool(dw.isnan().all())


def test_extreme_logits(loss):
    h, w, y, g = problem(30, 90, 64, BF16, ignored=0.0)
    h = h.abs()
    w[5] = -float("inf")                                     # a word that is masked: logit -inf
    w[40:72] = -float("inf")                                 # and a whole column of a tile
    y = torch.where((y == 5) | ((y >= 40) & (y < 72)), 3, y)
    h[h == 0] = 1
    losses, kept = loss.cross_entropy_forward(h, w, y)
    keep = torch.tensor([i for i in range(90) if i != 5 and not 40 <= i < 72], device="cuda")
    want, tol = ref.loss_and_gradients(h, w[keep], (keep[None, :] == y[:, None]).int().argmax(1), g)
    within(losses, want[0], tol[0] + 2.0 ** -19, "losses")
    few, _ = loss.cross_entropy_forward(h[:1], w, y[:1])
    within(few, want[0][:1], tol[0][:1] + 2.0 ** -19, "one token's loss")
    # logits that differ by hundreds: the target's probability is 0 or 1
    h, w, y, g = problem(64, 70, 128, F16, ignored=0.0)
    check_loss(loss, h * 20, w * 2, y, g)
    w[9, 9] = float("nan")
    losses, _ = loss.cross_entropy_forward(h, w, y)
    assert bool(losses.isnan().all())


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("T", [1, 2, 6, 200])
def test_tokens_that_are_sure(loss, T, dtype):
    # 1 - p between 1e-3 and 1e-6: the loss and the target's entry of dz are that small, and still themselves
    r = gen(T)
    w = torch.randn(120, 256, generator=r, device="cuda").mul_(0.02)
    y = torch.randint(0, 120, (T,), generator=r, device="cuda")
    h = (14 + 4 * torch.rand(T, 1, generator=r, device="cuda")) * w[y] / w[y].square().sum(1, keepdim=True) + torch.randn(T, 256, generator=r, device="cuda") * 0.1
    h, w = h.to(dtype), w.to(dtype)
    one = torch.ones(T, device="cuda")
    losses, kept = loss.cross_entropy_forward(h, w, y)
    dh, dw = loss.cross_entropy_backward(kept, one, dw_dtype=F32)
    z = h.double() @ w.double().t()
    p = torch.softmax(z, 1)
    p[torch.arange(T), y] = 0
    miss = p.sum(1)
    assert float(miss.max()) < 1e-3
    # sums of exponentials are 1 and a little: 2^-24 of them for each of up to 120 terms is 120 * 2^-24 / miss of the little, at the worst; logits as in the bounds of ref
    S = (h.double().abs() @ w.double().abs().t()).amax(1)
    error = 32 * 2.0 ** -23 + 4 * (2 * 256 / 16 + 34) * 2.0 ** -23 * S + 2.0 ** -19
    assert ((losses.double() + torch.log1p(-miss)).abs() <= error * miss + 120 * 2.0 ** -24).all()
    p[torch.arange(T), y] = -miss
    part = (error * miss + 120 * 2.0 ** -24)[:, None] + 0 * p
    within(dw, p.t() @ h.double(), (part + ref.HALF_STEP[dtype] * p.abs() + 2.0 ** -38).t() @ h.double().abs() * 1.01, "dw")
    if dtype == BF16:
        dz_tol = torch.where(p < 0, part, error[:, None] * p) + 2.0 ** -8 * p.abs()
        within(dh, p @ w.double(), dz_tol @ w.double().abs() * 1.01 + 2.0 ** -8 * (p @ w.double()).abs() + 2.0 ** -130, "dh")


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_a_sure_token_of_large_gradient_beside_others(loss, dtype):
    # the sure token's loss is 0 or next to it, so its entry says nothing of how large the others of its row are
    T, V, D = 6, 300, 256
    h, w, y, _ = problem(T, V, D, dtype)
    h[0] = w[y[0]] * (17 / w[y[0]].double().square().sum()).to(dtype)
    g = torch.full((T,), 1e-6, device="cuda")
    g[0] = 1.0
    losses, kept = loss.cross_entropy_forward(h, w, y)
    dh, dw = loss.cross_entropy_backward(kept, g, dw_dtype=F32)
    want, tol = ref.loss_and_gradients(h, w, y, g)
    within(dh, want[1], tol[1], "dh")
    within(dw, want[2], tol[2], "dw")


def test_a_row_that_is_not_a_number_leaves_the_others(loss):
    h, w, y, g = problem(9, 300, 64, F16)
    _, kept = loss.cross_entropy_forward(h, w, y)
    before = loss.cross_entropy_backward(kept, g)[0]
    bad = h.clone()
    bad[4, 3] = float("nan")
    g[4] = 1e-3 * g[4]
    _, kept = loss.cross_entropy_forward(bad, w, y)
    dh, _ = loss.cross_entropy_backward(kept, g)
    rest = [t for t in range(9) if t != 4]
    assert dh[4].isnan().all() and not dh[rest].isnan().any()
    want, tol = ref.loss_and_gradients(h, w, y, g)
    within(dh[rest], want[1][rest], tol[1][rest], "dh")
    within(before[rest], want[1][rest], tol[1][rest], "before")


@pytest.mark.parametrize("scale", [1e-30, 1e-8, 1.0, 1e4, 1e30])
def test_gradients_of_any_size_scale_fp16(loss, scale):
    # dz in fp16 is scaled to its largest entry; what comes out overflows or vanishes only where the result does
    h, w, y, g = problem(50, 60, 64, F16)
    losses, kept = loss.cross_entropy_forward(h, w, y)
    _, dw = loss.cross_entropy_backward(kept, g * scale, dw_dtype=F32)
    want, tol = ref.loss_and_gradients(h, w, y, g)
    within(dw.double() / scale, want[2], tol[2] + 2.0 ** -23 * want[2].abs(), "dw")
    g0 = torch.zeros_like(g)
    dh, dw = loss.cross_entropy_backward(kept, g0)
    assert not dh.any() and not dw.any()


def test_one_gradient_for_all(loss):
    h, w, y, g = problem(80, 60, 64, F16)
    losses, kept = loss.cross_entropy_forward(h, w, y)
    one = torch.full((1,), 0.0125, device="cuda").expand(80)
    for a, b in zip(loss.cross_entropy_backward(kept, one), loss.cross_entropy_backward(kept, one.contiguous())):
        assert torch.equal(a, b)
    bad = g.clone()
    bad[int((y != -100).nonzero()[0])] = float("inf")
    assert not torch.isfinite(loss.cross_entropy_backward(kept, bad)[1]).all()


def test_autograd(loss):
    h, w, y, g = problem(60, 50, 32, BF16, ignored=0.3)
    for reduction in ("mean", "sum", "none"):
        hp, wp = h.view(3, 20, 32).clone().requires_grad_(), w.clone().requires_grad_()
        out = loss.cross_entropy(hp, wp, y.view(3, 20), reduction=reduction)
        weight = torch.ones_like(out) if reduction != "none" else g.view(3, 20)
        out.backward(weight)
        n = int((y != -100).sum())
        gt = {"mean": torch.full((60,), 1.0 / n, device="cuda"), "sum": torch.ones(60, device="cuda"), "none": g}[reduction]
        want, tol = ref.loss_and_gradients(h, w, y, gt)
        within(hp.grad.view(60, 32), want[1], tol[1], "dh")
        within(wp.grad, want[2], tol[2], "dw")
        total = {"mean": want[0].sum() / n, "sum": want[0].sum(), "none": want[0].view(3, 20)}[reduction]
        assert out.shape == total.shape and torch.allclose(out.double(), total, rtol=1e-5, atol=1e-5)
    # only what is wanted, and nothing kept where nothing can be
    for grads in ((True, False), (False, True)):
        hp, wp = h.clone().requires_grad_(grads[0]), w.clone().requires_grad_(grads[1])
        loss.cross_entropy(hp, wp, y).backward()
        assert (hp.grad is not None, wp.grad is not None) == grads
    with torch.no_grad():
        assert not loss.cross_entropy(h.clone().requires_grad_(), w, y).requires_grad
    # a mean over nothing is 0, with gradients of 0
    hp = h.clone().requires_grad_()
    out = loss.cross_entropy(hp, w, torch.full_like(y, -100))
    out.backward()
    assert float(out.detach()) == 0 and not hp.grad.any()
    # second derivatives are an error
    hp = h.clone().requires_grad_()
    d, = torch.autograd.grad(loss.cross_entropy(hp, w, y), hp, create_graph=True)
    with pytest.raises(RuntimeError, match="once only"):
        d.float().sum().backward()


def test_gradient_against_differences(loss):
    # values that bf16 holds, moved by steps that it holds: the loss's own differences
    r = gen(5)
    h = torch.randint(-4, 5, (6, 16), generator=r, device="cuda").to(BF16) / 4
    w = torch.randint(-4, 5, (20, 16), generator=r, device="cuda").to(BF16) / 4
    y = torch.randint(0, 20, (6,), generator=r, device="cuda")
    one = torch.ones(6, device="cuda")
    dh, dw = loss.cross_entropy_backward(loss.cross_entropy_forward(h, w, y)[1], one, dw_dtype=F32)
    step = 1 / 16
    for t, i in ((0, 0), (3, 7), (5, 15)):
        moved = [h.clone(), h.clone()]
        moved[0][t, i] += step
        moved[1][t, i] -= step
        diff = (loss.cross_entropy_forward(moved[0], w, y)[0].double() - loss.cross_entropy_forward(moved[1], w, y)[0].double())[t] / (2 * step)
        # third derivative of a loss in one h: below 2 max|w|^3 = 2; 2^-8 a rounding of dz and of dh, of sums of |w| <= 1
        assert abs(float(diff) - float(dh[t, i])) <= 2 * step ** 2 / 6 + 2 * 2 * 2.0 ** -8 + 1e-4
    for v, i in ((0, 3), (11, 0), (int(y[2]), 9)):
        moved = [w.clone(), w.clone()]
        moved[0][v, i] += step
        moved[1][v, i] -= step
        diff = (loss.cross_entropy_forward(h, moved[0], y)[0].double() - loss.cross_entropy_forward(h, moved[1], y)[0].double()).sum() / (2 * step)
        assert abs(float(diff) - float(dw[v, i])) <= 6 * (2 * step ** 2 / 6 + 2 * 2.0 ** -8) + 1e-4


def test_loss_repeats_its_bits(loss):
    for T, V, D in ((2, 3000, 512), (100, 3000, 512), (600, 5000, 640)):
        h, w, y, g = problem(T, V, D, BF16)
        first = check_loss(loss, h, w, y, g)
        for _ in range(3):
            for a, b in zip(check_loss(loss, h, w, y, g), first):
                assert torch.equal(a, b)


def capture(f):
    """f captured into a graph, its outputs there."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        f()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = f()
    return graph, out


def test_loss_in_graphs_and_on_streams(loss):
    h, w, y, g = problem(300, 2000, 256, F16)
    h2, _, y2, g2 = problem(300, 2000, 256, F16, seed=9)
    want, want2 = check_loss(loss, h, w, y, g), check_loss(loss, h2, w, y2, g2)
    hs, ys, gs = h.clone(), y.clone(), g.clone()

    def both():
        losses, kept = loss.cross_entropy_forward(hs, w, ys)
        return (losses, *loss.cross_entropy_backward(kept, gs))
    graph, out = capture(both)
    other, out2 = capture(both)                              # two graphs, each with workspaces of its own
    for a, b, c, expected in ((h, y, g, want), (h2, y2, g2, want2), (h, y, g, want)):
        hs.copy_(a), ys.copy_(b), gs.copy_(c)
        graph.replay()
        other.replay()
        torch.cuda.synchronize()
        for got, again, e in zip(out, out2, expected):
            assert torch.equal(got, e) and torch.equal(again, e)
    # two calls at a time
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    results = [[], []]
    for _ in range(4):
        for s, (a, b, c), r in zip(streams, ((h, y, g), (h2, y2, g2)), results):
            with torch.cuda.stream(s):
                losses, kept = loss.cross_entropy_forward(a, w, b)
                r.append((losses, *loss.cross_entropy_backward(kept, c)))
    torch.cuda.synchronize()
    for r, e in zip(results, (want, want2)):
        for got in r:
            assert all(torch.equal(a, b) for a, b in zip(got, e))


def test_backward_captured_beside_an_eager_graph(loss):
    # While an eager graph of them lives, leaves belong to the stream that it was made on, and torch refuses to capture gradients of theirs (for
    # its own operators too): the passes as functions, and leaves of the capture's own, go.
    h, w, y, g = problem(100, 300, 64, BF16)
    hp, wp = h.clone().requires_grad_(), w.clone().requires_grad_()
    eager = loss.cross_entropy(hp, wp, y, reduction="none")
    want = torch.autograd.grad(eager, (hp, wp), g, retain_graph=True)

    def functions():
        with torch.no_grad():
            return loss.cross_entropy_backward(loss.cross_entropy_forward(hp, wp, y)[1], g)

    def leaves():
        mine = hp.detach().requires_grad_(), wp.detach().requires_grad_()
        return torch.autograd.grad(loss.cross_entropy(*mine, y, reduction="none"), mine, g)
    for f in (functions, leaves):
        graph, out = capture(f)
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(eager, (hp, wp), g), want))


def test_waits_that_run_out(loss, orthogonal):
    from paper_1802_04434_b200 import binding as B
    h, w, y, g = problem(200, 200, 128, BF16, ignored=0.0)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    losses, lse, kinds = torch.zeros(200, device="cuda"), torch.zeros(400, device="cuda"), torch.zeros(200, dtype=torch.uint8, device="cuda")
    ws = torch.zeros(B.xent_sizes(200, 200, 128)[0], dtype=torch.uint8, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    assert B.lib().ssgd_xent_wait_selftest(h.data_ptr(), 128, w.data_ptr(), 128, 1, 200, 200, 128, y.data_ptr(), -100, losses.data_ptr(), lse.data_ptr(),
                                           kinds.data_ptr(), ws.data_ptr(), status.data_ptr(), stream) == 0
    torch.cuda.synchronize()
    assert int(status) == 1
    check_loss(loss, h, w, y, g)
    f = (ctypes.c_float * 3)(*ref.MUON)
    for rows, cols, products in ((100, 60, 3), (200, 256, 3), (256, 140, 1)):
        u = torch.randn(rows, cols, device="cuda")
        out = torch.full((rows, cols), 7.0, device="cuda")
        ws = torch.zeros(B.orthogonal_ws_bytes(1, rows, cols), dtype=torch.uint8, device="cuda")
        status.zero_()
        assert B.lib().ssgd_orthogonal_wait_selftest(u.data_ptr(), 0, rows, cols, f, products, out.data_ptr(), 0, ws.data_ptr(), status.data_ptr(), stream) == 0
        torch.cuda.synchronize()
        assert int(status) == 1 and bool((out == 7.0).all())
        assert ref.off(orthogonal.orthogonalise(u), ref.orthogonal(u)) < 1e-5
    from paper_1802_04434_b200 import waits
    word, _ = waits.status_of(torch.device("cuda", torch.cuda.current_device()))
    word.fill_(1)
    with pytest.raises(RuntimeError, match="in time"):
        loss.check()
    loss.check()


# ---------------------------------------------------------------------------------------------------------------------
# orthogonalised updates


def updates(n, rows, cols, seed=0, rank=None):
    r = gen(seed * 131 + n + 17 * rows + 1003 * cols)
    u = torch.randn(n, rows, cols, generator=r, device="cuda")
    if rank:
        u = torch.randn(n, rows, rank, generator=r, device="cuda") @ torch.randn(n, rank, cols, generator=r, device="cuda")
    return u * torch.exp(0.5 * torch.randn(n, rows, 1, generator=r, device="cuda"))


def exact_enough(got, u, steps=5, f=ref.MUON):
    """As exact as the same products in fp32: within one and a half times their error, or a millionth."""
    want = ref.orthogonal(u, steps, f)
    plain = ref.off(ref.orthogonal(u, steps, f, double=False), want)
    error = ref.off(got, want, ref.KEPT_TO)
    assert error <= max(1.5 * plain, 2.0 ** -20), (error, plain)


# one CTA (up to 128 x 128); clusters of 2, 4, 8, 16 CTAs, one and more tiles each; launches: k split, tiles of 64, 128 and 256 columns, deflated (a short
# side below 256) and not
SHAPES = [(1, 1, 1), (1, 1, 7), (1, 9, 1), (2, 16, 16), (3, 17, 31), (1, 64, 64), (1, 128, 128), (5, 127, 65), (1, 65, 128), (40, 33, 20),
          (1, 129, 3), (1, 129, 129), (1, 3, 200), (2, 130, 64), (1, 200, 200), (3, 256, 256), (1, 140, 500), (1, 500, 140), (1, 384, 300), (9, 150, 140),
          (1, 1000, 17), (1, 17, 1000), (1, 40, 5000), (1, 5000, 40), (1, 503, 777), (1, 777, 503), (1, 512, 512), (2, 1000, 700), (1, 1024, 2048), (30, 256, 260),
          (1, 2048, 1100), (6, 1030, 1024)]


@pytest.mark.parametrize("n,rows,cols", SHAPES)
def test_orthogonalise(orthogonal, n, rows, cols):
    u = updates(n, rows, cols)
    exact_enough(orthogonal.orthogonalise(u), u)
    # 16 bits in, 16 bits out: one rounding of the result beside the error of the products
    for dtype, products, error in ((BF16, 3, 2.0 ** -19), (F16, 3, 2.0 ** -19), (BF16, 1, 4e-3), (BF16, None, 4e-3)):
        v = u.to(dtype)
        want = ref.orthogonal(v)
        got = orthogonal.orthogonalise(v, products=products)
        assert got.dtype == dtype and got.shape == v.shape
        plain = ref.off(ref.orthogonal(v, double=False), want)
        half = ref.HALF_STEP[dtype]
        assert ref.off(got, want) <= half + max(error, 1.5 * plain) + ref.SMALLEST[dtype] * cols
    assert ref.off(orthogonal.orthogonalise(u, dtype=F16), ref.orthogonal(u)) <= 2.0 ** -11 + 1e-5


@pytest.mark.parametrize("rows,cols", [(60, 90), (200, 170), (600, 300), (700, 1500)])
@pytest.mark.parametrize("steps,f", [(1, ref.MUON), (2, ref.MUON), (7, ref.MUON), (5, (1.5, -0.5, 0.0)), (6, (15 / 8, -10 / 8, 3 / 8)), (3, (2.0, -1.5, 0.01)),
                                     (1, (1.0, 0.0, 0.0)), (4, (0.0, 1.0, 0.0))])
def test_steps_and_coefficients(orthogonal, rows, cols, steps, f):
    u = updates(2, rows, cols, seed=steps)
    exact_enough(orthogonal.orthogonalise(u, steps=steps, coefficients=f), u, steps, f)
    assert ref.off(orthogonal.orthogonalise(u, steps=steps, coefficients=f, products=1), ref.orthogonal(u, steps, f), ref.KEPT_TO) <= 4e-3


@pytest.mark.parametrize("rows,cols", [(64, 64), (300, 300), (512, 1024), (1100, 600)])
def test_few_directions(orthogonal, rows, cols):
    # of low rank: what is not in those directions is 0, and grows where arithmetic puts something there
    for rank in (1, 8):
        u = updates(1, rows, cols, rank=rank)
        want = ref.orthogonal(u)
        plain = ref.off(ref.orthogonal(u, double=False), want)
        assert ref.off(orthogonal.orthogonalise(u), want) <= max(1.5 * plain, 2.0 ** -16)


@pytest.mark.parametrize("rows,cols", [(50, 60), (200, 260), (900, 400), (700, 1024)])
def test_sizes_of_numbers(orthogonal, rows, cols):
    u = updates(4, rows, cols)
    plain = orthogonal.orthogonalise(u)
    for scale in (2.0 ** -100, 2.0 ** 100):                  # powers of two change nothing
        assert torch.equal(orthogonal.orthogonalise(u * scale), plain)
    tiny = u * 1e-38                                         # subnormal: fewer bits, still a matrix
    assert ref.off(orthogonal.orthogonalise(tiny), ref.orthogonal(tiny)) < 1e-5
    huge = u / u.abs().max() * 3e38
    assert ref.off(orthogonal.orthogonalise(huge), ref.orthogonal(huge)) < 1e-5
    u[1] = 0
    u[2, 3, 4] = float("nan")
    u[3, 5, 6] = float("inf")
    for products in (1, 3):
        got = orthogonal.orthogonalise(u, products=products)
        assert not got[1].any() and bool(got[2].isnan().all()) and bool(got[3].isnan().all()) and bool(torch.isfinite(got[0]).all())
    assert torch.equal(got[0], plain[0])                     # its neighbours have not felt them


@pytest.mark.parametrize("rows,cols", [(33, 50), (128, 100), (200, 150), (130, 640), (700, 333)])
def test_places(orthogonal, rows, cols):
    u = updates(3, rows, cols)
    plain = orthogonal.orthogonalise(u)
    assert torch.equal(orthogonal.orthogonalise(u.transpose(1, 2).contiguous().transpose(1, 2)), plain)
    for ld, off_ in ((cols + 1, 0), (cols + 5, 3), ((cols + 7) // 4 * 4, 4 if cols % 4 == 0 else 1)):
        big = torch.full((3, rows + 2, ld + off_), 7.0, device="cuda")
        view = big[:, 1:1 + rows, off_:off_ + cols]
        view.copy_(u)
        assert torch.equal(orthogonal.orthogonalise(view), plain)
        for dtype in (F32, BF16, F16):
            out = torch.full_like(big, 7.0, dtype=dtype)
            place = out[:, 1:1 + rows, off_:off_ + cols]
            got = orthogonal.orthogonalise(view, out=place, products=3)
            assert got.data_ptr() == place.data_ptr() and torch.equal(place, orthogonal.orthogonalise(u, dtype=dtype, products=3))
            place.fill_(7.0)
            assert bool((out == 7.0).all())                  # what lies around is as it was
        assert torch.equal(orthogonal.orthogonalise(view, out=view), plain)      # in place
        view.fill_(7.0)
        assert bool((big == 7.0).all())
    assert torch.equal(orthogonal.orthogonalise(u[:1].expand(3, rows, cols)), orthogonal.orthogonalise(u[:1].repeat(3, 1, 1)))
    assert torch.equal(orthogonal.orthogonalise(u.view(3, 1, rows, cols)), plain.view(3, 1, rows, cols))
    assert torch.equal(orthogonal.orthogonalise(u[1]), orthogonal.orthogonalise(u[1:2])[0])


def test_nothing(orthogonal):
    for shape in ((0, 5, 6), (3, 0, 6), (3, 5, 0), (0, 5)):
        assert orthogonal.orthogonalise(torch.zeros(shape, device="cuda")).shape == shape
        x = torch.zeros(shape, device="cuda")
        orthogonal.momentum_step(x, x, x, 0.9, 0.1)
    with pytest.raises(ValueError, match="32768"):
        orthogonal.orthogonalise(torch.zeros(1, 40000, device="cuda"))


@pytest.mark.parametrize("g_type", [F32, BF16, F16])
@pytest.mark.parametrize("n,rows,cols", [(1, 5, 3), (2, 100, 64), (1, 130, 200), (2, 300, 129), (1, 700, 600), (1, 1999, 503)])
def test_momentum_step(orthogonal, n, rows, cols, g_type):
    for nesterov in (False, True):
        for products in (1, 3):
            # views of flat vectors with other things between the matrices, as a model's parameters lie
            span = rows * cols + 37
            flat = [torch.full((n * span,), 7.0, device="cuda") for _ in range(2)]
            x, m = [f.as_strided((n, rows, cols), (span, cols, 1)) for f in flat]
            x0, m0, g = updates(n, rows, cols, 1) * 0.02, updates(n, rows, cols, 2) * 1e-3, (updates(n, rows, cols, 3) * 1e-3).to(g_type)
            x.copy_(x0), m.copy_(m0)
            beta, delta = 0.9, 0.03
            orthogonal.momentum_step(x, g, m, beta, delta, nesterov=nesterov, products=products)
            # fl((1 - beta) g) and one rounding of beta m + that, beta in fp32; the sum in fp64 first, so off by an ulp where that rounds twice
            b32 = torch.tensor(beta, dtype=F32).item()
            part = (torch.tensor(1.0, dtype=F32) - torch.tensor(beta, dtype=F32)).item() * g.float()
            want = b32 * m0.double() + part.double()
            assert bool(((m.double() - want).abs() <= 2.0 ** -23 * want.abs() + 2.0 ** -149).all())
            u = b32 * m.double() + part.double() if nesterov else m.double()
            move = ref.orthogonal(u)
            error = 1e-5 if products == 3 else 4e-3
            assert ref.off(x, x0.double() - delta * move) <= 2.0 ** -24 + error * delta * float(move.norm()) / float((x0.double() - delta * move).norm()) + 1e-9
            between = torch.ones(n * span, dtype=torch.bool, device="cuda")
            between.as_strided((n, rows, cols), (span, cols, 1)).fill_(False)
            assert all(bool((f[between] == 7.0).all()) for f in flat)
    with pytest.raises(ValueError, match="share memory"):
        orthogonal.momentum_step(x, x, m, 0.9, 0.1)


def test_orthogonal_repeats_its_bits(orthogonal):
    for n, rows, cols in ((2, 100, 90), (2, 300, 200), (1, 1030, 600)):
        u = updates(n, rows, cols)
        for products in (1, 3):
            first = orthogonal.orthogonalise(u, products=products)
            for _ in range(4):
                assert torch.equal(orthogonal.orthogonalise(u, products=products), first)


def test_orthogonal_in_graphs_and_on_streams(orthogonal):
    shapes = ((2, 60, 90), (1, 300, 200), (1, 700, 1100))
    us = [updates(*s) for s in shapes]
    vs = [updates(*s, seed=4) for s in shapes]
    want, other = [[orthogonal.orthogonalise(u) for u in each] for each in (us, vs)]
    static = [u.clone() for u in us]
    graphs = [capture(lambda: [orthogonal.orthogonalise(u) for u in static]) for _ in range(2)]
    for source, expected in ((us, want), (vs, other), (us, want)):
        for s, u in zip(static, source):
            s.copy_(u)
        for graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for _, out in graphs:
            assert all(torch.equal(a, b) for a, b in zip(out, expected))
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    results = []
    for _ in range(4):
        for s, source, expected in zip(streams, (us, vs, us), (want, other, want)):
            with torch.cuda.stream(s):
                results.append(([orthogonal.orthogonalise(u) for u in source], expected))
    torch.cuda.synchronize()
    for got, expected in results:
        assert all(torch.equal(a, b) for a, b in zip(got, expected))


# ---------------------------------------------------------------------------------------------------------------------
# together


def test_align(loss):
    from paper_1802_04434_b200 import binding as B
    a, b = torch.randn(37, 50, device="cuda").half(), torch.randn(61, 9, device="cuda").half()
    out = torch.full((37 + 9, 56), 7.0, dtype=F16, device="cuda")
    assert B.lib().ssgd_xent_align(a.data_ptr(), 50, 1, 37, out.data_ptr(), b.data_ptr(), 1, 9, 9, out[37:].data_ptr(), 50, 56,
                                   torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(out[:37, :50], a) and torch.equal(out[37:, :50], b[:50].t()) and not out[:, 50:].any()


@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_the_example(fmt):
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import train_language_head as example
    losses, norms, model = example.train(steps=3, vocab=301, width=64, blocks=2, size=200, fmt=fmt)
    assert all(torch.isfinite(torch.tensor(v)).all() for v in (losses, norms)) and bool(torch.isfinite(model.flat).all())
    # its gradients: the loss's products alone, the layers' in fp32 on operands that 4 bits hold are as they are
    gen_ = gen(1)
    permutation = torch.randperm(301, generator=gen_, device="cuda")
    tokens, targets = example.batch(gen_, permutation, 200, "cuda")
    model.blocks, model.hidden = 0, model.hidden[:0]
    parameters = model.parameters()
    value = model.loss(parameters, tokens, targets)
    de, dw = torch.autograd.grad(value, parameters)
    e, w = parameters[0].detach(), parameters[1].detach()
    g = torch.full((200,), 1.0 / int((targets != -100).sum()), device="cuda")
    want, tol = ref.loss_and_gradients(e[tokens], w, targets, g)
    within(dw, want[2], tol[2], "head")
    # rows of the embedding are sums of dh over their tokens, rounded to bf16 each time one is added
    rows = torch.zeros(301, 64, dtype=torch.float64, device="cuda").index_add_(0, tokens, want[1])
    most = torch.bincount(tokens, minlength=301)[:, None]
    sizes = torch.zeros(301, 64, dtype=torch.float64, device="cuda").index_add_(0, tokens, want[1].abs() + tol[1])
    bound = torch.zeros(301, 64, dtype=torch.float64, device="cuda").index_add_(0, tokens, tol[1]) + most * 2.0 ** -8 * sizes
    within(de, rows, bound, "embedding")


def test_a_step_of_everything(loss, orthogonal):
    # a layer, the loss, one norm over all gradients, the orthogonalised step, against the same in fp64 on the layer's rounded operands
    from paper_1802_04434_b200 import binding as B, fp4
    r = gen(11)
    held = torch.tensor([-4.0, -2.0, -1.0, 0.0, 1.0, 3.0], device="cuda")      # values that 4 bits hold beside a 6 in every block
    x = held[torch.randint(0, 6, (96, 64), generator=r, device="cuda")]
    w = held[torch.randint(0, 6, (160, 64), generator=r, device="cuda")]
    for t in (x, w):
        t[::16], t[:, ::16] = 6.0, 6.0
    x, w = x.to(BF16), w * 2.0 ** -6
    head = (torch.randn(500, 160, generator=r, device="cuda") * 0.1).to(BF16)
    y = torch.where(torch.rand(96, generator=r, device="cuda") < 0.2, -100, torch.randint(0, 500, (96,), generator=r, device="cuda"))
    hidden, kept = fp4.linear_forward(x, w, "mx")
    losses, kept2 = loss.cross_entropy_forward(hidden, head, y)
    g = torch.full((96,), 1.0 / int((y != -100).sum()), device="cuda")
    dh, dhead = loss.cross_entropy_backward(kept2, g)
    want, tol = ref.loss_and_gradients(hidden, head, y, g)
    assert torch.equal(hidden, (x.float() @ w.t()).to(BF16))                   # exact in 4 bits, one rounding
    within(losses, want[0], tol[0], "losses")
    within(dh, want[1], tol[1], "dh")
    dx, dw = fp4.linear_backward(kept, dh)
    row = torch.zeros(160 * 64 + 500 * 160, device="cuda")
    norm = torch.zeros(1, device="cuda")
    B.tensors_clip(B.TensorTable([dw, dhead], [row[:160 * 64].view_as(dw), row[160 * 64:].view_as(dhead)]), 0.01, norm)
    both = torch.cat([dw.double().flatten(), dhead.double().flatten()])
    assert abs(float(norm) - float(both.norm())) <= 2.0 ** -22 * float(norm)
    p, m = w.clone(), torch.zeros_like(w)
    clipped = row[:160 * 64].view(160, 64)
    orthogonal.momentum_step(p, clipped, m, 0.9, 0.05)
    b32 = torch.tensor(0.9, dtype=F32)
    assert ref.off(m, (1 - b32).item() * clipped.double()) <= 2.0 ** -23
    move = ref.orthogonal(m)
    assert ref.off(p, w.double() - 0.05 * move) <= 2.0 ** -24 + 1e-5 * 0.05 * float(move.norm() / w.double().norm()) * 1.1
