"""Host-side checks of the loss over a large vocabulary and of orthogonalised updates: refusals and sizes, no GPU."""
import ctypes
import math

import pytest
import torch

A = 0x10000          # a fake, aligned address: these calls must fail before touching it
OK, NULL, ALIGN, SIZE, ARG = 0, 1, 2, 3, 4
F32, BF16, F16 = 0, 1, 2
MUON = (ctypes.c_float * 3)(3.4445, -4.7750, 2.0315)


@pytest.fixture(scope="module")
def B():
    from paper_1802_04434_b200 import _build, binding
    _build.build()
    binding.lib()
    return binding


def forward(B, **change):
    a = dict(h=A, ldh=64, w=A, ldw=64, dtype=BF16, T=4, V=10, D=60, targets=A, ignore=-100, losses=A, lse=A, kinds=A, ws=A, status=A, stream=None)
    a.update(change)
    return B.lib().ssgd_xent_forward(*a.values())


@pytest.mark.parametrize("change,status", [
    (dict(dtype=F32), ARG), (dict(dtype=7), ARG),
    (dict(h=None), NULL), (dict(w=None), NULL), (dict(targets=None), NULL), (dict(ws=None), NULL), (dict(status=None), NULL), (dict(losses=None), NULL),
    (dict(lse=None), NULL), (dict(kinds=None), NULL),
    (dict(h=A + 8), ALIGN), (dict(w=A + 2), ALIGN), (dict(ldh=68), ALIGN), (dict(ldw=100), ALIGN), (dict(ws=A + 4), ALIGN), (dict(targets=A + 4), ALIGN),
    (dict(losses=A + 2), ALIGN), (dict(lse=A + 1), ALIGN), (dict(status=A + 2), ALIGN),
    (dict(ldh=56), SIZE), (dict(ldw=32), SIZE), (dict(V=0), SIZE), (dict(D=0), SIZE), (dict(V=(1 << 30) + 1), SIZE), (dict(T=(1 << 30) + 1), SIZE),
    (dict(T=0), OK), (dict(T=0, h=None, w=None, targets=None, losses=None, ws=None), OK),
])
def test_forward_refusals(B, change, status):
    assert forward(B, **change) == status


def backward(B, **change):
    a = dict(h=A, ldh=64, w=A, ldw=64, dtype=F16, T=4, V=10, D=60, targets=A, lse=A, kinds=A, g=A, g_stride=0, dh=A, lddh=60, dw=A, dw_type=F32, lddw=60,
             ws=A, status=A, stream=None)
    a.update(change)
    return B.lib().ssgd_xent_backward(*a.values())


@pytest.mark.parametrize("change,status", [
    (dict(dtype=F32), ARG), (dict(dw_type=3), ARG), (dict(lddh=59), SIZE), (dict(lddw=59), SIZE), (dict(dh=A + 1), ALIGN), (dict(dw=A + 2), ALIGN),
    (dict(g=A + 2), ALIGN), (dict(lse=None), NULL), (dict(kinds=None), NULL), (dict(g=None), NULL), (dict(h=None), NULL), (dict(ldw=63), ALIGN),
    (dict(lddw=1 << 62), SIZE), (dict(dh=None, dw=None), OK), (dict(T=0, dw=None), OK),
])
def test_backward_refusals(B, change, status):
    assert backward(B, **change) == status


def test_sizes_and_blocks(B):
    L = B.lib()
    n = ctypes.c_size_t()
    assert L.ssgd_xent_sizes(1, 1, 1, None, ctypes.byref(n)) == NULL
    assert B.xent_sizes(0, 10, 10) == (16, 16)
    for f in (L.ssgd_xent_forward_block, L.ssgd_xent_backward_block, L.ssgd_orthogonalise_block, L.ssgd_orthogonal_step_block):
        assert f(None) == NULL
    assert L.ssgd_xent_forward_block(B.XENT_FORWARD_ARGS.pack(A, 64, A, 64, F32, 4, 10, 60, A, -100, A, A, A, A, A, 0)) == ARG
    assert L.ssgd_xent_backward_block(B.XENT_BACKWARD_ARGS.pack(A, 64, A, 64, F16, 4, 10, 60, A, A, A, A, 0, A, 60, A, 3, 60, A, A, 0)) == ARG
    assert L.ssgd_orthogonalise_block(B.ORTHOGONALISE_ARGS.pack(A, F32, 1, 4, 5, 5, 20, 1.0, math.nan, 1.0, 5, 3, A, F32, 5, 20, A, A, 0)) == ARG
    assert L.ssgd_orthogonal_step_block(B.ORTHOGONAL_STEP_ARGS.pack(A, 5, 20, A, F32, 5, 20, A, 5, 20, 1, 4, 5, 1.0, 0.1, 0, 1.0, 1.0, 1.0, 5, 3, A, A, 0)) == ARG
    # self-tests take one round of tiles
    assert L.ssgd_xent_wait_selftest(A, 64, A, 64, BF16, 257, 10, 60, A, -100, A, A, A, A, A, None) == SIZE
    assert L.ssgd_orthogonal_wait_selftest(A, F32, 257, 10, MUON, 3, A, F32, A, A, None) == SIZE


def test_orthogonal_workspace(B):
    ws = B.lib().ssgd_orthogonal_ws_bytes
    assert ws(0, 4, 4) == 0 and ws(1, 0, 4) == 0 and ws(1, 4, 0) == 0 and ws(1, 32769, 4) == 0 and ws(65536, 4, 4) == 0
    # at least both parts of X twice, and of the two squares
    assert ws(3, 100, 200) >= 3 * (8 * 100 * 200 + 8 * 100 * 100) and ws(1, 200, 100) >= 8 * 200 * 100 + 8 * 100 * 100
    with pytest.raises(ValueError, match="32768"):
        B.orthogonal_ws_bytes(1, 40000, 4)


def orthogonalise(B, **change):
    a = dict(u=A, u_type=F32, n=2, rows=4, cols=5, ldu=5, su=20, c=MUON, steps=5, products=3, out=A, out_type=BF16, ldo=5, so=20, ws=A, status=A, stream=None)
    a.update(change)
    return B.lib().ssgd_orthogonalise(*a.values())


@pytest.mark.parametrize("change,status", [
    (dict(u=None), NULL), (dict(out=None), NULL), (dict(c=None), NULL), (dict(ws=None), NULL), (dict(status=None), NULL),
    (dict(u_type=5), ARG), (dict(out_type=-1), ARG), (dict(products=2), ARG), (dict(products=0), ARG), (dict(c=(ctypes.c_float * 3)(1, math.inf, 1)), ARG),
    (dict(u=A + 2), ALIGN), (dict(out=A + 1), ALIGN), (dict(ws=A + 8), ALIGN), (dict(status=A + 1), ALIGN),
    (dict(steps=0), SIZE), (dict(steps=101), SIZE), (dict(rows=0), SIZE), (dict(cols=0), SIZE), (dict(rows=32769), SIZE), (dict(n=65536), SIZE),
    (dict(ldu=4), SIZE), (dict(ldo=4), SIZE), (dict(so=19), SIZE), (dict(so=0), SIZE), (dict(n=0), OK), (dict(n=0, u=None), OK),
])
def test_orthogonalise_refusals(B, change, status):
    assert orthogonalise(B, **change) == status


def step(B, **change):
    a = dict(x=A, ldx=5, sx=20, g=A, g_type=BF16, ldg=5, sg=20, m=A, ldm=5, sm=20, n=2, rows=4, cols=5, beta=0.9, delta=0.1, nesterov=0, c=MUON, steps=5,
             products=3, ws=A, status=A, stream=None)
    a.update(change)
    return B.lib().ssgd_orthogonal_step(*a.values())


@pytest.mark.parametrize("change,status", [
    (dict(beta=1.0), ARG), (dict(beta=-0.1), ARG), (dict(beta=math.nan), ARG), (dict(delta=math.inf), ARG), (dict(delta=math.nan), ARG), (dict(g_type=9), ARG),
    (dict(x=None), NULL), (dict(g=None), NULL), (dict(m=None), NULL), (dict(x=A + 2), ALIGN), (dict(m=A + 2), ALIGN), (dict(g=A + 1), ALIGN),
    (dict(sx=10), SIZE), (dict(sm=0), SIZE), (dict(ldm=3), SIZE), (dict(ldx=4), SIZE), (dict(products=4), ARG), (dict(steps=1000), SIZE), (dict(n=0), OK),
])
def test_step_refusals(B, change, status):
    assert step(B, **change) == status


# ---------------------------------------------------------------------------------------------------------------------
# the layers over torch tensors: what is refused before a device is asked for anything


def test_loss_arguments():
    from paper_1802_04434_b200 import loss
    h, w, y = torch.zeros(3, 8, dtype=torch.bfloat16), torch.zeros(5, 8, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError, match="device memory"):
        loss.cross_entropy_forward(h, w, y)
    with pytest.raises(TypeError, match="bfloat16 or float16"):
        loss.cross_entropy_forward(h.float(), w.float(), y)
    with pytest.raises(TypeError, match="one dtype"):
        loss.cross_entropy_forward(h, w.half(), y)
    with pytest.raises(TypeError, match="int64"):
        loss.cross_entropy_forward(h, w, y.int())
    for bad in ((h[0], w, y), (h, w[0], y), (h, w, y[:2]), (h, w[:, :4], y), (h, w, y.view(3, 1))):
        with pytest.raises(ValueError):
            loss.cross_entropy_forward(*bad)
    with pytest.raises(ValueError, match="reduction"):
        loss.cross_entropy(h, w, y, reduction="max")
    with pytest.raises(ValueError, match="last side"):
        loss.cross_entropy(h, w, y[:2])


def test_loss_backward_arguments():
    from paper_1802_04434_b200 import loss
    kept = loss.Kept(torch.zeros(3, 8, dtype=torch.float16), torch.zeros(5, 8, dtype=torch.float16), None, None, (8, 8), (3, 5, 8))
    g = torch.zeros(3)
    with pytest.raises(TypeError, match="float32"):
        loss.cross_entropy_backward(kept, g.double())
    with pytest.raises(ValueError, match="one gradient"):
        loss.cross_entropy_backward(kept, g[:2])
    with pytest.raises(TypeError, match="float32, bfloat16 or float16"):
        loss.cross_entropy_backward(kept, g, dw_dtype=torch.float64)
    for bad in (torch.zeros(5, 9), torch.zeros(8, 5).t(), torch.zeros(5, 16)[:, ::2]):
        with pytest.raises(ValueError, match="unit column stride"):
            loss.cross_entropy_backward(kept, g, dw=bad)


def test_orthogonal_arguments():
    from paper_1802_04434_b200 import orthogonal
    u = torch.zeros(4, 5)
    with pytest.raises(ValueError, match="device memory"):
        orthogonal.orthogonalise(u)
    with pytest.raises(TypeError, match="float32, bfloat16 or float16"):
        orthogonal.orthogonalise(u.double())
    with pytest.raises(TypeError):
        orthogonal.momentum_step(u.bfloat16(), u, u, 0.9, 0.1)
    with pytest.raises(TypeError):
        orthogonal.momentum_step(u, u, u.half(), 0.9, 0.1)
    with pytest.raises(ValueError, match="device memory"):
        orthogonal.momentum_step(u, u, u, 0.9, 0.1)
    for bad in (dict(steps=0), dict(steps=101), dict(products=2), dict(coefficients=(1.0, 2.0))):
        with pytest.raises(ValueError):
            orthogonal._options(**{**dict(steps=5, coefficients=orthogonal.COEFFICIENTS, products=3), **bad})


def test_batches_of_matrices():
    from paper_1802_04434_b200.orthogonal import _batch
    t, n, ld, stride = _batch(torch.zeros(4, 5), "t", True)
    assert (n, ld, stride) == (1, 5, 20)
    flat = torch.zeros(200)
    t, n, ld, stride = _batch(flat.as_strided((3, 4, 5), (64, 8, 1)), "t", True)      # matrices among other things
    assert (n, ld, stride) == (3, 8, 64) and t.data_ptr() == flat.data_ptr()
    t, n, ld, stride = _batch(torch.zeros(2, 3, 4, 5), "t", True)
    assert (t.shape[0], n, ld, stride) == (6, 6, 5, 20)
    t, n, ld, stride = _batch(torch.zeros(5, 4).t(), "t", False)                      # read only: a copy
    assert t.is_contiguous() and (n, ld, stride) == (1, 5, 20)
    t, n, ld, stride = _batch(torch.zeros(1, 5).expand(4, 5), "t", False)
    assert t.is_contiguous()
    t, n, ld, stride = _batch(torch.zeros(1, 4, 5).expand(3, 4, 5), "t", False)       # one matrix for all
    assert (n, ld, stride) == (3, 5, 0)
    for bad in (torch.zeros(5, 4).t(), torch.zeros(1, 5).expand(4, 5), torch.zeros(1, 4, 5).expand(3, 4, 5), torch.zeros(5),
                torch.zeros(3, 2, 4, 5).transpose(0, 1)):
        with pytest.raises(ValueError):
            _batch(bad, "t", True)


def test_rows_that_copies_can_read():
    from paper_1802_04434_b200.loss import _stride_as_it_is
    whole = torch.arange(7 * 32, dtype=torch.float16).view(7, 32)
    for t, ld in ((whole, 32), (whole[:, 8:20], 32), (whole[::2], 64), (whole[:, 1:9], 0), (whole[:, :30][1:2], 32), (whole.t(), 0), (whole[:1, :30].t(), 0),
                  (torch.zeros(7, 9, dtype=torch.float16), 0), (torch.zeros(9, 1, dtype=torch.float16), 0), (whole[:, ::2], 0), (whole[:1, :9], 16),
                  (whole[:1].expand(5, 32), 0)):
        assert _stride_as_it_is(t, t.shape[1]) == ld


def test_align_refusals(B):
    def align(**change):
        a = dict(a=A + 2, lda=5, step_a=1, rows_a=3, to_a=A, b=A, ldb=1, step_b=9, rows_b=4, to_b=A, cols=5, ldo=8, stream=None)
        a.update(change)
        return B.lib().ssgd_xent_align(*a.values())
    for change, status in ((dict(a=None), NULL), (dict(to_b=None), NULL), (dict(a=A + 1), ALIGN), (dict(to_a=A + 8), ALIGN), (dict(ldo=12), ALIGN), (dict(ldo=0), SIZE),
                           (dict(cols=0), SIZE), (dict(rows_b=(1 << 30) + 1), SIZE), (dict(rows_a=0, rows_b=0), OK), (dict(rows_a=0, rows_b=0, a=None, b=None), OK)):
        assert align(**change) == status


# ---------------------------------------------------------------------------------------------------------------------
# devices, with stand-ins for device tensors, the runtime and the library


class Standin:
    """A device tensor as far as the host side looks at it."""

    def __init__(self, *shape, dtype=torch.float32, index=0, address=0x10000):
        self.shape, self.dtype, self.device, self.is_cuda, self.address = torch.Size(shape), dtype, torch.device("cuda", index), True, address

    def dim(self):
        return len(self.shape)

    def stride(self, dim=None):
        s = [1]
        for n in self.shape[:0:-1]:
            s.insert(0, s[0] * n)
        return tuple(s) if dim is None else s[dim]

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return self.address


@pytest.fixture
def runtime(B, monkeypatch):
    """current: the current device; calls: (call, device that was current, words of its block)."""
    from paper_1802_04434_b200 import loss, orthogonal, waits

    class Runtime:
        current, calls = 0, []
    r = Runtime()
    r.calls = []

    class Switch:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            self.before, r.current = r.current, self.index

        def __exit__(self, *exc):
            r.current = self.before

    class Library:
        def __getattr__(self, name):
            def call(block):
                r.calls.append((name, r.current, [int.from_bytes(block[i:i + 8], "little") for i in range(0, len(block), 8)]))
                return 0
            return call
    monkeypatch.setattr(B, "lib", Library)
    monkeypatch.setattr(B, "_on", Switch)
    monkeypatch.setattr(torch, "empty", lambda *shape, dtype=torch.float32, device=None: Standin(
        *(shape[0] if isinstance(shape[0], (tuple, torch.Size)) else shape), dtype=dtype, index=device.index, address=0x900000))
    for m in (loss, orthogonal):
        monkeypatch.setattr(m, "_current_device", lambda: r.current)
        monkeypatch.setattr(m, "_stream_of", lambda index: 1000 + index)
        monkeypatch.setattr(m, "status_of", lambda device: (None, 0x500 + device.index))
    monkeypatch.setattr(loss, "_sizes", lambda index, *sides: (2 << 20, 64))
    monkeypatch.setattr(orthogonal, "_ws_bytes", lambda *sides: 64)
    return r


@pytest.mark.parametrize("index", [0, 1])
def test_calls_go_to_their_operands_device(runtime, index):
    from paper_1802_04434_b200 import loss, orthogonal
    half = dict(dtype=torch.float16, index=index)
    h, w, y = Standin(6, 16, **half), Standin(9, 16, address=0x20000, **half), Standin(6, dtype=torch.int64, index=index)
    losses, kept = loss.cross_entropy_forward(h, w, y)
    loss.cross_entropy_backward(kept, Standin(6, index=index))
    odd = Standin(6, 13, **half), Standin(9, 13, **half)
    u = Standin(3, 4, 5, index=index)
    orthogonal.orthogonalise(u)
    orthogonal.momentum_step(u, Standin(3, 4, 5, dtype=torch.bfloat16, index=index, address=0x30000), Standin(3, 4, 5, index=index, address=0x40000), 0.9, 0.1)
    assert [c[0] for c in runtime.calls] == ["ssgd_xent_forward_block", "ssgd_xent_backward_block", "ssgd_orthogonalise_block", "ssgd_orthogonal_step_block"]
    for name, current, words in runtime.calls:
        assert current == index and words[-1] == 1000 + index and words[-2] == 0x500 + index, name
    assert runtime.current == 0
    forward, backward, alone, step_ = [c[2] for c in runtime.calls]
    assert forward[:9] == [0x10000, 16, 0x20000, 16, 2, 6, 9, 16, 0x10000] and forward[9] == (1 << 64) - 100
    assert backward[11:13] == [0x10000, 1] and backward[16] == 2
    assert alone[:7] == [0x10000, 0, 3, 4, 5, 5, 20] and alone[10:12] == [5, 3]
    assert step_[3:5] == [0x30000, 1] and step_[7] == 0x40000 and step_[19:21] == [5, 3]
    assert loss._stride_as_it_is(odd[0], 13) == 0


def test_operands_of_two_devices_are_refused(runtime):
    from paper_1802_04434_b200 import loss, orthogonal
    half = dict(dtype=torch.float16)
    h, w, y = Standin(6, 16, **half), Standin(9, 16, **half), Standin(6, dtype=torch.int64)
    for bad in ((h, Standin(9, 16, index=1, **half), y), (h, w, Standin(6, dtype=torch.int64, index=1))):
        with pytest.raises(ValueError, match="one device"):
            loss.cross_entropy_forward(*bad)
    kept = loss.Kept(h, w, y, None, (16, 16), (6, 9, 16))
    with pytest.raises(ValueError, match="operands' device"):
        loss.cross_entropy_backward(kept, Standin(6, index=1))
    with pytest.raises(ValueError, match="operands' device"):
        loss.cross_entropy_backward(kept, Standin(6), dw=Standin(9, 16, index=1))
    u, other = Standin(4, 5), Standin(4, 5, index=1)
    with pytest.raises(ValueError, match="its device"):
        orthogonal.orthogonalise(u, out=other)
    for bad in ((other, u, u), (u, other, u), (u, u, other)):
        with pytest.raises(ValueError, match="one device"):
            orthogonal.momentum_step(*bad, 0.9, 0.1)
    assert runtime.calls == []


def test_products_by_the_results_type(runtime):
    from paper_1802_04434_b200 import orthogonal
    for shape, kind, want in (((256, 300), torch.bfloat16, 1), ((255, 4000), torch.bfloat16, 3), ((300, 300), torch.float16, 3), ((300, 300), torch.float32, 3)):
        orthogonal.orthogonalise(Standin(*shape, dtype=kind))
        assert runtime.calls[-1][2][11] == want
    orthogonal.orthogonalise(Standin(300, 300), dtype=torch.bfloat16, products=3)
    assert runtime.calls[-1][2][11] == 3
