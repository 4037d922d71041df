"""Host side of the operands, the linear layer and the tables of tensors at their edges: refusals, devices and gradients, with
stand-ins for device tensors and for the library, no GPU."""
import os
import sys

import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
torch = pytest.importorskip("torch")
import torch.utils.checkpoint  # noqa: E402

F32, BF16, U8 = torch.float32, torch.bfloat16, torch.uint8


@pytest.fixture(scope="module")
def B():
    from paper_1802_04434_b200 import _build, binding
    _build.build()
    binding.lib()
    return binding


@pytest.fixture(scope="module")
def fp4(B):
    from paper_1802_04434_b200 import fp4
    return fp4


class Standin:
    """A device tensor as far as the host side looks at it."""

    def __init__(self, *shape, dtype=F32, index=0, address=0x10000):
        self.shape, self.dtype, self.device, self.is_cuda, self._address = shape, dtype, torch.device("cuda", index), True, address

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def stride(self, dim=None):
        s = [1]
        for n in self.shape[:0:-1]:
            s.insert(0, s[0] * n)
        return tuple(s) if dim is None else s[dim]

    def is_contiguous(self):
        return True

    def get_device(self):
        return self.device.index

    def element_size(self):
        return 2 if self.dtype == BF16 else 1 if self.dtype == U8 else 4

    def data_ptr(self):
        return self._address if self.numel() else 0


def test_an_empty_maximum_or_tensor_scale_is_refused(fp4, B, monkeypatch):
    """Their address is 0, which the library would read as one that was not given: it would look for the maximum itself, in a
    workspace that is not there, or take the scale as 1."""
    monkeypatch.setattr(fp4, "_new", lambda *a: pytest.fail("went on"))
    monkeypatch.setattr(torch, "empty", lambda *a, **k: pytest.fail("went on"))
    none = Standin(0)
    for call in (fp4.quantise, fp4.quantise_columns, fp4.quantise_both):
        with pytest.raises(ValueError, match="amax holds 0"):
            call(Standin(300, 200), "nv", none)
    with pytest.raises(ValueError, match="tensor_scale holds 0"):
        fp4.Packed(Standin(4, 32, dtype=U8), Standin(512, dtype=U8), none, 4, 64, "nv")
    codes, scales, ts = Standin(4096, dtype=U8), Standin(4096, dtype=U8), Standin(4)
    with pytest.raises(ValueError, match="amax holds 0"):
        B.fp4_quantise(Standin(4, 64), 4, 64, 64, "nv", none, ts, codes, scales, None, None, 0)
    with pytest.raises(ValueError, match="tensor_scale holds 0"):
        B.fp4_dequantise(codes, scales, none, "nv", 4, 64, Standin(4, 64), 64, 0)
    for a, b, name in ((none, None, "a_tensor_scale"), (ts, none, "b_tensor_scale")):
        with pytest.raises(ValueError, match=name + " holds 0"):
            B.fp4_matmul(codes, scales, a, codes, scales, b, 4, 4, 64, "nv", Standin(4, 4), 4, Standin(1, dtype=torch.int32), 0)


class Devices:
    """Stands in for the runtime: the current device, a device's stream, and what the library was called with on which device."""

    def __init__(self, fp4, B, monkeypatch):
        self.current, self.calls = 0, []
        outer = self

        class Switch:
            def __init__(self, index):
                self.index = index

            def __enter__(self):
                self.before, outer.current = outer.current, self.index

            def __exit__(self, *exc):
                outer.current = self.before

        class Library:
            def __getattr__(self, name):
                def call(*args):
                    if name == "ssgd_fp4_scale_bytes":
                        return 512
                    words = args
                    if name.endswith("_block"):
                        pack = {"ssgd_fp4_quantise_block": B.FP4_QUANTISE_ARGS, "ssgd_fp4_dequantise_block": B.FP4_DEQUANTISE_ARGS,
                                "ssgd_fp4_matmul_block": B.FP4_MATMUL_ARGS, "ssgd_tensors_clip_block": B._CLIP_ARGS}[name]
                        words = pack.unpack(args[0])
                    outer.calls.append((name, outer.current, words[-1]))
                    return 0
                return call

        monkeypatch.setattr(torch.cuda, "device", Switch)
        monkeypatch.setattr(B, "_current_device", lambda: outer.current, raising=False)
        monkeypatch.setattr(fp4, "_current_device", lambda: outer.current, raising=False)
        monkeypatch.setattr(B, "lib", lambda: Library())
        monkeypatch.setattr(B, "_ptr", lambda t, *a: None if t is None else t.data_ptr())
        monkeypatch.setattr(B, "_typed_ptr", lambda t, *a: t.data_ptr())
        monkeypatch.setattr(B, "_stream_of", lambda index: 1000 + index)
        monkeypatch.setattr(fp4, "_stream_of", lambda index: 1000 + index)
        monkeypatch.setattr(B, "_stream", lambda stream: 1000 + outer.current if stream is None else stream)
        monkeypatch.setattr(torch, "empty", lambda *s, dtype=F32, device=None: Standin(*s, dtype=dtype, index=device.index))
        for i in (0, 1):
            monkeypatch.setitem(fp4._status, torch.device("cuda", i), (None, 0x7000))


def test_calls_run_on_their_operands_device(fp4, B, monkeypatch):
    """With device 0 current, operands on device 1: that device is current when the library is called, with its stream, and 0 again
    afterwards."""
    d = Devices(fp4, B, monkeypatch)
    for index in (1, 0):
        at = {"index": index}
        x = Standin(64, 96, **at)
        p = fp4.quantise(x, "nv", Standin(1, **at))
        fp4.quantise_columns(x)
        fp4.quantise_both(x, "nv")
        fp4.dequantise(p)
        fp4.matmul(p, p)
        u8 = Standin(1 << 16, dtype=U8, **at)
        B.fp4_quantise(x, 64, 96, 96, "mx", None, None, u8, u8, None, None)
        B.fp4_dequantise(u8, u8, None, "mx", 64, 96, x, 96)
        B.fp4_matmul(u8, u8, None, u8, u8, None, 64, 64, 96, "mx", Standin(64, 64, **at), 64, Standin(1, **at))
        table = object.__new__(B.TensorTable)
        table.workers, table.device, table._index, table._args, table._ws = 1, torch.device("cuda", index), index, (0x1000, 1, 1), 0x2000
        B.tensors_norm(table, Standin(1, **at))
        B.tensors_clip(table, 1.0, Standin(1, **at))
        names = {c[0] for c in d.calls}
        assert len(d.calls) == 10 and len(names) == 8 and d.current == 0
        assert all(c[1:] == (index, 1000 + index) for c in d.calls), d.calls
        d.calls.clear()


def test_operands_of_two_devices_are_refused(fp4, B, monkeypatch):
    d = Devices(fp4, B, monkeypatch)
    x, other, u8, elsewhere = Standin(64, 96), Standin(4, index=1), Standin(1 << 16, dtype=U8), Standin(1 << 16, dtype=U8, index=1)
    table = object.__new__(B.TensorTable)
    table.workers, table.device, table._index, table._args, table._ws = 1, torch.device("cuda", 0), 0, (0x1000, 1, 1), 0x2000
    for call in (lambda: fp4.quantise(x, "nv", other), lambda: B.tensors_norm(table, other), lambda: B.tensors_clip(table, 1.0, other),
                 lambda: B.fp4_quantise(x, 64, 96, 96, "nv", other, Standin(4), u8, u8, None, None),
                 lambda: B.fp4_quantise(x, 64, 96, 96, "mx", None, None, u8, elsewhere, None, None),
                 lambda: B.fp4_quantise(x, 64, 96, 96, "mx", None, None, None, None, elsewhere, u8),
                 lambda: B.fp4_dequantise(u8, u8, other, "nv", 64, 96, x, 96),
                 lambda: B.fp4_dequantise(elsewhere, elsewhere, None, "mx", 64, 96, x, 96),
                 lambda: B.fp4_matmul(u8, u8, None, elsewhere, u8, None, 64, 64, 96, "mx", Standin(64, 64), 64, Standin(1)),
                 lambda: B.fp4_matmul(u8, u8, None, u8, u8, None, 64, 64, 96, "mx", Standin(64, 64), 64, other)):
        with pytest.raises(ValueError, match="device"):
            call()
    assert d.calls == []


def test_mx_has_no_tensor_scale(fp4, B):
    """Values of the mx format have a block scale alone: a product used to multiply by a tensor scale that reading back left out."""
    codes, scales, ts = Standin(64, dtype=U8), Standin(512, dtype=U8), Standin(1)
    with pytest.raises(ValueError, match="mx"):
        fp4.Packed(codes, scales, ts, 4, 32, "mx")
    assert fp4.Packed(codes, scales, None, 4, 32, "mx").tensor_scale is None
    assert fp4.Packed(codes, scales, ts, 4, 32, "nv").tensor_scale is ts
    A, OK, ARG = 0x10000, 0, 4
    f = B.lib().ssgd_fp4_matmul
    for a, b in ((A, None), (None, A), (A, A)):
        assert f(A, A, a, A, A, b, 4, 8, 64, 0, A, 1, 8, A, None) == ARG
        assert f(A, A, a, A, A, b, 0, 8, 64, 0, A, 1, 8, A, None) == ARG
    assert f(A, A, A, A, A, A, 0, 8, 64, 1, A, 1, 8, A, None) == OK and f(A, A, None, A, A, None, 0, 8, 64, 0, A, 1, 8, A, None) == OK


class OnDevice(torch.Tensor):
    """A host tensor that says it lives on device 0."""
    device = property(lambda self: torch.device("cuda", 0))

    def get_device(self):
        return 0


def on_device(*shape):
    return torch.zeros(*shape).as_subclass(OnDevice)


def test_a_table_leaves_no_work_pending_on_its_stream(B, monkeypatch):
    """The workspace is not filled: the fill would be pending on the stream that builds the table, and could clear the partial sums of
    a call on another."""
    made = []

    def make(name, real):
        def f(*shape, device=None, **k):
            if device is not None and torch.device(device).type == "cuda":
                made.append(name)
            return real(*shape, **k)
        return f

    for name in ("zeros", "ones", "full", "empty"):
        monkeypatch.setattr(torch, name, make(name, getattr(torch, name)))
    monkeypatch.setattr(torch.Tensor, "to", lambda self, *a, **k: self)
    table = B.TensorTable([on_device(5), on_device(9000)], [on_device(5), None], [0, 1])
    assert made == ["empty"] and table.ws.numel() == 32 and table.tiles == 3


# ---------------------------------------------------------------------------------------------------------------------
# the linear layer with quantisation and product replaced by exact ones on the host


@pytest.fixture
def exact(fp4, monkeypatch):
    """Packed matrices whose buffer holds the float32 values themselves; what was packed, in order."""
    packed = []

    def quantise(x, fmt, amax, by_rows, by_columns):
        assert x.dim() == 2
        packed.append((tuple(x.shape), by_rows, by_columns))
        rows, cols = x.shape
        values = x.detach().float().contiguous()
        buffer = torch.cat([values.reshape(-1), values.t().reshape(-1)]).view(U8)
        r = fp4._packed_in(buffer, buffer.data_ptr(), 0, 0, None, rows, cols, fmt, x.device)
        c = fp4._packed_in(buffer, buffer.data_ptr(), 4 * rows * cols, 0, None, cols, rows, fmt, x.device)
        return (r, c) if by_rows and by_columns else r if by_rows else c

    def values(p):
        buffer, (at, _, _) = p._buffer
        assert p.pointers[0] == buffer.data_ptr() + at
        return buffer[at:at + 4 * p.rows * p.cols].view(F32).view(p.rows, p.cols)

    def matmul(a, b, dtype=BF16, out=None):
        assert a.fmt == b.fmt and a.cols == b.cols
        y = (values(a) @ values(b).t()).to(dtype)
        return y if out is None else out.copy_(y)

    monkeypatch.setattr(fp4, "_quantise", quantise)
    monkeypatch.setattr(fp4, "matmul", matmul)
    return packed


def leaf(*shape, seed=0):
    g = torch.Generator()
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g).requires_grad_()


def test_second_derivatives_of_the_layer_are_an_error(fp4, exact):
    """They would have been left out in silence: a gradient penalty added to a loss changed nothing."""
    for loss_of in (lambda y: y.sum(), lambda y: y.square().sum()):            # a gradient of y that depends on nothing, and one that does
        x, w = leaf(5, 8, seed=1), leaf(3, 8, seed=2)
        y = fp4.linear(x, w)
        for wanted in ((x,), (w,), (x, w)):
            first = torch.autograd.grad(loss_of(y), wanted, create_graph=True)
            plain = torch.autograd.grad(loss_of(torch.nn.functional.linear(x, w)), wanted)
            assert all(torch.allclose(a, b, rtol=1e-5, atol=1e-6) for a, b in zip(first, plain))
            with pytest.raises(RuntimeError, match="once"):
                (loss_of(y) + sum(g.square().sum() for g in first)).backward(retain_graph=True)
        loss_of(fp4.linear(x, w)).backward(create_graph=True)                  # first derivatives alone go on as before
        assert x.grad.shape == x.shape and w.grad.shape == w.shape


@pytest.mark.parametrize("mode", [torch.no_grad, torch.inference_mode])
def test_without_gradients_only_rows_are_packed(fp4, exact, mode):
    """Parameters that want gradients, and a call that can have none: nothing is packed for a backward pass."""
    x, w = leaf(2, 5, 8, seed=1), leaf(3, 8, seed=2)
    with mode():
        y = fp4.linear(x, w)
        assert torch.allclose(y, torch.nn.functional.linear(x, w), rtol=1e-5, atol=1e-6) and not y.requires_grad
    assert exact == [((10, 8), True, False), ((3, 8), True, False)]
    del exact[:]
    fp4.linear(x, w)
    fp4.linear(x, w.detach())
    fp4.linear(x.detach(), w)
    fp4.linear(x.detach(), w.detach())
    assert [p[2] for p in exact] == [True, True, False, True, True, False, False, False]


@pytest.mark.parametrize("lead,n_in,n_out", [((5,), 0, 3), ((2, 5), 0, 3), ((5,), 8, 0), ((2, 5), 8, 0), ((5,), 0, 0), ((0,), 8, 3), ((0, 4), 0, 3), ((2, 0), 8, 0),
                                             ((), 8, 3), ((), 0, 3)])
def test_layers_without_inputs_outputs_or_tokens(fp4, exact, lead, n_in, n_out):
    x, w = leaf(*lead, n_in, seed=1), leaf(n_out, n_in, seed=2)
    y = fp4.linear(x, w)
    want = torch.nn.functional.linear(x, w)
    assert y.shape == want.shape == (*lead, n_out) and torch.allclose(y, want, rtol=1e-5, atol=1e-6)
    y.sum().backward()
    got, x.grad, w.grad = (x.grad, w.grad), None, None
    want.sum().backward()
    assert all(a.shape == b.shape and torch.allclose(a, b, rtol=1e-5, atol=1e-6) for a, b in zip(got, (x.grad, w.grad)))


def test_what_the_layer_keeps_is_saved_the_way_of_autograd(fp4, exact):
    """Hooks on saved tensors (offloading, checkpointing) see the packed operands, and a backward pass frees them."""
    x, w = leaf(5, 8, seed=1), leaf(3, 8, seed=2)
    seen = []

    def pack(t):
        seen.append(t)
        return t.clone()

    with torch.autograd.graph.saved_tensors_hooks(pack, lambda t: t.clone()):
        y = fp4.linear(x, w)
    assert [t.dtype for t in seen] == [U8, U8]
    got = torch.autograd.grad(y.sum(), (x, w), retain_graph=True)
    want = torch.autograd.grad(torch.nn.functional.linear(x, w).sum(), (x, w))
    assert all(torch.allclose(a, b, rtol=1e-5, atol=1e-6) for a, b in zip(got, want))
    torch.autograd.grad(y.sum(), (x, w))                       # the graph goes, and what it kept with it
    with pytest.raises(RuntimeError, match="retain_graph"):
        torch.autograd.grad(y.sum(), (x, w))
    for a, b in ((x, w.detach()), (x.detach(), w)):
        y = fp4.linear(a, b)
        got, = torch.autograd.grad(y.sum(), [t for t in (a, b) if t.requires_grad])
        assert torch.allclose(got, want[0] if a is x else want[1], rtol=1e-5, atol=1e-6)
    y = torch.utils.checkpoint.checkpoint(lambda a, b: fp4.linear(a, b).square(), x, w, use_reentrant=False)
    got = torch.autograd.grad(y.sum(), (x, w))
    want = torch.autograd.grad(torch.nn.functional.linear(x, w).square().sum(), (x, w))
    assert all(torch.allclose(a, b, rtol=1e-4, atol=1e-5) for a, b in zip(got, want))


def test_unknown_types_formats_and_kinds_are_refused_by_name(fp4, B, monkeypatch):
    """As quantise refuses them, and before anything is allocated."""
    d = Devices(fp4, B, monkeypatch)
    monkeypatch.setattr(torch, "empty", lambda *a, **k: pytest.fail("allocated"))
    u8 = Standin(1 << 16, dtype=U8)
    p = fp4.Packed(u8, u8, None, 64, 96, "mx")
    for dtype in (torch.float64, torch.int32, None):
        with pytest.raises(TypeError, match="float32, bfloat16 or float16"):
            fp4.dequantise(p, dtype)
        with pytest.raises(TypeError, match="float32, bfloat16 or float16"):
            fp4.matmul(p, p, dtype)
    with pytest.raises(TypeError, match="float32, bfloat16 or float16"):
        fp4.matmul(p, p, out=Standin(64, 64, dtype=torch.float64))
    x, out, status = Standin(64, 96), Standin(64, 96), Standin(1, dtype=torch.int32)
    for call in (lambda f: B.fp4_scale_bytes(f, 64, 96), lambda f: B.fp4_quantise(x, 64, 96, 96, f, None, None, u8, u8, None, None),
                 lambda f: B.fp4_dequantise(u8, u8, None, f, 64, 96, out, 96),
                 lambda f: B.fp4_matmul(u8, u8, None, u8, u8, None, 64, 64, 96, f, out, 64, status)):
        with pytest.raises(ValueError, match="fmt must be 'mx' or 'nv'"):
            call("e4")
    table = object.__new__(B.TensorTable)
    table.workers, table.device, table._index, table._args, table._ws = 1, torch.device("cuda", 0), 0, (0x1000, 1, 1), 0x2000
    for call in (lambda: B.tensors_norm(table, Standin(1), "l2"), lambda: B.tensors_clip(table, 1.0, Standin(1), "l2")):
        with pytest.raises(ValueError, match="kind must be 'two' or 'max'"):
            call()
    with pytest.raises(ValueError, match="tensor_scale"):
        B.fp4_quantise(x, 64, 96, 96, "nv", None, None, u8, u8, None, None)
    with pytest.raises(ValueError, match="scales of codes_t"):
        B.fp4_quantise(x, 64, 96, 96, "mx", None, None, None, None, u8, None)
    assert d.calls == []


def test_forms_of_the_product(B):
    f = B.fp4_matmul_form
    assert f(8192, 8192, 8192) == (2, 256, 1, True, 14) and f(777, 1111, 1500) == (2, 64, 1, False, 1) and f(777, 1104, 1500, ldo=1112).wide
    assert f(1, 4096, 1024) == (1, 16, 1, False, 1) and f(128, 3000, 3300) == (1, 128, 4, False, 1) and f(129, 3000, 3300).ctas == 2
    assert not f(777, 1104, 1500, ldo=1110).wide and not f(777, 1111, 1500, ldo=1112).wide
    assert f(777, 1108, 1500, torch.float32, 1112).wide and not f(777, 1108, 1500, torch.float32, 1110).wide and not f(777, 1108, 1500, ldo=1112).wide
    import ctypes
    out = (ctypes.c_uint * 5)()
    g = B.lib().ssgd_fp4_matmul_form
    assert g(1, 1, 1, 0, 1, 148, None) == 1 and g(1, 1, 1, 3, 1, 148, out) == 4 and g(1, 1, 1, 0, 1, 1, out) == 4
    for M, N, K, ldo in ((0, 1, 1, 1), (1, 0, 1, 1), (1, 1, 0, 1), (1 << 31, 1, 1, 1), (1, 1 << 31, 1, 1 << 31), (1, 1, 1 << 31, 1), (1, 2, 1, 1)):
        assert g(M, N, K, 0, ldo, 148, out) == 3
