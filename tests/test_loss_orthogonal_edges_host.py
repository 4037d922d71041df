"""Host side of the loss over a large vocabulary and of orthogonalised updates: layouts, devices' words, what torch's autograd is told.  No GPU."""
import pytest
import torch


def test_batches_of_empty_matrices():
    from paper_1802_04434_b200.orthogonal import _batch
    for shape in ((2, 3, 0, 5), (2, 3, 4, 0), (2, 0, 4, 5), (0, 3, 4, 5), (2, 0, 3, 0, 0), (1, 2, 3, 0, 5)):
        for written in (False, True):
            t, n, ld, stride = _batch(torch.zeros(shape), "t", written)
            assert t.shape == (torch.Size(shape[:-2]).numel(), *shape[-2:]) and n == t.shape[0]


def test_matrices_whose_rows_lie_in_turn():
    from paper_1802_04434_b200.orthogonal import _batch
    flat = torch.zeros(400)
    for n, rows, cols, stride, ld in ((3, 4, 5, 5, 15), (3, 4, 5, 8, 24), (2, 7, 3, 4, 9), (3, 2, 5, 5, 15)):
        t, *got = _batch(flat.as_strided((n, rows, cols), (stride, ld, 1)), "t", True)
        assert t.data_ptr() == flat.data_ptr() and got == [n, ld, stride]
    for n, rows, cols, stride, ld in ((3, 4, 5, 5, 14), (3, 4, 5, 4, 15), (2, 7, 3, 2, 9), (3, 2, 5, 0, 15), (3, 4, 5, 7, 7)):
        with pytest.raises(ValueError, match="share no elements"):
            _batch(flat.as_strided((n, rows, cols), (stride, ld, 1)), "t", True)


def test_shared_elements_at_the_boundary():
    import ctypes
    from paper_1802_04434_b200 import _build, binding as B
    _build.build()
    A, f, SIZE = 0x10000, (ctypes.c_float * 3)(3.4445, -4.7750, 2.0315), 3       # a fake address: these calls fail before touching it
    for n, rows, cols, stride, ld in ((3, 4, 5, 5, 14), (3, 4, 5, 4, 15), (2, 7, 3, 2, 9), (3, 2, 5, 0, 15), (3, 4, 5, 7, 7)):
        assert B.lib().ssgd_orthogonalise(A, 0, n, rows, cols, cols, rows * cols, f, 5, 3, A, 0, ld, stride, A, A, None) == SIZE
        assert B.lib().ssgd_orthogonal_step(A, ld, stride, A, 0, cols, rows * cols, A, cols, rows * cols, n, rows, cols, 0.9, 0.1, 0, f, 5, 3, A, A, None) == SIZE
        assert B.lib().ssgd_orthogonal_step(A, cols, rows * cols, A, 0, cols, rows * cols, A, ld, stride, n, rows, cols, 0.9, 0.1, 0, f, 5, 3, A, A, None) == SIZE


def test_results_that_autograd_would_differentiate(monkeypatch):
    # the library's call replaced: what torch is told of a result
    import types
    from paper_1802_04434_b200 import binding as B, orthogonal

    class Device(torch.Tensor):
        """A tensor that says that it lives in device memory."""
        is_cuda = True
        device = types.SimpleNamespace(index=0)
    monkeypatch.setattr(B, "lib", lambda: types.SimpleNamespace(ssgd_orthogonalise_block=lambda block: 0))
    monkeypatch.setattr(orthogonal, "_current_device", lambda: 0)
    monkeypatch.setattr(orthogonal, "_stream_of", lambda index: 0)
    monkeypatch.setattr(orthogonal, "status_of", lambda device: (None, 0))
    monkeypatch.setattr(orthogonal, "_ws_bytes", lambda *sides: 64)
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *s, dtype=None, device=None: empty(*s, dtype=dtype))
    u = torch.zeros(4, 5).as_subclass(Device).requires_grad_()
    got = orthogonal.orthogonalise(u)
    assert got.requires_grad and got.shape == (4, 5)
    with pytest.raises(RuntimeError, match="no derivative"):
        got.sum().backward()
    with torch.no_grad():
        assert not orthogonal.orthogonalise(u).requires_grad
    assert not orthogonal.orthogonalise(u.detach()).requires_grad
    out = empty(4, 5).as_subclass(Device)
    assert orthogonal.orthogonalise(u, out=out) is out and not out.requires_grad


def test_threads_share_a_devices_word(monkeypatch):
    import threading
    import time
    from paper_1802_04434_b200 import fp4, loss, orthogonal, waits
    made = []

    def zeros(*a, **k):
        time.sleep(0.05)
        made.append(torch.ones(1))
        return made[-1]
    device = torch.device("cuda", 63)
    monkeypatch.setattr(torch, "zeros", zeros)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda device: None)
    words = []
    threads = [threading.Thread(target=lambda: words.append(waits.status_of(device))) for _ in range(8)]
    try:
        for t in threads:
            t.start()
        for t in threads:
            t.join()
    finally:
        waits._status.pop(device, None)
    assert len(made) == 1 and {w[1] for w in words} == {made[0].data_ptr()}
    # one word and one check for the products of every kind
    assert fp4._status is waits._status and fp4.check is loss.check is orthogonal.check is waits.check


def test_results_may_be_changed_in_place():
    # scaled before it is added to something, as an update is
    from paper_1802_04434_b200.orthogonal import _NoDerivative
    u = torch.ones(3, 4, requires_grad=True)
    result = torch.full((3, 4), 2.0)
    got = _NoDerivative.apply(result, u)
    got.mul_(0.5).add_(1.0)
    assert got.data_ptr() == result.data_ptr() and bool((got == 2.0).all()) and got.requires_grad
    with pytest.raises(RuntimeError, match="no derivative"):
        got.sum().backward()
