"""Host side of the operands, the linear layer and the tables of tensors at their edges: refusals, devices and gradients, with
stand-ins for device tensors and for the library, no GPU."""
import os
import sys

import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
torch = pytest.importorskip("torch")

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
