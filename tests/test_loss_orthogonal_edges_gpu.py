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
