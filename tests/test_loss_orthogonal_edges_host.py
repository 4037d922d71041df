"""Host side of the loss over a large vocabulary and of orthogonalised updates: layouts, devices' words, what torch's autograd is told.  No GPU."""
import pytest
import torch


def test_batches_of_empty_matrices():
    from paper_1802_04434_b200.orthogonal import _batch
    for shape in ((2, 3, 0, 5), (2, 3, 4, 0), (2, 0, 4, 5), (0, 3, 4, 5), (2, 0, 3, 0, 0), (1, 2, 3, 0, 5)):
        for written in (False, True):
            t, n, ld, stride = _batch(torch.zeros(shape), "t", written)
            assert t.shape == (torch.Size(shape[:-2]).numel(), *shape[-2:]) and n == t.shape[0]
