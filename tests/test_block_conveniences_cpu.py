"""What the allocating calls of the transformer-block operators do with the tensors they are given, before anything reaches a GPU."""
import pytest
import torch

from paper_2412_05781_amd import binding as B


def test_rows_that_start_off_a_boundary_are_copied():
    x = torch.arange(5 * 77, dtype=torch.float16).view(5, 77)
    assert x.data_ptr() % 16 == 0
    for t in (x[1:], x.flatten()[3:3 + 4 * 77].view(4, 77), x[:, 1:], x[2:].view(1, 3, 77)):
        assert t.data_ptr() % 16
        f = B._flat(t)
        assert f.data_ptr() % 16 == 0 and torch.equal(f, t.reshape(-1, t.shape[-1])) and f.stride(1) == 1
    assert B._flat(x[:, :70]).data_ptr() == x.data_ptr()               # at a boundary: where it is
