"""What the Python binding of the training operators refuses before anything is enqueued; without a GPU: its tensors are stand-ins that
say they are on one."""
import pytest
import torch

from paper_2509_11254_amd import psgd


class OnGpu:
    """A tensor's shape, strides and type, on a GPU that is not there."""

    def __init__(self, tensor, device=0):
        self.tensor, self.index = tensor, device

    is_cuda = True
    device = property(lambda self: torch.device("cuda", self.index))

    def get_device(self):
        return self.index

    def data_ptr(self):
        return 1 << 20

    def __getattr__(self, name):
        return getattr(self.tensor, name)


def matrix(rows, cols, dtype=torch.float32, device=0):
    return OnGpu(torch.empty((rows, (cols + 15) // 16 * 16), dtype=dtype)[:, :cols], device)


def test_rows_that_lie_over_each_other():
    """An expanded row has stride 0, which the head's descriptor would take for d; any stride below the columns is refused."""
    x = torch.empty((1, 64))
    for t in (x.expand(5, 64), torch.empty(1000).as_strided((5, 64), (56, 1)), torch.empty((1, 1)).expand(5, 1)):
        with pytest.raises(ValueError, match="X"):
            psgd._matrix("X", OnGpu(t), *t.shape)
    for t, ld in ((torch.empty((5, 64)), 64), (torch.empty((5, 80))[:, :61], 80), (x, 64), (torch.empty((0, 64)), 64), (torch.empty((5, 8))[:, :1], 8)):
        assert psgd._matrix("X", OnGpu(t), *t.shape) == ld
