"""What goes wrong inside the module on PyTorch's tensors comes out as from PyTorch's own functions."""
import pytest
import torch
from torch.utils._python_dispatch import TorchDispatchMode

from paper_2604_17861_amd import model  # noqa: F401
from paper_2604_17861_amd import _binding as B


class Raising(TorchDispatchMode):
    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        raise KeyError("no " + str(func))


def test_what_a_dispatch_mode_raises_keeps_its_type():
    x = torch.zeros(4)
    with Raising(), pytest.raises(KeyError, match="no aten"):
        torch.empty(4)
    with Raising(), pytest.raises(KeyError, match="no aten"):
        B.like(x)
