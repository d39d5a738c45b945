"""Arguments of the replica operators: what the binding and the host checks make of unusual ones (fake addresses, no GPU)."""
import sys

import pytest
import torch


class Stubborn(torch.Tensor):
    """Says that it is a CUDA tensor, and has no answer to questions about its shape."""

    @staticmethod
    def __new__(cls, *shape):
        return torch.Tensor._make_wrapper_subclass(cls, shape, device="cuda:0", dtype=torch.float32, dispatch_sizes_strides_policy="sizes")

    @classmethod
    def __torch_dispatch__(cls, func, types, args=(), kwargs=None):
        raise ValueError("no shape")


@pytest.mark.parametrize("mode", [0, 1])
def test_a_tensor_that_raises_is_given_back(mode):
    from paper_2403_04206_b200 import build
    build.build_marshal()
    from paper_2403_04206_b200 import _marshal
    x = [Stubborn(4, 8) for _ in range(2)]
    before = sys.getrefcount(x), sys.getrefcount(x[0])
    for _ in range(5):
        with pytest.raises(ValueError, match="no shape"):
            _marshal.tables(x, 0, (("x", x, 4, 8, mode),))
    assert (sys.getrefcount(x), sys.getrefcount(x[0])) == before
