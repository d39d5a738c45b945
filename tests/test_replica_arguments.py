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


class Shaped(torch.Tensor):
    """Says that it is a CUDA tensor, with a shape but without memory."""

    @staticmethod
    def __new__(cls, *shape):
        return torch.Tensor._make_wrapper_subclass(cls, shape, device="cuda:0", dtype=torch.float32)

    @classmethod
    def __torch_dispatch__(cls, func, types, args=(), kwargs=None):
        raise NotImplementedError


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


def test_a_matrix_of_another_shape_is_refused():
    """[d_in, d_hidden] weights in the place of [d_hidden, d_in] ones have as many elements, in another order."""
    from paper_2403_04206_b200 import build
    build.build_marshal()
    from paper_2403_04206_b200 import _marshal

    def tables(*shape):
        return _marshal.tables([Shaped(*shape)], 0, (("w_up", [Shaped(*shape)], 6, 8, 0),))

    for shape in ((8, 6), (3, 16)):
        with pytest.raises(ValueError, match=r"w_up: expected shape \[6, 8\]"):
            tables(*shape)
    for shape in ((6, 8), (48,), (1, 48), (48, 1), (2, 3, 8)):       # the matrix, and the same elements as a vector or by batches
        assert len(tables(*shape)) == 3
    vector = [Shaped(2, 24)]                                  # where a vector is meant, any shape of as many elements will do
    assert len(_marshal.tables(vector, 0, (("x", vector, 48, 1, 0),))) == 3


def test_a_counter_without_elements_is_refused():
    """Its address is 0, which would stand for no counter at all."""
    from paper_2403_04206_b200 import binding
    with pytest.raises(ValueError, match="offset_counter"):
        binding._counter(torch.empty(0, dtype=torch.int64), -1)
    one = torch.zeros(1, dtype=torch.int64)                   # (get_device() of a CPU tensor is -1)
    assert binding._counter(one, -1) == one.data_ptr() and binding._counter(None, -1) is None
