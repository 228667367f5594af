"""Sizes that the C ABI's 32-bit fields cannot hold are refused by the binding, not cut to what they can.  No GPU needed."""
import pytest


@pytest.fixture(scope="module")
def ends():
    import os
    from paper_2503_16815_amd import binding, build, ends as e
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    return e


@pytest.mark.parametrize("which", ["max_rows", "max_vocab", "max_hidden", "max_top_k", "device"])
@pytest.mark.parametrize("value", [(1 << 32) + 8, 1 << 31, -(1 << 31) - 1])
def test_limits_beyond_32_bits(ends, which, value):
    import torch
    sizes = dict(max_rows=8, max_vocab=100, max_hidden=64, max_top_k=4)
    sizes[which] = value
    with pytest.raises(ValueError):
        ends.DeftEnds(ends.OPERATORS, torch.float32, **sizes)


def test_tensors_beyond_32_bits(ends):
    """(Tensors of no elements: what is refused is the number of rows or columns.)"""
    import torch
    e = object.__new__(ends.DeftEnds)
    e._h, e.dtype, e.device, e._index = None, torch.float32, torch.device("cpu"), -1
    for shape in ((1 << 31, 0), ((1 << 32) + 3, 0), (0, 1 << 31)):
        with pytest.raises(ValueError):
            e._rows("x", torch.empty(shape), None, None)
        with pytest.raises(ValueError):
            e._words("x", torch.empty(shape, dtype=torch.int32), torch.int32, (None, None))
    assert e._rows("x", torch.empty((3, 5)), 3, None) == (3, 5)
