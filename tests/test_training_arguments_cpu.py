"""Arguments on their way into the library, without a GPU: numbers of other kinds, and sizes that would not fit."""
import numpy as np
import pytest
import torch

from paper_2506_17974_b200 import training as tr


class Matrix:
    """What the checks ask of a tensor, of any size."""
    dtype = torch.bfloat16

    def __init__(self, rows, cols):
        self.shape = rows, cols

    def stride(self):
        return self.shape[1], 1

    def get_device(self):
        return 0

    def data_ptr(self):
        return 0x7f0000000000


@pytest.mark.parametrize("cols", [1 << 31, (1 << 32) + 8, 1 << 40])
def test_more_columns_than_the_library_counts(cols):
    """32 bits hold the number of columns on the way: 2^32 + 8 of them would arrive as 8, and the call would leave the rest of the row undone."""
    with pytest.raises(ValueError, match="columns"):
        tr._matrix(Matrix(1, cols), "x", 0)
    assert tr._matrix(Matrix(1, (1 << 31) - 1), "x", 0) == (0x7f0000000000, (1 << 31) - 1)
    assert tr._matrix(Matrix(1 << 33, 4), "x", 0) == (0x7f0000000000, 4)


def test_whole_numbers_of_numpy():
    want = tr._drop(0.25, 5, 3, 0)
    for kind in (np.int64, np.int32, np.uint32, np.uint64):
        assert tr._drop(0.25, kind(5), kind(3), 0) == want
    assert tr._drop(0.25, np.int64(-4), np.int32(-1), 0) == tr._drop(0.25, -4, -1, 0) == (0.25, 0, 2 ** 64 - 4, 2 ** 64 - 1, 0)
    for seed in (2.5, "5"):
        with pytest.raises(TypeError):
            tr._drop(0.25, seed, 0, 0)


@pytest.mark.parametrize("value", [1e39, -1e39, 1e300, float("inf")])
def test_numbers_past_the_range_of_float32(value):
    with pytest.raises(ValueError, match="eps"):
        tr._real(value, "eps")
    with pytest.raises(ValueError, match="p must"):
        tr._drop(value, 0, 0, 0)
    assert tr._real(1e-5, "eps") == 1e-5 and tr._real(3.4028234663852886e38, "eps") > 3e38      # what a float32 holds is the library's to judge
    assert tr._drop(-0.5, 0, 0, 0)[0] == -0.5 and tr._drop(float("nan"), 0, 0, 0)[0] != tr._drop(float("nan"), 0, 0, 0)[0]
