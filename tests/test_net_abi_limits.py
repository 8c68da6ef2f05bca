"""Sizes at the ends of their types' ranges that the C entries of the operators around the layers refuse before anything is launched."""
import os

import pytest

from paper_2408_11200_amd import binding, build, net

UNSUPPORTED = binding.KAN_ERR_UNSUPPORTED
A = 4096          # stands for an aligned device address: nothing here gets as far as reading it


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    return net.load()


@pytest.mark.parametrize("n", [(1 << 30) + 1, (1 << 31) - 8, (1 << 31) - 1])
def test_embedding_of_rows_past_32_bit_channels_is_refused(lib, n):
    """A row's pieces, rounded up, and the channels past its end would not be numbers of 32 bits."""
    assert lib.kan_embedding_forward(4, 10, n, A, A, 1, 1.0, A, 1, None) == UNSUPPORTED
    assert lib.kan_embedding_workspace_bytes(4, 10, n) == 0
    assert lib.kan_embedding_backward(4, 10, n, A, A, 1, 1.0, A, 1, A, 1 << 40, None) == UNSUPPORTED
