"""Sizes that a 32-bit count does not hold are refused before a call, not cut to their low bits.  No GPU: tensors without memory."""
import pytest
import torch

from paper_2609_25405_b200 import binding as B


def _meta(*shape):
    return torch.empty(shape, dtype=torch.float16, device="meta")


@pytest.mark.parametrize("shape", [(2 ** 32 + 4, 1), (2 ** 31, 1), (1, 2 ** 31), (2, 2 ** 33)])
def test_too_many_rows_or_columns(shape):
    t = _meta(*shape)
    with pytest.raises(ValueError, match=r"2\^31"):
        B._matrix(t, t.get_device(), "x")


def test_the_largest_counts_are_taken():
    t = _meta(2 ** 31 - 1, 1)
    assert B._matrix(t, t.get_device(), "x")[1:4] == (2 ** 31 - 1, 1, 1)
