"""CPU-only: outputs that the calls allocate have their rows one after the other, whatever strides the input's dimensions of one entry carry."""
import pytest
import torch

from paper_2607_21446_b200 import binding as kb


@pytest.mark.parametrize("shape,stride", [((1, 8), (0, 1)), ((1, 8), (3, 1)), ((1, 8), (999, 1)), ((1, 1, 8), (2, 4, 1)), ((5, 8), (8, 1)), ((5, 8), (9, 1)), ((5, 1, 8), (8, 0, 1))])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_one_after_the_other(shape, stride, dtype):
    like = torch.zeros(2000).as_strided(shape, stride)
    out = kb._empty_rows(like, dtype, None)
    assert out.dtype is dtype and out.stride() == torch.empty(shape).stride()
