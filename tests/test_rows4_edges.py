"""Shapes at the edge of what the operators over 4-bit rows take, on the host: nothing is launched."""
import pytest
import torch

from paper_2607_26444_b200 import binding as B


@pytest.mark.parametrize("shape", [(1, 4), (1, 1, 4)])
def test_scales_whose_last_dimension_is_one_element(shape):
    """A transposed row is contiguous, but the stride of its last dimension, of one element, is not the distance of its scales."""
    scale = torch.ones(shape).transpose(-1, 0)
    assert scale.is_contiguous() and scale.stride(-1) == 4
    assert B._scale_stride(scale, 4) == 1
    codes = torch.zeros((4, 32), dtype=torch.uint8)
    block = torch.zeros((4, 16), dtype=torch.uint8).view(torch.float8_e4m3fn)[:, :4]
    assert B.Rows4(codes, block, scale).c.scale_stride == 1


def test_scales_of_experts_with_one_channel():
    """Weights [E, 1, inner] with scales [E, 1] that were stored as a row."""
    codes = torch.zeros((6, 1, 32), dtype=torch.uint8)
    block = torch.zeros((6, 1, 16), dtype=torch.uint8).view(torch.float8_e4m3fn)[..., :4]
    row = torch.arange(6, dtype=torch.float32)[None]
    q = B.Rows4(codes, block, row.t())
    assert q.rows == 6 and q.c.scale == row.data_ptr() and q.c.scale_stride == 1
    assert B._scale_stride(torch.ones(6, 3)[:, :1], 6) == 3
