"""What the torch-level calls of the layer operators refuse before any address reaches the library (no GPU needed)."""
import pytest
import torch

from paper_2607_26444_b200 import binding as B


def test_scales_are_fp32():
    """A narrower tensor would be written and read beyond its end, a wider or an integer one misread."""
    for dtype in (torch.bfloat16, torch.float16, torch.int8, torch.float64, torch.int32):
        with pytest.raises(ValueError):
            B._scale_stride(torch.ones(16, dtype=dtype), 16)
    assert B._scale_stride(torch.ones(16), 16) == 1


def test_broadcast_scales_are_refused():
    """A stride of zero would be taken for one, and rows - 1 scales read behind the only one there is."""
    for t in (torch.ones(1).expand(16), torch.ones(1, 1).expand(4, 4), torch.ones(()).expand(16)):
        with pytest.raises(ValueError):
            B._scale_stride(t, 16)
    with pytest.raises(ValueError):
        B._scale_stride(torch.ones(4, 1).expand(4, 4), 16)
    assert B._scale_stride(torch.ones(1).expand(1), 1) == 1 and B._scale_stride(torch.ones(()), 1) == 1
    assert B._scale_stride(torch.ones(16, 3)[:, 1], 16) == 3 and B._scale_stride(torch.ones(4, 4, 5)[..., 2], 16) == 5
