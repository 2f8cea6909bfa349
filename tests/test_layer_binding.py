"""What the torch-level calls of the layer operators refuse before any address reaches the library (no GPU needed)."""
import types

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


def host_context():
    """The attributes that the calls use, with a library call that must not be reached."""
    def reached(*args):
        raise AssertionError("the call reached the library")
    entries = types.SimpleNamespace(strata_moe_route=reached, strata_moe_route_grad=reached)
    return types.SimpleNamespace(h=None, _norm=reached, _c=entries, _raw_stream=lambda index: 0, _stream=lambda: 0,
                                 device=torch.device("cuda", 0), n_tok=4, n_items=8, E=16)


def test_norm_outputs_come_in_pairs():
    """residual_out without a residual, or a scale without codes, would be left as they were."""
    x, w = torch.zeros((4, 64), dtype=torch.bfloat16), torch.ones(64)
    h, scale, q = torch.empty_like(x), torch.empty(4), torch.empty((4, 64), dtype=torch.int8)
    for kw in (dict(residual_out=h), dict(residual=x), dict(q_scale=scale), dict(q=q)):
        with pytest.raises(ValueError):
            B.MoEContext.norm(host_context(), x, w, 1e-6, out=torch.empty_like(x), **kw)
    with pytest.raises(AssertionError):
        B.MoEContext.norm(host_context(), x, w, 1e-6, residual=x, residual_out=h, q=q, q_scale=scale)


def test_ids_weights_and_scales_are_of_their_type():
    """Ids and gate weights have the same shape and element size: swapped, each would be read as the other."""
    ids, w = torch.zeros((4, 2), dtype=torch.int32), torch.zeros((4, 2))
    logits = torch.zeros((4, 16))
    params = B.make_route()
    for args in ((w, ids), (w, w), (ids, ids), (ids.long(), w), (ids, w.double())):
        with pytest.raises(ValueError):
            B.MoEContext.route(host_context(), params, logits, *args)
        with pytest.raises(ValueError):
            B.MoEContext.route_grad(host_context(), params, logits, *args, torch.zeros_like(logits))
    with pytest.raises(ValueError):
        B.MoEContext.route(host_context(), params, logits, ids, w, bias=torch.zeros(16, dtype=torch.int32))
    assert B._flat(ids, B._INT32, 8, "ids") == ids.data_ptr() and B._flat(w, B.STRATA_T_F32, 8, "w") == w.data_ptr()
    with pytest.raises(ValueError):
        B._float_type(ids)
    with pytest.raises(ValueError):
        B._code_type(ids)
