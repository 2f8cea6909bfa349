"""ctypes binding of the C-ABI library: argument marshalling only.

Every function named ``strata_*`` forwards to the C entry point of the same
name (see ``include/strata_moe.h``).  ``MoEContext`` is a small convenience
wrapper that uses torch for device memory and streams; it performs no
arithmetic of its own.  There is no CPU fallback: if the CUDA library has not
been built, loading raises.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional, Tuple

_HERE = os.path.dirname(os.path.abspath(__file__))
# STRATA_MOE_LIB names another build of the same library (the test-hooks variant in the time-out test)
LIB_PATH = os.environ.get("STRATA_MOE_LIB") or os.path.join(_HERE, "libstrata_moe.so")

STRATA_OK = 0
STRATA_ERR_INVALID_ARG = 1
STRATA_ERR_SHAPE = 2
STRATA_ERR_ALIGNMENT = 3
STRATA_ERR_NOT_REGISTERED = 4
STRATA_ERR_CAPACITY = 5
STRATA_ERR_BAD_EXPERT_ID = 6
STRATA_ERR_WORKSPACE = 7
STRATA_ERR_CUDA = 8
STRATA_ERR_TIMEOUT = 9
STRATA_ERR_BAD_ROW = 10

STRATA_BF16 = 0
STRATA_FP8_E4M3_B128 = 1
STRATA_Q8_ROW = 2
STRATA_MXF4_ROW = 3
STRATA_NVF4_ROW = 4
STRATA_Q8_TRAILER = 32               # bytes behind the codes of a Q8_ROW row; the first four are its scale
STRATA_FLAG_ALLOW_UNROUTED = 1

EXPORTS = [
    "strata_status_string", "strata_ctx_create", "strata_ctx_destroy", "strata_moe_workspace_bytes",
    "strata_ctx_set_workspace", "strata_ctx_launch_count", "strata_pool_register", "strata_pool_is_ready",
    "strata_pool_unregister", "strata_pool_carve", "strata_pool_reset", "strata_moe_layout",
    "strata_moe_dispatch", "strata_moe_combine", "strata_moe_recv_view", "strata_device_status",
    "strata_moe_roundtrip_host", "strata_moe_layout_noalloc", "strata_ctx_set_trace",
    "strata_moe_partition_max_units", "strata_moe_partition", "strata_moe_dispatch_windows",
    "strata_moe_recv_rows",
    "strata_ctx_set_timeline", "strata_timeline_decode", "strata_ctx_set_sm_budget", "strata_moe_row_experts",
    "strata_moe_mask_ragged", "strata_moe_expert_affine_inplace", "strata_ctx_set_x_early",
    "strata_allgather", "strata_alltoall", "strata_broadcast", "strata_reducescatter", "strata_allreduce",
    "strata_p2p", "strata_alltoallv",
    "strata_moe_route", "strata_moe_route_grad", "strata_norm", "strata_norm_grad_scratch_bytes", "strata_norm_grad",
    "strata_quantize_rows", "strata_moe_expert_matmul",
    "strata_quantize_rows4", "strata_dequantize_rows4", "strata_moe_expert_matmul4", "strata_moe_balance_scratch_bytes",
    "strata_moe_balance_loss", "strata_moe_balance_grad",
]

# element types and modes of the layer operators (include/strata_layer.h)
STRATA_T_BF16, STRATA_T_F32, STRATA_T_INT8, STRATA_T_E4M3, STRATA_T_MXF4, STRATA_T_NVF4 = 0, 1, 2, 3, 4, 5
STRATA_SCORE_SOFTMAX, STRATA_SCORE_SIGMOID = 0, 1
STRATA_GROUP_MAX, STRATA_GROUP_TOP2 = 0, 1


class strata_moe_shape(ctypes.Structure):
    _fields_ = [("R", ctypes.c_int32), ("T", ctypes.c_int32), ("H", ctypes.c_int32),
                ("E", ctypes.c_int32), ("K", ctypes.c_int32), ("dispatch_dtype", ctypes.c_int32),
                ("segment_align", ctypes.c_int32), ("flags", ctypes.c_int32), ("slot_capacity", ctypes.c_int32)]


class strata_moe_layout_t(ctypes.Structure):
    _fields_ = [("expert_count", ctypes.c_void_p), ("expert_offset", ctypes.c_void_p),
                ("rank_count", ctypes.c_void_p), ("rank_offset", ctypes.c_void_p),
                ("src_expert_count", ctypes.c_void_p), ("dst_row", ctypes.c_void_p),
                ("src_of_row", ctypes.c_void_p)]


class strata_moe_device_buffers(ctypes.Structure):
    _fields_ = [("ids", ctypes.c_void_p), ("x", ctypes.c_void_p), ("w", ctypes.c_void_p),
                ("recv", ctypes.c_void_p), ("out", ctypes.c_void_p), ("layout", strata_moe_layout_t)]


class strata_span(ctypes.Structure):
    _fields_ = [("cta", ctypes.c_uint32), ("kernel", ctypes.c_uint8), ("stage", ctypes.c_uint8),
                ("flags", ctypes.c_uint16), ("begin_ns", ctypes.c_uint64), ("end_ns", ctypes.c_uint64)]


class strata_tier(ctypes.Structure):
    _fields_ = [("alpha", ctypes.c_int64), ("beta", ctypes.c_int64), ("unit_rows", ctypes.c_int64),
                ("fanout_cap", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class strata_partition_policy(ctypes.Structure):
    _fields_ = [("n_tiers", ctypes.c_int32), ("g0", ctypes.c_int32), ("g1", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("tiers", strata_tier * 3)]


class strata_partition_t(ctypes.Structure):
    _fields_ = [("win_base", ctypes.c_void_p), ("unit_desc", ctypes.c_void_p), ("unit_cost", ctypes.c_void_p),
                ("n_units", ctypes.c_void_p), ("task_offset", ctypes.c_void_p), ("task_unit", ctypes.c_void_p),
                ("core_load", ctypes.c_void_p), ("scratch", ctypes.c_void_p), ("task_stripe", ctypes.c_void_p)]


class strata_route_params(ctypes.Structure):
    _fields_ = [("score", ctypes.c_int32), ("renormalise", ctypes.c_int32), ("n_group", ctypes.c_int32),
                ("topk_group", ctypes.c_int32), ("group_score", ctypes.c_int32), ("scale", ctypes.c_float)]


class strata_norm_args(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int32), ("weight_type", ctypes.c_int32),
                ("eps", ctypes.c_float), ("q_type", ctypes.c_int32), ("x", ctypes.c_void_p),
                ("residual", ctypes.c_void_p), ("weight", ctypes.c_void_p), ("residual_out", ctypes.c_void_p),
                ("out", ctypes.c_void_p), ("q", ctypes.c_void_p), ("q_scale", ctypes.c_void_p),
                ("x_stride", ctypes.c_int64), ("residual_stride", ctypes.c_int64),
                ("residual_out_stride", ctypes.c_int64), ("out_stride", ctypes.c_int64), ("q_stride", ctypes.c_int64),
                ("q_scale_stride", ctypes.c_int64)]


# The same layout for a one-call pack: half the cost of filling a ctypes structure (the call takes 2.8 us, its arguments had
# taken 4).
_NORM_ARGS = struct.Struct("@qiifiPPPPPPPqqqqqq")
assert _NORM_ARGS.size == ctypes.sizeof(strata_norm_args)


class strata_norm_grad_args(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int32), ("weight_type", ctypes.c_int32),
                ("eps", ctypes.c_float), ("reserved", ctypes.c_int32), ("dy", ctypes.c_void_p), ("h", ctypes.c_void_p),
                ("weight", ctypes.c_void_p), ("dresidual", ctypes.c_void_p), ("dx", ctypes.c_void_p),
                ("dweight", ctypes.c_void_p), ("scratch", ctypes.c_void_p), ("scratch_bytes", ctypes.c_size_t),
                ("dy_stride", ctypes.c_int64), ("h_stride", ctypes.c_int64), ("dresidual_stride", ctypes.c_int64),
                ("dx_stride", ctypes.c_int64)]


class strata_matmul_args(ctypes.Structure):
    _fields_ = [("type", ctypes.c_int32), ("gated", ctypes.c_int32), ("inner", ctypes.c_int32),
                ("channels", ctypes.c_int32), ("a_rows", ctypes.c_int64), ("a", ctypes.c_void_p),
                ("a_scale", ctypes.c_void_p), ("w", ctypes.c_void_p), ("w_scale", ctypes.c_void_p),
                ("out", ctypes.c_void_p), ("a_stride", ctypes.c_int64), ("a_scale_stride", ctypes.c_int64),
                ("out_stride", ctypes.c_int64)]


class strata_rows4(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("block", ctypes.c_void_p), ("scale", ctypes.c_void_p),
                ("code_stride", ctypes.c_int64), ("block_stride", ctypes.c_int64), ("scale_stride", ctypes.c_int64)]


class strata_matmul4_args(ctypes.Structure):
    _fields_ = [("type", ctypes.c_int32), ("gated", ctypes.c_int32), ("inner", ctypes.c_int32),
                ("channels", ctypes.c_int32), ("a_rows", ctypes.c_int64), ("a", strata_rows4), ("w", strata_rows4),
                ("out", ctypes.c_void_p), ("out_stride", ctypes.c_int64)]


class strata_balance_params(ctypes.Structure):
    _fields_ = [("score", ctypes.c_int32), ("per_rank", ctypes.c_int32), ("weight", ctypes.c_float),
                ("z_weight", ctypes.c_float)]


class strata_balance_stats(ctypes.Structure):
    _fields_ = [("count", ctypes.c_void_p), ("tokens", ctypes.c_void_p), ("prob", ctypes.c_void_p)]


_SCORES = {"softmax": STRATA_SCORE_SOFTMAX, "sigmoid": STRATA_SCORE_SIGMOID}


def make_balance(score: str = "softmax", weight: float = 1.0, z_weight: float = 0.0,
                 per_rank: bool = False) -> strata_balance_params:
    """score: "softmax" or "sigmoid" (normalised); per_rank: a loss for each source rank's tokens, averaged."""
    if score not in _SCORES:
        raise ValueError(f"unknown score {score!r}")
    return strata_balance_params(_SCORES[score], int(per_rank), weight, z_weight)


def make_route(score: str = "softmax", renormalise: bool = True, scale: float = 1.0, n_group: int = 1,
               topk_group: int = 1, group_score: str = "max") -> strata_route_params:
    """score: "softmax" or "sigmoid"; group_score: "max" or "top2" (read if n_group > 1)."""
    scores = {"softmax": STRATA_SCORE_SOFTMAX, "sigmoid": STRATA_SCORE_SIGMOID}
    groups = {"max": STRATA_GROUP_MAX, "top2": STRATA_GROUP_TOP2}
    if score not in scores or group_score not in groups:
        raise ValueError(f"unknown score {score!r} or group score {group_score!r}")
    return strata_route_params(scores[score], int(renormalise), n_group, topk_group, groups[group_score], scale)


def make_policy(tiers, g0: int = 1, g1: int = 1) -> strata_partition_policy:
    """tiers: list of (alpha, beta, unit_rows, fanout_cap), at most 3."""
    p = strata_partition_policy()
    p.n_tiers, p.g0, p.g1 = len(tiers), g0, g1
    for i, (a, be, ur, cap) in enumerate(tiers):
        p.tiers[i] = strata_tier(a, be, ur, cap, 0)
    return p


class StrataError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = int(code)
        super().__init__(f"{where}: status {self.code} ({strata_status_string(self.code)})")


_lib: Optional[ctypes.CDLL] = None


def lib() -> ctypes.CDLL:
    """The loaded C-ABI library; raises if it has not been built (no fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                           f"`python -m paper_2607_26444_b200.build` (there is no CPU fallback)")
    L = ctypes.CDLL(LIB_PATH)
    vp, sz, i32, u64, i64 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_uint64, ctypes.c_int64
    P = ctypes.POINTER
    L.strata_status_string.restype = ctypes.c_char_p
    L.strata_status_string.argtypes = [i32]
    sigs = {
        "strata_ctx_create": [P(vp), P(strata_moe_shape), i32],
        "strata_ctx_destroy": [vp],
        "strata_moe_workspace_bytes": [P(strata_moe_shape), P(sz)],
        "strata_moe_recv_rows": [P(strata_moe_shape), P(sz)],
        "strata_ctx_set_workspace": [vp, vp, sz],
        "strata_ctx_launch_count": [vp, P(u64)],
        "strata_pool_register": [vp, vp, sz, P(u64)],
        "strata_pool_is_ready": [vp, vp, sz],
        "strata_pool_unregister": [vp, u64],
        "strata_pool_carve": [vp, u64, sz, sz, P(vp)],
        "strata_pool_reset": [vp, u64],
        "strata_moe_layout": [vp, vp, P(strata_moe_layout_t), vp],
        "strata_moe_dispatch": [vp, P(strata_moe_layout_t), vp, vp, vp, sz, vp],
        "strata_moe_combine": [vp, P(strata_moe_layout_t), vp, sz, vp, vp, vp],
        "strata_moe_recv_view": [vp, vp, i32, vp, P(vp), P(ctypes.c_int64)],
        "strata_device_status": [vp, vp, P(i32)],
        "strata_moe_roundtrip_host": [vp, P(strata_moe_device_buffers), vp, vp, vp, vp, vp],
        "strata_moe_layout_noalloc": [P(strata_moe_shape), vp, P(strata_moe_layout_t), vp, vp],
        "strata_ctx_set_trace": [vp, vp, sz],
        "strata_moe_partition_max_units": [P(strata_moe_shape), P(strata_partition_policy), P(sz)],
        "strata_moe_partition": [vp, P(strata_moe_layout_t), P(strata_partition_policy), i32,
                                 P(strata_partition_t), sz, vp],
        "strata_moe_dispatch_windows": [vp, P(strata_moe_layout_t), P(strata_partition_t), i32, vp, vp, sz, vp],
        "strata_ctx_set_sm_budget": [vp, i32],
        "strata_ctx_set_x_early": [vp, i32],
        "strata_moe_row_experts": [vp, P(strata_moe_layout_t), vp, sz, vp],
        "strata_moe_mask_ragged": [vp, vp, vp, vp],
        "strata_moe_expert_affine_inplace": [vp, P(strata_moe_layout_t), vp, sz, vp, vp, i32, vp],
        "strata_ctx_set_timeline": [vp, vp, sz, sz],
        "strata_timeline_decode": [vp, sz, sz, vp, sz, P(sz), P(sz)],
        "strata_allgather": [vp, i32, vp, vp, sz, vp],
        "strata_alltoall": [vp, i32, vp, vp, sz, vp],
        "strata_broadcast": [vp, i32, i32, vp, vp, sz, vp],
        "strata_p2p": [vp, i32, i32, i32, vp, vp, sz, vp],
        "strata_alltoallv": [vp, i32, vp, sz, vp, sz, vp, vp, vp, vp],
        "strata_reducescatter": [vp, i32, vp, vp, sz, vp],
        "strata_allreduce": [vp, i32, vp, vp, sz, vp],
        "strata_moe_route": [vp, P(strata_route_params), vp, i32, i64, vp, vp, vp, vp],
        "strata_moe_route_grad": [vp, P(strata_route_params), vp, i32, i64, vp, vp, vp, i64, vp],
        "strata_norm": [vp, P(strata_norm_args), vp],
        "strata_norm_grad_scratch_bytes": [vp, i64, i32, P(sz)],
        "strata_norm_grad": [vp, P(strata_norm_grad_args), vp],
        "strata_quantize_rows": [vp, vp, i64, i64, i32, i32, vp, i64, vp, i64, vp, vp],
        "strata_moe_expert_matmul": [vp, P(strata_moe_layout_t), P(strata_matmul_args), vp],
        "strata_quantize_rows4": [vp, vp, i64, i64, i32, i32, P(strata_rows4), vp, vp],
        "strata_dequantize_rows4": [vp, P(strata_rows4), i64, i32, i32, vp, i32, i64, vp, vp],
        "strata_moe_expert_matmul4": [vp, P(strata_moe_layout_t), P(strata_matmul4_args), vp],
        "strata_moe_balance_scratch_bytes": [vp, P(strata_balance_params), P(sz)],
        "strata_moe_balance_loss": [vp, P(strata_balance_params), vp, i32, i64, vp, vp, P(strata_balance_stats), vp, sz, vp],
        "strata_moe_balance_grad": [vp, P(strata_balance_params), vp, i32, i64, vp, P(strata_balance_stats), vp, vp, i64, vp,
                                    i64, vp],
    }
    for name, args in sigs.items():
        fn = getattr(L, name)
        fn.restype = i32
        fn.argtypes = args
    _lib = L
    return L


# ---- one Python function per C entry point (same names, raw pointers) -------

def strata_status_string(code: int) -> str:
    return lib().strata_status_string(int(code)).decode()


def strata_ctx_create(shape: strata_moe_shape, device: int) -> Tuple[int, Optional[int]]:
    h = ctypes.c_void_p()
    rc = lib().strata_ctx_create(ctypes.byref(h), ctypes.byref(shape), device)
    return rc, h.value


def strata_ctx_destroy(ctx) -> int:
    return lib().strata_ctx_destroy(ctx)


def strata_moe_workspace_bytes(shape: strata_moe_shape) -> Tuple[int, int]:
    n = ctypes.c_size_t()
    rc = lib().strata_moe_workspace_bytes(ctypes.byref(shape), ctypes.byref(n))
    return rc, n.value


def strata_moe_recv_rows(shape: strata_moe_shape) -> Tuple[int, int]:
    n = ctypes.c_size_t()
    rc = lib().strata_moe_recv_rows(ctypes.byref(shape), ctypes.byref(n))
    return rc, n.value


def strata_ctx_set_workspace(ctx, dptr: int, nbytes: int) -> int:
    return lib().strata_ctx_set_workspace(ctx, dptr, nbytes)


def strata_ctx_set_trace(ctx, dptr: Optional[int], capacity_ctas: int) -> int:
    return lib().strata_ctx_set_trace(ctx, dptr, capacity_ctas)


def strata_ctx_launch_count(ctx) -> Tuple[int, int]:
    n = ctypes.c_uint64()
    rc = lib().strata_ctx_launch_count(ctx, ctypes.byref(n))
    return rc, n.value


def strata_pool_register(ctx, dbase: int, nbytes: int) -> Tuple[int, int]:
    rid = ctypes.c_uint64()
    rc = lib().strata_pool_register(ctx, dbase, nbytes, ctypes.byref(rid))
    return rc, rid.value


def strata_pool_is_ready(ctx, dptr: int, nbytes: int) -> int:
    return lib().strata_pool_is_ready(ctx, dptr, nbytes)


def strata_pool_unregister(ctx, region_id: int) -> int:
    return lib().strata_pool_unregister(ctx, region_id)


def strata_pool_carve(ctx, region_id: int, nbytes: int, align: int) -> Tuple[int, Optional[int]]:
    p = ctypes.c_void_p()
    rc = lib().strata_pool_carve(ctx, region_id, nbytes, align, ctypes.byref(p))
    return rc, p.value


def strata_pool_reset(ctx, region_id: int) -> int:
    return lib().strata_pool_reset(ctx, region_id)


def strata_moe_layout(ctx, topk_ids: int, layout: strata_moe_layout_t, stream: int) -> int:
    return lib().strata_moe_layout(ctx, topk_ids, ctypes.byref(layout), stream)


def strata_moe_dispatch(ctx, layout: strata_moe_layout_t, x: int, recv: int, recv_scale: Optional[int],
                        capacity_rows: int, stream: int) -> int:
    return lib().strata_moe_dispatch(ctx, ctypes.byref(layout), x, recv, recv_scale, capacity_rows, stream)


def strata_moe_combine(ctx, layout: strata_moe_layout_t, y: int, y_rows: int, topk_w: int, out: int,
                       stream: int) -> int:
    return lib().strata_moe_combine(ctx, ctypes.byref(layout), y, y_rows, topk_w, out, stream)


def strata_moe_recv_view(ctx, h_rank_offset, rank: int, recv: int) -> Tuple[int, Optional[int], int]:
    """h_rank_offset: a host numpy int32 array [R+1]."""
    base, rows = ctypes.c_void_p(), ctypes.c_int64()
    rc = lib().strata_moe_recv_view(ctx, h_rank_offset.ctypes.data, rank, recv, ctypes.byref(base),
                                    ctypes.byref(rows))
    return rc, base.value, rows.value


def strata_device_status(ctx, stream: int) -> Tuple[int, int]:
    out = ctypes.c_int()
    rc = lib().strata_device_status(ctx, stream, ctypes.byref(out))
    return rc, out.value


def strata_moe_roundtrip_host(ctx, dev: strata_moe_device_buffers, h_ids: int, h_x: int, h_w: int, h_out: int,
                              stream: int) -> int:
    return lib().strata_moe_roundtrip_host(ctx, ctypes.byref(dev), h_ids, h_x, h_w, h_out, stream)


def strata_moe_layout_noalloc(shape: strata_moe_shape, topk_ids: int, layout: strata_moe_layout_t,
                              device_status: Optional[int], stream: int) -> int:
    """Routing layout on the current device with the library's built-in scratch: no context, no
    workspace, nothing allocated.  For callers that cannot allocate device memory (see the header)."""
    return lib().strata_moe_layout_noalloc(ctypes.byref(shape), topk_ids, ctypes.byref(layout), device_status,
                                           stream)


def strata_moe_partition_max_units(shape: strata_moe_shape, policy: strata_partition_policy) -> Tuple[int, int]:
    n = ctypes.c_size_t()
    rc = lib().strata_moe_partition_max_units(ctypes.byref(shape), ctypes.byref(policy), ctypes.byref(n))
    return rc, n.value


def strata_moe_partition(ctx, layout: strata_moe_layout_t, policy: strata_partition_policy, n_cores: int,
                         out: strata_partition_t, max_units: int, stream: int) -> int:
    return lib().strata_moe_partition(ctx, ctypes.byref(layout), ctypes.byref(policy), n_cores, ctypes.byref(out),
                                      max_units, stream)


def strata_moe_dispatch_windows(ctx, layout: strata_moe_layout_t, partition: strata_partition_t, n_cores: int,
                                x: int, recv: int, capacity_rows: int, stream: int) -> int:
    return lib().strata_moe_dispatch_windows(ctx, ctypes.byref(layout), ctypes.byref(partition), n_cores, x, recv,
                                             capacity_rows, stream)


def strata_moe_row_experts(ctx, layout: strata_moe_layout_t, row_expert: int, capacity_rows: int, stream: int) -> int:
    return lib().strata_moe_row_experts(ctx, ctypes.byref(layout), row_expert, capacity_rows, stream)


def strata_moe_mask_ragged(ctx, tokens_per_rank: int, topk_ids: int, stream: int) -> int:
    return lib().strata_moe_mask_ragged(ctx, tokens_per_rank, topk_ids, stream)


def strata_moe_expert_affine_inplace(ctx, layout: strata_moe_layout_t, recv: int, capacity_rows: int, scale: int,
                                     bias: int, tile_rows: int, stream: int) -> int:
    return lib().strata_moe_expert_affine_inplace(ctx, ctypes.byref(layout), recv, capacity_rows, scale, bias,
                                                  tile_rows, stream)


def strata_ctx_set_x_early(ctx, on: int) -> int:
    return lib().strata_ctx_set_x_early(ctx, int(on))


def strata_ctx_set_sm_budget(ctx, n_sm: int) -> int:
    return lib().strata_ctx_set_sm_budget(ctx, n_sm)


def strata_ctx_set_timeline(ctx, buf: Optional[int], n_ctas: int, events_per_cta: int) -> int:
    return lib().strata_ctx_set_timeline(ctx, buf, n_ctas, events_per_cta)


def strata_timeline_decode(host_buf: int, n_ctas: int, events_per_cta: int, spans: Optional[int],
                           max_spans: int) -> Tuple[int, int, int]:
    """Returns (status, spans found, events dropped); host_buf and spans are host addresses."""
    n, lost = ctypes.c_size_t(), ctypes.c_size_t()
    rc = lib().strata_timeline_decode(host_buf, n_ctas, events_per_cta, spans, max_spans, ctypes.byref(n),
                                      ctypes.byref(lost))
    return rc, n.value, lost.value


def strata_allgather(ctx, R: int, src: int, dst: int, bytes_per_rank: int, stream: int) -> int:
    return lib().strata_allgather(ctx, R, src, dst, bytes_per_rank, stream)


def strata_alltoall(ctx, R: int, src: int, dst: int, bytes_per_slice: int, stream: int) -> int:
    return lib().strata_alltoall(ctx, R, src, dst, bytes_per_slice, stream)


def strata_broadcast(ctx, R: int, root: int, src: int, dst: int, nbytes: int, stream: int) -> int:
    return lib().strata_broadcast(ctx, R, root, src, dst, nbytes, stream)


def strata_p2p(ctx, R: int, src_rank: int, dst_rank: int, src: int, dst: int, nbytes: int, stream: int) -> int:
    return lib().strata_p2p(ctx, R, src_rank, dst_rank, src, dst, nbytes, stream)


def strata_alltoallv(ctx, R: int, src: int, in_stride: int, dst: int, out_stride: int, send_bytes: int,
                     send_offset: int, recv_offset: int, stream: int) -> int:
    return lib().strata_alltoallv(ctx, R, src, in_stride, dst, out_stride, send_bytes, send_offset, recv_offset, stream)


def strata_reducescatter(ctx, R: int, src: int, dst: int, elems_per_slice: int, stream: int) -> int:
    return lib().strata_reducescatter(ctx, R, src, dst, elems_per_slice, stream)


def strata_allreduce(ctx, R: int, src: int, dst: int, elems: int, stream: int) -> int:
    return lib().strata_allreduce(ctx, R, src, dst, elems, stream)


def strata_moe_route(ctx, params: strata_route_params, logits: int, logits_type: int, logits_stride: int,
                     bias: Optional[int], topk_ids: int, topk_w: int, stream: int) -> int:
    return lib().strata_moe_route(ctx, ctypes.byref(params), logits, logits_type, logits_stride, bias, topk_ids, topk_w,
                                  stream)


def strata_moe_route_grad(ctx, params: strata_route_params, logits: int, logits_type: int, logits_stride: int,
                          topk_ids: int, dtopk_w: int, dlogits: int, dlogits_stride: int, stream: int) -> int:
    return lib().strata_moe_route_grad(ctx, ctypes.byref(params), logits, logits_type, logits_stride, topk_ids, dtopk_w,
                                       dlogits, dlogits_stride, stream)


def strata_norm(ctx, args: strata_norm_args, stream: int) -> int:
    return lib().strata_norm(ctx, ctypes.byref(args), stream)


def strata_norm_grad_scratch_bytes(ctx, rows: int, cols: int) -> Tuple[int, int]:
    n = ctypes.c_size_t()
    rc = lib().strata_norm_grad_scratch_bytes(ctx, rows, cols, ctypes.byref(n))
    return rc, n.value


def strata_norm_grad(ctx, args: strata_norm_grad_args, stream: int) -> int:
    return lib().strata_norm_grad(ctx, ctypes.byref(args), stream)


def strata_quantize_rows(ctx, x: int, x_stride: int, rows: int, cols: int, q_type: int, q: int, q_stride: int,
                         q_scale: int, q_scale_stride: int, n_valid: Optional[int], stream: int) -> int:
    return lib().strata_quantize_rows(ctx, x, x_stride, rows, cols, q_type, q, q_stride, q_scale, q_scale_stride,
                                      n_valid, stream)


def strata_moe_expert_matmul(ctx, layout: strata_moe_layout_t, args: strata_matmul_args, stream: int) -> int:
    return lib().strata_moe_expert_matmul(ctx, ctypes.byref(layout), ctypes.byref(args), stream)


def strata_quantize_rows4(ctx, x: int, x_stride: int, rows: int, cols: int, type_: int, q: strata_rows4,
                          n_valid: Optional[int], stream: int) -> int:
    return lib().strata_quantize_rows4(ctx, x, x_stride, rows, cols, type_, ctypes.byref(q), n_valid, stream)


def strata_dequantize_rows4(ctx, q: strata_rows4, rows: int, cols: int, type_: int, out: int, out_type: int,
                            out_stride: int, n_valid: Optional[int], stream: int) -> int:
    return lib().strata_dequantize_rows4(ctx, ctypes.byref(q), rows, cols, type_, out, out_type, out_stride, n_valid,
                                         stream)


def strata_moe_expert_matmul4(ctx, layout: strata_moe_layout_t, args: strata_matmul4_args, stream: int) -> int:
    return lib().strata_moe_expert_matmul4(ctx, ctypes.byref(layout), ctypes.byref(args), stream)


def strata_moe_balance_scratch_bytes(ctx, params: strata_balance_params) -> Tuple[int, int]:
    n = ctypes.c_size_t()
    rc = lib().strata_moe_balance_scratch_bytes(ctx, ctypes.byref(params), ctypes.byref(n))
    return rc, n.value


def strata_moe_balance_loss(ctx, params: strata_balance_params, logits: int, logits_type: int, logits_stride: int,
                            topk_ids: int, loss: int, stats: strata_balance_stats, scratch: int, scratch_bytes: int,
                            stream: int) -> int:
    return lib().strata_moe_balance_loss(ctx, ctypes.byref(params), logits, logits_type, logits_stride, topk_ids, loss,
                                         ctypes.byref(stats), scratch, scratch_bytes, stream)


def strata_moe_balance_grad(ctx, params: strata_balance_params, logits: int, logits_type: int, logits_stride: int,
                            topk_ids: int, stats: strata_balance_stats, dloss: Optional[int], add: Optional[int],
                            add_stride: int, dlogits: int, dlogits_stride: int, stream: int) -> int:
    return lib().strata_moe_balance_grad(ctx, ctypes.byref(params), logits, logits_type, logits_stride, topk_ids,
                                         ctypes.byref(stats), dloss, add, add_stride, dlogits, dlogits_stride, stream)


# ---- convenience wrapper over torch tensors (memory + streams only) ---------

def _check(rc: int, where: str) -> None:
    if rc != STRATA_OK:
        raise StrataError(rc, where)


def _strides(t):
    """(rows, columns, row stride in elements) of a tensor [..., columns] whose rows are evenly spaced."""
    cols = t.size(-1)
    if t.is_contiguous():
        return (t.numel() // cols if cols else 0), cols, cols
    if t.dim() == 2 and t.stride(1) == 1:
        return t.size(0), cols, (t.stride(0) if t.size(0) > 1 else cols)
    stride, rows = cols, 1
    for d in range(t.dim() - 2, -1, -1):
        if t.shape[d] > 1:
            if rows == 1:
                stride = t.stride(d)
            elif t.stride(d) != rows * stride:
                raise ValueError("rows are not evenly spaced: pass a contiguous tensor")
        rows *= t.shape[d]
    if t.stride(-1) != 1 and cols > 1:
        raise ValueError("the last dimension is not contiguous")
    return rows, cols, stride


def _stride(t, rows: int, cols: int, what: str) -> int:
    """Row stride of a tensor that must hold rows x cols."""
    if t.is_contiguous() and t.numel() == rows * cols and t.size(-1) == cols:
        return cols
    r, c, stride = _strides(t)
    if r != rows or c != cols:
        raise ValueError(f"{what}: {rows} rows of {cols} are needed, not {r} of {c}")
    return stride


def _scale_stride(t, rows: int) -> int:
    """Distance of a row's scale to the next one's, for at least `rows` fp32 scales that each have a place of their own."""
    n = t.numel()
    if _types[t.dtype] != STRATA_T_F32:
        raise ValueError(f"scales are fp32, not {t.dtype}")
    if n < rows:
        raise ValueError("one scale per row is needed")
    if t.dim() == 1:
        stride = t.stride(0)
    elif t.is_contiguous():
        stride = 1                                        # a last dimension of one element may have any stride of its own
    else:
        stride = _strides(t[..., None])[2]
    if stride == 0 and rows > 1:
        raise ValueError("one scale broadcast to all rows (stride 0): pass a tensor that holds one per row")
    return max(1, stride)


_INT32 = -2                          # expert ids: no operand type of the library


class _Types(dict):
    """Element types by torch dtype, filled on first use (torch is imported by the callers that need it)."""

    def __missing__(self, dtype):
        import torch
        self.update({torch.float32: STRATA_T_F32, torch.bfloat16: STRATA_T_BF16, torch.int16: STRATA_T_BF16,
                     torch.int8: STRATA_T_INT8, torch.float8_e4m3fn: STRATA_T_E4M3, torch.int32: _INT32})
        return self.setdefault(dtype, -1)


_types = _Types()


def _code_type(t) -> int:
    code = _types[t.dtype]
    if code != STRATA_T_INT8 and code != STRATA_T_E4M3:
        raise ValueError(f"8-bit codes are torch.int8 or torch.float8_e4m3fn, not {t.dtype}")
    return code


def _float_type(t) -> int:
    """bf16 (also as 16-bit patterns) or fp32."""
    code = _types[t.dtype]
    if code != STRATA_T_BF16 and code != STRATA_T_F32:
        raise ValueError(f"bf16 or fp32 is needed, not {t.dtype}")
    return code


def _bf16(t) -> int:
    """Address of a bf16 tensor (also as 16-bit patterns)."""
    if _types[t.dtype] != STRATA_T_BF16:
        raise ValueError(f"bf16 is needed, not {t.dtype}")
    return t.data_ptr()


_NAMES = {STRATA_T_BF16: "bf16", STRATA_T_F32: "fp32", STRATA_T_INT8: "int8", STRATA_T_E4M3: "e4m3", _INT32: "int32"}


def _flat(t, code: int, n: int, what: str) -> int:
    """Address of a contiguous tensor of n elements of type `code`."""
    if t.numel() != n or not t.is_contiguous() or _types[t.dtype] != code:
        raise ValueError(f"{what}: {n} contiguous {_NAMES[code]} elements are needed")
    return t.data_ptr()


def q8_rows(buf, code_dtype):
    """The two views of a uint8 buffer [..., H + STRATA_Q8_TRAILER] of STRATA_Q8_ROW rows: codes [..., H] of code_dtype
    and scales [...] (float)."""
    import torch
    h = buf.shape[-1] - STRATA_Q8_TRAILER
    scale = buf.view(torch.float32)[..., h // 4]
    return buf[..., :h].view(code_dtype), scale


_BLOCK4 = {STRATA_T_MXF4: 32, STRATA_T_NVF4: 16}          # values that share a scale
_KINDS4 = {"mxfp4": STRATA_T_MXF4, "nvfp4": STRATA_T_NVF4}


def _kind4(kind: str) -> int:
    if kind not in _KINDS4:
        raise ValueError(f"4-bit rows are mxfp4 or nvfp4, not {kind!r}")
    return _KINDS4[kind]


class _Blocks4(dict):
    """(type, values per scale) by the torch dtype of block scales, filled on first use."""

    def __missing__(self, dtype):
        import torch
        self.update({torch.float8_e8m0fnu: (STRATA_T_MXF4, 32), torch.float8_e4m3fn: (STRATA_T_NVF4, 16)})
        _codes4.update((torch.uint8, torch.float4_e2m1fn_x2))
        if dtype not in self:
            raise ValueError(f"block scales are torch.float8_e8m0fnu or torch.float8_e4m3fn, not {dtype}")
        return self[dtype]


_blocks4 = _Blocks4()
_codes4 = set()


class Rows4:
    """Rows in 4 bits: codes uint8 (or torch.float4_e2m1fn_x2) [.., cols / 2], two to a byte and the first in its low half;
    block scales [.., cols / 32] of torch.float8_e8m0fnu (mxfp4) or [.., cols / 16] of torch.float8_e4m3fn (nvfp4); scales
    of the rows fp32 [..] or None (1).  Rows of codes and of block scales start on 16 bytes."""

    def __init__(self, codes, block, scale=None):
        self.type, per = _blocks4[block.dtype]
        if codes.dtype not in _codes4:
            raise ValueError(f"4-bit codes are torch.uint8 or torch.float4_e2m1fn_x2, not {codes.dtype}")
        self.codes, self.block, self.scale = codes, block, scale
        if codes.is_contiguous():
            code_stride = codes.size(-1)
            rows = codes.numel() // code_stride if code_stride else 0
            cols = 2 * code_stride
        else:
            rows, half, code_stride = _strides(codes)
            cols = 2 * half
        if cols % 32:
            raise ValueError("4-bit rows have a multiple of 32 columns")
        block_stride = _stride(block, rows, cols // per, "block scales")
        if rows == 1:                                     # nothing is read between rows that are not there
            code_stride, block_stride = -(-code_stride // 16) * 16, -(-block_stride // 16) * 16
        self.rows, self.cols = rows, cols
        if scale is None:
            self.c = strata_rows4(codes.data_ptr(), block.data_ptr(), None, code_stride, block_stride, 0)
        else:
            self.c = strata_rows4(codes.data_ptr(), block.data_ptr(), scale.data_ptr(), code_stride, block_stride,
                                  _scale_stride(scale, rows))


def empty_rows4(shape, cols: int, kind: str, device="cuda") -> Rows4:
    """Uninitialised 4-bit rows [*shape, cols] of kind "mxfp4" or "nvfp4", as quantize_rows4 writes them."""
    import torch
    code = _kind4(kind)
    n = cols // _BLOCK4[code]
    block = torch.empty((*shape, -(-n // 16) * 16), dtype=torch.uint8, device=device)
    block = block.view(torch.float8_e8m0fnu if code == STRATA_T_MXF4 else torch.float8_e4m3fn)[..., :n]
    scale = torch.empty(shape, dtype=torch.float32, device=device) if code == STRATA_T_NVF4 else None
    return Rows4(torch.empty((*shape, cols // 2), dtype=torch.uint8, device=device), block, scale)


def row4_bytes(cols: int, kind: str) -> int:
    """Bytes of a row of dispatch type STRATA_MXF4_ROW or STRATA_NVF4_ROW."""
    if _kind4(kind) == STRATA_T_MXF4:
        return (cols // 2 + cols // 32 + 31) // 32 * 32
    return ((cols // 2 + cols // 16 + 15) // 16 * 16 + 4 + 31) // 32 * 32


def q4_rows(buf, cols: int, kind: str) -> Rows4:
    """The 4-bit rows in a uint8 buffer [.., row4_bytes(cols, kind)] of STRATA_MXF4_ROW or STRATA_NVF4_ROW rows."""
    import torch
    if buf.shape[-1] != row4_bytes(cols, kind):
        raise ValueError(f"rows of {row4_bytes(cols, kind)} bytes are needed, not of {buf.shape[-1]}")
    half, n = cols // 2, cols // _BLOCK4[_kind4(kind)]
    block = buf[..., half:half + n]
    if kind == "mxfp4":
        return Rows4(buf[..., :half], block.view(torch.float8_e8m0fnu))
    return Rows4(buf[..., :half], block.view(torch.float8_e4m3fn), buf.view(torch.float32)[..., (half + n + 15) // 16 * 4])


class BalanceStats:
    """What balance_loss leaves for its gradient and for the books: count int32 and prob fp32 [groups, E], tokens int32
    [groups]; and its scratch."""

    def __init__(self, groups: int, E: int, scratch_bytes: int, device):
        import torch
        self.count = torch.empty((groups, E), dtype=torch.int32, device=device)
        self.tokens = torch.empty(groups, dtype=torch.int32, device=device)
        self.prob = torch.empty((groups, E), dtype=torch.float32, device=device)
        self.scratch = torch.empty(scratch_bytes, dtype=torch.uint8, device=device)
        self.groups, self.E = groups, E
        self.c = strata_balance_stats(self.count.data_ptr(), self.tokens.data_ptr(), self.prob.data_ptr())


class Layout:
    """Device tensors holding the routing metadata, plus the C struct pointing at them."""

    def __init__(self, R: int, T: int, K: int, E: int, device, with_optional: bool = True,
                 recv_rows: Optional[int] = None):
        import torch
        i32 = dict(dtype=torch.int32, device=device)
        self.expert_count = torch.empty(E, **i32)
        self.expert_offset = torch.empty(E + 1, **i32)
        self.rank_count = torch.empty(R, **i32)
        self.rank_offset = torch.empty(R + 1, **i32)
        self.src_expert_count = torch.empty((R, E), **i32) if with_optional else None
        self.dst_row = torch.empty((R, T, K), **i32)
        self.src_of_row = torch.empty(recv_rows or R * T * K, **i32) if with_optional else None
        self.c = strata_moe_layout_t(
            self.expert_count.data_ptr(), self.expert_offset.data_ptr(), self.rank_count.data_ptr(),
            self.rank_offset.data_ptr(),
            self.src_expert_count.data_ptr() if with_optional else None,
            self.dst_row.data_ptr(),
            self.src_of_row.data_ptr() if with_optional else None)


class Partition:
    """Device tensors of a window-partitioning policy, plus the C struct pointing at them."""

    def __init__(self, R: int, E: int, n_cores: int, max_units: int, device):
        import torch
        i32 = dict(dtype=torch.int32, device=device)
        i64 = dict(dtype=torch.int64, device=device)
        self.n_cores, self.max_units = n_cores, max_units
        self.win_base = torch.zeros((R, E), **i32)
        self.unit_desc = torch.zeros((max_units, 4), **i32)
        self.unit_cost = torch.zeros(max_units, **i64)
        self.n_units = torch.zeros(1, **i32)
        self.task_offset = torch.zeros(n_cores + 1, **i32)
        self.task_unit = torch.zeros(max_units, **i32)
        self.core_load = torch.zeros(n_cores, **i64)
        self.scratch = torch.zeros(max_units * (R + 2), **i32)
        self.task_stripe = torch.zeros(max_units, **i32)
        self.c = strata_partition_t(self.win_base.data_ptr(), self.unit_desc.data_ptr(), self.unit_cost.data_ptr(),
                                    self.n_units.data_ptr(), self.task_offset.data_ptr(), self.task_unit.data_ptr(),
                                    self.core_load.data_ptr(), self.scratch.data_ptr(), self.task_stripe.data_ptr())


class MoEContext:
    """One shape on one GPU.  Owns a strata_ctx and its workspace tensor."""

    def __init__(self, R: int, T: int, H: int, E: int, K: int, dispatch_dtype: int = STRATA_BF16,
                 device: int = 0, segment_align: int = 0, allow_unrouted: bool = False,
                 slot_capacity: int = 0):
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("MoEContext needs a CUDA device (there is no CPU fallback)")
        self.shape = strata_moe_shape(R, T, H, E, K, dispatch_dtype, segment_align,
                                      STRATA_FLAG_ALLOW_UNROUTED if allow_unrouted else 0, slot_capacity)
        self.R, self.T, self.H, self.E, self.K = R, T, H, E, K
        self.fp8 = dispatch_dtype == STRATA_FP8_E4M3_B128
        self.n_tok, self.n_items = R * T, R * T * K
        self.device = torch.device("cuda", device)
        self._c = lib()
        self._norm = self._c._FuncPtr(("strata_norm", self._c))          # takes its arguments packed (_NORM_ARGS)
        self._norm.restype, self._norm.argtypes = ctypes.c_int, [ctypes.c_void_p, ctypes.c_char_p, ctypes.c_void_p]
        self._raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda index: torch.cuda.current_stream(index).cuda_stream)
        rc, h = strata_ctx_create(self.shape, device)
        _check(rc, "strata_ctx_create")
        self.h = h
        rc, self.recv_rows = strata_moe_recv_rows(self.shape)     # rows a receive buffer must hold
        _check(rc, "strata_moe_recv_rows")
        rc, nbytes = strata_moe_workspace_bytes(self.shape)
        _check(rc, "strata_moe_workspace_bytes")
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        _check(strata_ctx_set_workspace(self.h, self.workspace.data_ptr(), nbytes), "strata_ctx_set_workspace")
        self._regions = {}

    def close(self) -> None:
        if getattr(self, "h", None):
            strata_ctx_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _stream(self) -> int:
        """The current stream of the context's device (the raw handle: building a Stream object costs a microsecond)."""
        return self._raw_stream(self.device.index)

    # pool -----------------------------------------------------------------
    def register(self, tensor) -> int:
        rc, rid = strata_pool_register(self.h, tensor.data_ptr(), tensor.numel() * tensor.element_size())
        _check(rc, "strata_pool_register")
        self._regions[rid] = tensor          # keep the allocation alive while registered
        return rid

    def unregister(self, rid: int) -> None:
        _check(strata_pool_unregister(self.h, rid), "strata_pool_unregister")
        self._regions.pop(rid, None)

    def carve(self, rid: int, shape, dtype, align: int = 256):
        """A tensor view of a sub-range carved from a registered region (zero copy)."""
        import torch
        base = self._regions[rid]
        n = 1
        for d in shape:
            n *= int(d)
        nbytes = n * torch.empty((), dtype=dtype).element_size()
        rc, p = strata_pool_carve(self.h, rid, nbytes, align)
        _check(rc, "strata_pool_carve")
        off = p - base.data_ptr()
        return base.view(torch.uint8).reshape(-1)[off:off + nbytes].view(dtype).reshape(*shape)

    def new_layout(self, with_optional: bool = True) -> Layout:
        return Layout(self.R, self.T, self.K, self.E, self.device, with_optional, self.recv_rows)

    # hot path ---------------------------------------------------------------
    def layout(self, ids, layout: Optional[Layout] = None) -> Layout:
        layout = layout or self.new_layout()
        _check(strata_moe_layout(self.h, ids.data_ptr(), layout.c, self._stream()), "strata_moe_layout")
        return layout

    def dispatch(self, layout: Layout, x, recv, recv_scale=None) -> None:
        _check(strata_moe_dispatch(self.h, layout.c, x.data_ptr(), recv.data_ptr(),
                                   recv_scale.data_ptr() if recv_scale is not None else None,
                                   recv.shape[0], self._stream()), "strata_moe_dispatch")

    def combine(self, layout: Layout, y, w, out) -> None:
        _check(strata_moe_combine(self.h, layout.c, y.data_ptr(), y.shape[0], w.data_ptr(), out.data_ptr(),
                                  self._stream()), "strata_moe_combine")

    def mask_ragged(self, tokens_per_rank, ids) -> None:
        """Marks, in place, the slots of the tokens t >= tokens_per_rank[r] as not routed (-1)."""
        _check(strata_moe_mask_ragged(self.h, tokens_per_rank.data_ptr(), ids.data_ptr(), self._stream()),
               "strata_moe_mask_ragged")

    def expert_affine_inplace(self, layout: Layout, recv, scale, bias, tile_rows: int = 1) -> None:
        """recv[row] = bf16(fma(recv[row], scale[e], bias[e])) for every occupied row, in place, tile by tile."""
        _check(strata_moe_expert_affine_inplace(self.h, layout.c, recv.data_ptr(), recv.shape[0], scale.data_ptr(),
                                                bias.data_ptr(), tile_rows, self._stream()),
               "strata_moe_expert_affine_inplace")

    # the layer around the routing path ------------------------------------------------------------
    def route(self, params: strata_route_params, logits, ids, w, bias=None) -> None:
        """Router logits [.., E] (bf16 or fp32) -> ids int32 [.., K] and gate weights fp32 [.., K]; bias fp32 [E] takes part
        in the choice only."""
        n = self.n_items
        _check(self._c.strata_moe_route(
            self.h, params, logits.data_ptr(), _float_type(logits), _stride(logits, self.n_tok, self.E, "logits"),
            None if bias is None else _flat(bias, STRATA_T_F32, self.E, "bias"), _flat(ids, _INT32, n, "ids"),
            _flat(w, STRATA_T_F32, n, "w"),
            self._stream()), "strata_moe_route")

    def route_grad(self, params: strata_route_params, logits, ids, dw, dlogits) -> None:
        """Gradient of the logits (in their type) from the gradient dw [.., K] of the gate weights."""
        n = self.n_items
        if dlogits.dtype != logits.dtype:
            raise ValueError("dlogits has the type of logits")
        _check(self._c.strata_moe_route_grad(
            self.h, params, logits.data_ptr(), _float_type(logits), _stride(logits, self.n_tok, self.E, "logits"),
            _flat(ids, _INT32, n, "ids"), _flat(dw, STRATA_T_F32, n, "dw"), dlogits.data_ptr(),
            _stride(dlogits, self.n_tok, self.E, "dlogits"), self._stream()), "strata_moe_route_grad")

    def norm(self, x, weight, eps: float, out=None, residual=None, residual_out=None, q=None, q_scale=None) -> None:
        """h = x + residual (stored in residual_out), then h * rsqrt(mean(h^2) + eps) * weight to `out` (bf16) and / or
        to 8-bit codes `q` (torch.int8 or torch.float8_e4m3fn) with one fp32 scale per row."""
        cols, dtype, n = weight.numel(), x.dtype, x.numel()
        if _types[dtype] != STRATA_T_BF16 or x.size(-1) != cols or cols == 0:
            raise ValueError("x is bf16 [.., cols] and weight [cols]")
        rows = n // cols
        x_stride = r_stride = h_stride = o_stride = cols
        if not x.is_contiguous():
            x_stride = _strides(x)[2]
        rp = hp = op = qp = sp = q_stride = s_stride = q_type = 0
        if (residual is None) != (residual_out is None):
            raise ValueError("residual and residual_out come together")
        if (q is None) != (q_scale is None):
            raise ValueError("q comes with q_scale")
        if residual is not None:
            rp, hp = residual.data_ptr(), residual_out.data_ptr()
            if not (residual.numel() == n and residual.is_contiguous() and residual.size(-1) == cols and residual.dtype == dtype):
                rp, r_stride = _bf16(residual), _stride(residual, rows, cols, "residual")
            if not (residual_out.numel() == n and residual_out.is_contiguous() and residual_out.size(-1) == cols
                    and residual_out.dtype == dtype):
                hp, h_stride = _bf16(residual_out), _stride(residual_out, rows, cols, "residual_out")
        if out is not None:
            op = out.data_ptr()
            if not (out.numel() == n and out.is_contiguous() and out.size(-1) == cols and out.dtype == dtype):
                op, o_stride = _bf16(out), _stride(out, rows, cols, "out")
        if q is not None:
            qp, q_type, q_stride = q.data_ptr(), _code_type(q), _stride(q, rows, cols, "q")
            sp, s_stride = q_scale.data_ptr(), _scale_stride(q_scale, rows)
        wt = _float_type(weight)
        if not weight.is_contiguous():
            raise ValueError("weight is contiguous")
        rc = self._norm(self.h, _NORM_ARGS.pack(
            rows, cols, wt, eps, q_type, x.data_ptr(), rp, weight.data_ptr(), hp, op, qp, sp, x_stride, r_stride, h_stride,
            o_stride, q_stride, s_stride), self._raw_stream(self.device.index))
        if rc:
            _check(rc, "strata_norm")

    def norm_grad_scratch(self, rows: int, cols: int):
        """Scratch of norm_grad for this many rows and columns."""
        import torch
        rc, n = strata_norm_grad_scratch_bytes(self.h, rows, cols)
        _check(rc, "strata_norm_grad_scratch_bytes")
        return torch.empty(max(n, 16), dtype=torch.uint8, device=self.device)

    def norm_grad(self, dy, h, weight, eps: float, dx, dweight, dresidual=None, scratch=None) -> None:
        """Gradients of norm's bf16 output: dx (of x and of residual alike, dresidual added) and dweight (fp32 [cols])."""
        rows, cols, dy_stride = _strides(dy)
        rp = r_stride = 0
        if dresidual is not None:
            rp, r_stride = _bf16(dresidual), _stride(dresidual, rows, cols, "dresidual")
        if scratch is None:
            scratch = self.norm_grad_scratch(rows, cols)
        wt = _float_type(weight)
        _check(self._c.strata_norm_grad(self.h, strata_norm_grad_args(
            rows, cols, wt, eps, 0, _bf16(dy), _bf16(h), _flat(weight, wt, cols, "weight"), rp,
            _bf16(dx), _flat(dweight, STRATA_T_F32, cols, "dweight"), scratch.data_ptr(), scratch.nbytes, dy_stride,
            _stride(h, rows, cols, "h"), r_stride, _stride(dx, rows, cols, "dx")), self._stream()), "strata_norm_grad")

    def quantize_rows(self, x, q, q_scale, layout: Optional[Layout] = None) -> None:
        """bf16 rows -> 8-bit codes with one fp32 scale per row; with a layout, only the rows it has in use."""
        rows, cols, stride = _strides(x)
        n_valid = layout.expert_offset.data_ptr() + 4 * self.E if layout is not None else None
        _check(self._c.strata_quantize_rows(
            self.h, _bf16(x), stride, rows, cols, _code_type(q), q.data_ptr(), _stride(q, rows, cols, "q"),
            q_scale.data_ptr(), _scale_stride(q_scale, rows), n_valid, self._stream()), "strata_quantize_rows")

    def expert_matmul(self, layout: Layout, a, a_scale, w, w_scale, out, gated: bool = False) -> None:
        """out[r] = (a[r] . w[e]) * a_scale[r] * w_scale[e] for the rows of every expert's segment; gated: silu(first half
        of the channels) * second half.  a [rows, inner] and w [E, channels, inner]: torch.int8 or torch.float8_e4m3fn."""
        rows, inner, a_stride = _strides(a)
        channels = w.size(1)
        if w.dtype != a.dtype or w.dim() != 3:
            raise ValueError("w is [E, channels, inner] of a's type")
        kind = _code_type(a)
        wide = channels // 2 if gated else channels
        _check(self._c.strata_moe_expert_matmul(self.h, layout.c, strata_matmul_args(
            kind, 1 if gated else 0, inner, channels, rows, a.data_ptr(), a_scale.data_ptr(),
            _flat(w, kind, self.E * channels * inner, "w"), _flat(w_scale, STRATA_T_F32, self.E * channels, "w_scale"),
            _bf16(out),
            a_stride, _scale_stride(a_scale, rows), _stride(out, rows, wide, "out")), self._stream()),
            "strata_moe_expert_matmul")

    def quantize_rows4(self, x, q: Rows4, layout: Optional[Layout] = None) -> None:
        """bf16 rows -> 4-bit codes with their scales; with a layout, only the rows it has in use."""
        rows, cols, stride = _strides(x)
        if q.rows != rows or q.cols != cols:
            raise ValueError(f"q: {rows} rows of {cols} are needed, not {q.rows} of {q.cols}")
        n_valid = layout.expert_offset.data_ptr() + 4 * self.E if layout is not None else None
        _check(self._c.strata_quantize_rows4(self.h, _bf16(x), stride, rows, cols, q.type, q.c, n_valid, self._stream()),
               "strata_quantize_rows4")

    def dequantize_rows4(self, q: Rows4, out, layout: Optional[Layout] = None) -> None:
        """The values of 4-bit rows in bf16 or fp32; with a layout, only of the rows it has in use."""
        n_valid = layout.expert_offset.data_ptr() + 4 * self.E if layout is not None else None
        _check(self._c.strata_dequantize_rows4(self.h, q.c, q.rows, q.cols, q.type, out.data_ptr(), _float_type(out),
                                               _stride(out, q.rows, q.cols, "out"), n_valid, self._stream()),
               "strata_dequantize_rows4")

    def expert_matmul4(self, layout: Layout, a: Rows4, w: Rows4, out, gated: bool = False) -> None:
        """expert_matmul over 4-bit rows a [rows, inner] and 4-bit weights w [E, channels, inner] of the same kind."""
        if w.codes.dim() != 3 or w.type != a.type or w.cols != a.cols or w.codes.size(0) != self.E:
            raise ValueError("w is [E, channels, inner] of a's kind")
        channels = w.codes.size(1)
        _check(self._c.strata_moe_expert_matmul4(self.h, layout.c, strata_matmul4_args(
            a.type, 1 if gated else 0, a.cols, channels, a.rows, a.c, w.c, _bf16(out),
            _stride(out, a.rows, channels // 2 if gated else channels, "out")), self._stream()),
            "strata_moe_expert_matmul4")

    def balance_stats(self, params: strata_balance_params) -> BalanceStats:
        """Outputs and scratch of balance_loss for these parameters."""
        rc, n = strata_moe_balance_scratch_bytes(self.h, params)
        _check(rc, "strata_moe_balance_scratch_bytes")
        return BalanceStats(self.R if params.per_rank else 1, self.E, n, self.device)

    def _balance_stats(self, params: strata_balance_params, stats: BalanceStats):
        if stats.groups != (self.R if params.per_rank else 1) or stats.E != self.E:
            raise ValueError("stats were made for other parameters")
        return stats.c

    def balance_loss(self, params: strata_balance_params, logits, ids, loss, stats: BalanceStats) -> None:
        """loss fp32 [2] = the balance loss and the mean square of the logits' log-sum-exp, each with its weight; stats: the
        counts per expert and the mean scores."""
        _check(self._c.strata_moe_balance_loss(
            self.h, params, logits.data_ptr(), _float_type(logits), _stride(logits, self.n_tok, self.E, "logits"),
            _flat(ids, _INT32, self.n_items, "ids"), _flat(loss, STRATA_T_F32, 2, "loss"), self._balance_stats(params, stats),
            stats.scratch.data_ptr(), stats.scratch.nbytes, self._stream()), "strata_moe_balance_loss")

    def balance_grad(self, params: strata_balance_params, logits, ids, stats: BalanceStats, dlogits, dloss=None,
                     add=None) -> None:
        """dlogits (of the type of logits) = the gradient of both losses, times dloss (fp32 [2] on the device, or None: 1), plus
        `add`, which may be dlogits itself."""
        if dlogits.dtype != logits.dtype or (add is not None and add.dtype != logits.dtype):
            raise ValueError("dlogits and add have the type of logits")
        n, e = self.n_tok, self.E
        _check(self._c.strata_moe_balance_grad(
            self.h, params, logits.data_ptr(), _float_type(logits), _stride(logits, n, e, "logits"),
            _flat(ids, _INT32, self.n_items, "ids"), self._balance_stats(params, stats),
            None if dloss is None else _flat(dloss, STRATA_T_F32, 2, "dloss"), None if add is None else add.data_ptr(),
            0 if add is None else _stride(add, n, e, "add"), dlogits.data_ptr(), _stride(dlogits, n, e, "dlogits"),
            self._stream()), "strata_moe_balance_grad")

    def row_experts(self, layout: Layout, out=None):
        """int32 [recv_rows]: the expert of every occupied receive row, -1 for padding and empty rows."""
        import torch
        if out is None:
            out = torch.empty((self.recv_rows,), dtype=torch.int32, device=self.device)
        _check(strata_moe_row_experts(self.h, layout.c, out.data_ptr(), out.shape[0], self._stream()),
               "strata_moe_row_experts")
        return out

    def trace(self, capacity_ctas: int = 4096):
        """Turns per-CTA probes on; returns the tensor [capacity, 4] = (start_ns, end_ns, wait_in_ns, wait_out_ns)."""
        import torch
        t = torch.zeros((capacity_ctas, 4), dtype=torch.int64, device=self.device)
        _check(strata_ctx_set_trace(self.h, t.data_ptr(), capacity_ctas), "strata_ctx_set_trace")
        self._trace = t
        return t

    @staticmethod
    def trace_summary(trace) -> dict:
        """Decodes a trace tensor after a launch (see timeline.trace_summary)."""
        from .timeline import trace_summary
        return trace_summary(trace.cpu().numpy())

    def trace_off(self) -> None:
        _check(strata_ctx_set_trace(self.h, None, 0), "strata_ctx_set_trace")
        self._trace = None

    def x_early(self, on: bool = True) -> None:
        """Promise that x is complete before the call preceding each dispatch starts (see the header)."""
        _check(strata_ctx_set_x_early(self.h, 1 if on else 0), "strata_ctx_set_x_early")

    def sm_budget(self, n_sm: int) -> None:
        """Sizes the persistent grids for n_sm SMs (0: the whole GPU)."""
        _check(strata_ctx_set_sm_budget(self.h, n_sm), "strata_ctx_set_sm_budget")

    def timeline(self, n_ctas: int = 2048, events_per_cta: int = 2048, pinned: bool = False):
        """Turns the event timeline on; returns the zeroed buffer [n_ctas, 1 + events_per_cta] (int64), in
        device memory or, with pinned=True, in page-locked host memory that the kernels write in place."""
        import torch
        if pinned:
            t = torch.zeros((n_ctas, 1 + events_per_cta), dtype=torch.int64, pin_memory=True)
        else:
            t = torch.zeros((n_ctas, 1 + events_per_cta), dtype=torch.int64, device=self.device)
        torch.cuda.synchronize(self.device)
        _check(strata_ctx_set_timeline(self.h, t.data_ptr(), n_ctas, events_per_cta), "strata_ctx_set_timeline")
        self._timeline = t
        return t

    def timeline_off(self) -> None:
        _check(strata_ctx_set_timeline(self.h, None, 0, 0), "strata_ctx_set_timeline")
        self._timeline = None

    @staticmethod
    def timeline_spans(t):
        """Synchronises and decodes a timeline buffer (see timeline.decode_timeline); returns (spans, dropped)."""
        import torch
        from .timeline import decode_timeline
        torch.cuda.synchronize()
        return decode_timeline(t.cpu().numpy().view("uint64"))

    # the paper's static window partitioning, as an alternative to run-time work claiming ------------
    def partition(self, layout: Layout, policy: strata_partition_policy, n_cores: int,
                  part: Optional[Partition] = None) -> Partition:
        if part is None:
            rc, mu = strata_moe_partition_max_units(self.shape, policy)
            _check(rc, "strata_moe_partition_max_units")
            part = Partition(self.R, self.E, n_cores, mu, self.device)
        _check(strata_moe_partition(self.h, layout.c, policy, n_cores, part.c, part.max_units, self._stream()),
               "strata_moe_partition")
        return part

    def dispatch_windows(self, layout: Layout, part: Partition, x, recv) -> None:
        _check(strata_moe_dispatch_windows(self.h, layout.c, part.c, part.n_cores, x.data_ptr(), recv.data_ptr(),
                                           recv.shape[0], self._stream()), "strata_moe_dispatch_windows")

    # full-mesh collectives over emulated ranks: tensors are [R, ...] slabs, one part per rank ------
    def allgather(self, src, dst) -> None:
        """src [R, n] -> dst [R, R, n] (any dtype; moved as bytes)."""
        R = src.shape[0]
        _check(strata_allgather(self.h, R, src.data_ptr(), dst.data_ptr(), src[0].numel() * src.element_size(),
                                self._stream()), "strata_allgather")

    def alltoall(self, src, dst) -> None:
        """src [R, R, n] -> dst [R, R, n], dst[r, p] = src[p, r]."""
        R = src.shape[0]
        _check(strata_alltoall(self.h, R, src.data_ptr(), dst.data_ptr(), src[0, 0].numel() * src.element_size(),
                               self._stream()), "strata_alltoall")

    def broadcast(self, src, dst, root: int) -> None:
        """src [R, n] -> dst [R, n], dst[r] = src[root]."""
        R = src.shape[0]
        _check(strata_broadcast(self.h, R, root, src.data_ptr(), dst.data_ptr(),
                                src[0].numel() * src.element_size(), self._stream()), "strata_broadcast")

    def p2p(self, src, dst, src_rank: int, dst_rank: int) -> None:
        """src, dst [R, n]: dst[dst_rank] = src[src_rank]."""
        R = src.shape[0]
        _check(strata_p2p(self.h, R, src_rank, dst_rank, src.data_ptr(), dst.data_ptr(),
                          src[0].numel() * src.element_size(), self._stream()), "strata_p2p")

    def alltoallv(self, src, dst, send_bytes, send_offset, recv_offset) -> None:
        """src [R, in_stride] and dst [R, out_stride] uint8; the three int64 [R, R] device tensors give, per
        (sender, receiver), the byte count, the offset in the sender's part and (indexed [receiver, sender])
        the offset in the receiver's part."""
        R = src.shape[0]
        for t in (src, dst, send_bytes, send_offset, recv_offset):
            if not t.is_contiguous():
                raise ValueError("alltoallv needs contiguous tensors")
        _check(strata_alltoallv(self.h, R, src.data_ptr(), src[0].numel() * src.element_size(), dst.data_ptr(),
                                dst[0].numel() * dst.element_size(), send_bytes.data_ptr(), send_offset.data_ptr(),
                                recv_offset.data_ptr(), self._stream()), "strata_alltoallv")

    def reducescatter(self, src, dst) -> None:
        """src bf16 [R, R, n] -> dst bf16 [R, n], dst[r] = sum over p of src[p, r] (rank order, fp32)."""
        R = src.shape[0]
        _check(strata_reducescatter(self.h, R, src.data_ptr(), dst.data_ptr(), src[0, 0].numel(), self._stream()),
               "strata_reducescatter")

    def allreduce(self, src, dst) -> None:
        """src bf16 [R, n] -> dst bf16 [R, n], dst[r] = sum over p of src[p] (rank order, fp32)."""
        R = src.shape[0]
        _check(strata_allreduce(self.h, R, src.data_ptr(), dst.data_ptr(), src[0].numel(), self._stream()),
               "strata_allreduce")

    def device_status(self) -> int:
        rc, st = strata_device_status(self.h, self._stream())
        _check(rc, "strata_device_status")
        return st

    def launch_count(self) -> int:
        rc, n = strata_ctx_launch_count(self.h)
        _check(rc, "strata_ctx_launch_count")
        return n
