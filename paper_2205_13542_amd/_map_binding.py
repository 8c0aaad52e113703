"""ctypes binding of the map operators in libbevpool.so: the C ABI of
include/bevmap.h under the same names, with argument marshalling only.
Addresses are device addresses as ints, 0 for NULL.
"""
from __future__ import annotations

import ctypes

from . import _binding

BEVMAP_ACT_NONE, BEVMAP_ACT_RELU, BEVMAP_ACT_SILU, BEVMAP_ACT_GELU = 0, 1, 2, 3
BEVMAP_POSITION_I32, BEVMAP_POSITION_I64, BEVMAP_POSITION_F32 = 0, 1, 2

EXPORTED = ("bevmap_group_norm_workspace", "bevmap_group_norm", "bevmap_group_norm_backward",
            "bevmap_attention_workspace", "bevmap_attention", "bevmap_attention_backward", "bevmap_dropout",
            "bevmap_rms_norm", "bevmap_rms_norm_backward_workspace", "bevmap_rms_norm_backward",
            "bevmap_rms_norm_int8", "bevmap_quantize_int8", "bevmap_linear_int8", "bevmap_rotary",
            "bevmap_gated_act", "bevmap_gated_act_backward")

_i32, _i64, _u64, _vp, _f32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64, ctypes.c_void_p, ctypes.c_float


class bevmap_norm(ctypes.Structure):
    _fields_ = [("batch", _i32), ("pixels", _i32), ("channels", _i32), ("groups", _i32), ("row_stride", _i64),
                ("eps", _f32), ("act", _i32), ("x_dtype", _i32), ("y_dtype", _i32), ("weight_dtype", _i32)]


class bevmap_attend(ctypes.Structure):
    _fields_ = [("batch", _i32), ("queries", _i32), ("keys", _i32), ("heads", _i32), ("key_heads", _i32),
                ("dim", _i32), ("dtype", _i32), ("scale", _f32),
                ("q_batch", _i64), ("q_row", _i64), ("q_head", _i64),
                ("k_batch", _i64), ("k_row", _i64), ("k_head", _i64),
                ("v_batch", _i64), ("v_row", _i64), ("v_head", _i64), ("mask_batch", _i64)]


class bevmap_rms(ctypes.Structure):
    _fields_ = [("rows", _i64), ("channels", _i32), ("x_dtype", _i32), ("y_dtype", _i32), ("weight_dtype", _i32),
                ("x_stride", _i64), ("residual_stride", _i64), ("eps", _f32)]


class bevmap_linear(ctypes.Structure):
    _fields_ = [("rows", _i64), ("channels", _i32), ("features", _i32), ("x_stride", _i64), ("w_stride", _i64),
                ("y_dtype", _i32)]


class bevmap_turn(ctypes.Structure):
    _fields_ = [("batch", _i32), ("tokens", _i32), ("heads", _i32), ("dim", _i32), ("pairs", _i32), ("axes", _i32),
                ("interleaved", _i32), ("positions_type", _i32), ("dtype", _i32), ("amplitude", _f32),
                ("x_batch", _i64), ("x_row", _i64), ("x_head", _i64)]


class bevmap_gate(ctypes.Structure):
    _fields_ = [("rows", _i64), ("features", _i32), ("act", _i32), ("dtype", _i32), ("x_stride", _i64)]


_lib = None


def load():
    global _lib
    if _lib is None:
        lib = _binding.load()
        norm, attend = ctypes.POINTER(bevmap_norm), ctypes.POINTER(bevmap_attend)
        lib.bevmap_group_norm_workspace.argtypes = [norm, _i32]
        lib.bevmap_group_norm_workspace.restype = _i64
        lib.bevmap_group_norm.argtypes = [norm] + [_vp] * 7 + [_i64, _vp]
        lib.bevmap_group_norm_backward.argtypes = [norm] + [_vp] * 10 + [_i64, _vp]
        lib.bevmap_attention_workspace.argtypes = [attend, _i32]
        lib.bevmap_attention_workspace.restype = _i64
        lib.bevmap_attention.argtypes = [attend] + [_vp] * 9 + [_i64, _vp]
        lib.bevmap_attention_backward.argtypes = [attend] + [_vp] * 13 + [_i64, _vp]
        lib.bevmap_dropout.argtypes = [_vp, _i64, _vp, _i64, _vp, _i64, _i64, _i32, _i32, _u64, _u64, _vp]
        rms, linear = ctypes.POINTER(bevmap_rms), ctypes.POINTER(bevmap_linear)
        turn, gate = ctypes.POINTER(bevmap_turn), ctypes.POINTER(bevmap_gate)
        lib.bevmap_rms_norm.argtypes = [rms] + [_vp] * 7
        lib.bevmap_rms_norm_backward_workspace.argtypes = [rms]
        lib.bevmap_rms_norm_backward_workspace.restype = _i64
        lib.bevmap_rms_norm_backward.argtypes = [rms] + [_vp] * 9 + [_i64, _vp]
        lib.bevmap_rms_norm_int8.argtypes = [rms] + [_vp] * 7
        lib.bevmap_quantize_int8.argtypes = [_vp, _i64, _vp, _vp, _i64, _i32, _i32, _vp]
        lib.bevmap_linear_int8.argtypes = [linear] + [_vp] * 7
        lib.bevmap_rotary.argtypes = [turn] + [_vp] * 4 + [_i32, _vp]
        lib.bevmap_gated_act.argtypes = [gate] + [_vp] * 5
        lib.bevmap_gated_act_backward.argtypes = [gate] + [_vp] * 6
        _lib = lib
    return _lib


def _check(rc: int) -> int:
    """A workspace's bytes, or nothing; a negative code is raised."""
    if rc < 0:
        raise _binding.BevpoolError(rc, _binding.bevpool_last_error())
    return rc


def bevmap_group_norm_workspace(norm: bevmap_norm, backward: bool) -> int:
    return _check(load().bevmap_group_norm_workspace(norm, backward))


def bevmap_group_norm(norm: bevmap_norm, x: int, weight: int, bias: int, y: int, mean: int, rstd: int,
                      workspace: int, workspace_bytes: int, hip_stream: int = 0) -> None:
    _check(load().bevmap_group_norm(norm, x, weight, bias, y, mean, rstd, workspace, workspace_bytes, hip_stream))


def bevmap_group_norm_backward(norm: bevmap_norm, grad_y: int, x: int, weight: int, bias: int, mean: int, rstd: int,
                               grad_x: int, grad_weight: int, grad_bias: int, workspace: int, workspace_bytes: int,
                               hip_stream: int = 0) -> None:
    _check(load().bevmap_group_norm_backward(norm, grad_y, x, weight, bias, mean, rstd, grad_x, grad_weight,
                                             grad_bias, workspace, workspace_bytes, hip_stream))


def bevmap_attention_workspace(attend: bevmap_attend, backward: bool) -> int:
    return _check(load().bevmap_attention_workspace(attend, backward))


def bevmap_attention(attend: bevmap_attend, q: int, k: int, v: int, key_lengths: int, key_mask: int, out: int,
                     out_low: int, lse: int, workspace: int, workspace_bytes: int, hip_stream: int = 0) -> None:
    _check(load().bevmap_attention(attend, q, k, v, key_lengths, key_mask, out, out_low, lse, workspace,
                                   workspace_bytes, hip_stream))


def bevmap_attention_backward(attend: bevmap_attend, grad_out: int, q: int, k: int, v: int, key_lengths: int,
                              key_mask: int, out: int, out_low: int, lse: int, grad_q: int, grad_k: int,
                              grad_v: int, workspace: int, workspace_bytes: int, hip_stream: int = 0) -> None:
    _check(load().bevmap_attention_backward(attend, grad_out, q, k, v, key_lengths, key_mask, out, out_low, lse,
                                            grad_q, grad_k, grad_v, workspace, workspace_bytes, hip_stream))


def bevmap_dropout(x: int, x_stride: int, residual: int, residual_stride: int, y: int, rows: int, columns: int,
                   dtype: int, threshold: int, seed: int, offset: int, hip_stream: int = 0) -> None:
    _check(load().bevmap_dropout(x, x_stride, residual, residual_stride, y, rows, columns, dtype, threshold, seed,
                                 offset, hip_stream))


def bevmap_rms_norm(norm: bevmap_rms, x: int, residual: int, weight: int, sum: int, y: int, rstd: int,
                    hip_stream: int = 0) -> None:
    _check(load().bevmap_rms_norm(norm, x, residual, weight, sum, y, rstd, hip_stream))


def bevmap_rms_norm_backward_workspace(norm: bevmap_rms) -> int:
    return _check(load().bevmap_rms_norm_backward_workspace(norm))


def bevmap_rms_norm_backward(norm: bevmap_rms, grad_y: int, grad_sum: int, x: int, residual: int, weight: int,
                             rstd: int, grad_x: int, grad_weight: int, workspace: int, workspace_bytes: int,
                             hip_stream: int = 0) -> None:
    _check(load().bevmap_rms_norm_backward(norm, grad_y, grad_sum, x, residual, weight, rstd, grad_x, grad_weight,
                                           workspace, workspace_bytes, hip_stream))


def bevmap_rms_norm_int8(norm: bevmap_rms, x: int, residual: int, weight: int, sum: int, held: int, scale: int,
                         hip_stream: int = 0) -> None:
    _check(load().bevmap_rms_norm_int8(norm, x, residual, weight, sum, held, scale, hip_stream))


def bevmap_quantize_int8(x: int, x_stride: int, held: int, scale: int, rows: int, columns: int, dtype: int,
                         hip_stream: int = 0) -> None:
    _check(load().bevmap_quantize_int8(x, x_stride, held, scale, rows, columns, dtype, hip_stream))


def bevmap_linear_int8(linear: bevmap_linear, x: int, x_scale: int, w: int, w_scale: int, bias: int, y: int,
                       hip_stream: int = 0) -> None:
    _check(load().bevmap_linear_int8(linear, x, x_scale, w, w_scale, bias, y, hip_stream))


def bevmap_rotary(turn: bevmap_turn, x: int, positions: int, frequencies: int, out: int, backward: bool,
                  hip_stream: int = 0) -> None:
    _check(load().bevmap_rotary(turn, x, positions, frequencies, out, backward, hip_stream))


def bevmap_gated_act(gate: bevmap_gate, x: int, y: int, held: int, exponents: int, hip_stream: int = 0) -> None:
    _check(load().bevmap_gated_act(gate, x, y, held, exponents, hip_stream))


def bevmap_gated_act_backward(gate: bevmap_gate, grad_y: int, x: int, held: int, exponents: int, grad_x: int,
                              hip_stream: int = 0) -> None:
    _check(load().bevmap_gated_act_backward(gate, grad_y, x, held, exponents, grad_x, hip_stream))
