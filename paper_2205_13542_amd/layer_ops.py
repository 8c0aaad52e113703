"""Operators around attention in a model that reads a pooled map, channels last.

With gradients:

    normed, stream = rms_norm_add(heard, stream, w, out_dtype=torch.bfloat16)
    q = rotary(q, positions, frequencies)                  # pairs of channels turned by a token's place
    y = gated_act(linear(normed), act="silu", checkpoint="int8")

For serving, in 8-bit integers:

    held, scale, stream = rms_norm_add_int8(heard, stream, w)
    y = linear_int8(held, scale, weight, weight_scale)     # weight, weight_scale = quantize_int8(w)

Each runs in libbevpool.so (include/bevmap.h) as the operators of ``map_ops`` do: on
the current stream of its inputs' device, with temporaries from torch's allocator,
and with tensors elsewhere, types and layouts that a call does not take refused
with a BevpoolError.
"""
from __future__ import annotations

import math

import torch
from torch.autograd import forward_ad

from . import _binding, _map_binding
from .map_ops import (_ACTS, _MOST, _call, _code, _device, _empty_like, _first_order_only, _learns, _ptr, _refuse,
                      _row_stride)

_POSITIONS = {torch.int32: _map_binding.BEVMAP_POSITION_I32, torch.int64: _map_binding.BEVMAP_POSITION_I64,
              torch.float32: _map_binding.BEVMAP_POSITION_F32}
_HELD_BLOCK = 32        # channels that share an exponent in a checkpoint


def _rows(t, name):
    """Rows, columns and the row stride of t, its last dimension the columns."""
    if t.dim() < 1:
        _refuse(f"{name} must have a channel dimension", _binding.BEVPOOL_ERR_SHAPE_MISMATCH)
    stride = _row_stride(t)
    if stride is None:
        _refuse(f"rows of {name} must be evenly spaced, their channels adjacent")
    columns = t.shape[-1]
    rows = math.prod(t.shape[:-1])
    if rows > _MOST or columns > _MOST:
        _refuse(f"{name} {tuple(t.shape)}: too large", _binding.BEVPOOL_ERR_OVERFLOW)
    return rows, columns, stride


def _vector(t, n, name):
    if t is not None and (t.dim() != 1 or t.shape[0] != n or not t.is_contiguous()):
        _refuse(f"{name} must be a contiguous tensor of {n} elements", _binding.BEVPOOL_ERR_SHAPE_MISMATCH)


def _no_gradient(call, *tensors):
    """Refuses tensors through which a gradient or a tangent would have to pass."""
    if _learns(*tensors):
        for t in tensors:
            if t is not None and ((torch.is_grad_enabled() and t.requires_grad)
                                  or forward_ad.unpack_dual(t).tangent is not None):
                _refuse(f"{call} has no gradient: call it under torch.no_grad(), on tensors without a tangent")


def _rms_of(x, residual, weight, eps, out_dtype):
    """The device and the description of a norm."""
    index = _device(x, residual, weight)
    rows, channels, stride = _rows(x, "x")
    residual_stride = channels
    if residual is not None:
        if residual.shape != x.shape or residual.dtype != x.dtype:
            _refuse("residual must have the shape and dtype of x", _binding.BEVPOOL_ERR_SHAPE_MISMATCH)
        residual_stride = _rows(residual, "residual")[2]
    _vector(weight, channels, "weight")
    return index, _map_binding.bevmap_rms(
        rows, channels, _code(x.dtype), _code(out_dtype or x.dtype),
        _binding.BEVPOOL_F32 if weight is None else _code(weight.dtype), stride, residual_stride, eps)


def _rms_forward(x, residual, weight, eps, out_dtype, train):
    """y, x + residual (x where there is none), rstd for the backward, and the description."""
    index, norm = _rms_of(x, residual, weight, eps, out_dtype)
    y = x.new_empty(x.shape, dtype=out_dtype or x.dtype)
    total = None if residual is None else _empty_like(x)
    rstd = x.new_empty(norm.rows, dtype=torch.float32) if train else None
    _call(_map_binding.bevmap_rms_norm, index, norm, x.data_ptr(), _ptr(residual), _ptr(weight), _ptr(total),
          y.data_ptr(), _ptr(rstd))
    return y, total, rstd, norm


def _rms_backward(norm, dy, dtotal, x, residual, weight, rstd, want_weight):
    dy = dy.contiguous()
    if dtotal is not None:
        dtotal = dtotal.contiguous()
    dx = _empty_like(x)
    dw = torch.empty_like(weight) if want_weight else None
    size = _map_binding.bevmap_rms_norm_backward_workspace(norm) if want_weight else 0
    space = x.new_empty(size, dtype=torch.uint8) if size else None
    _call(_map_binding.bevmap_rms_norm_backward, x.get_device(), norm, dy.data_ptr(), _ptr(dtotal), x.data_ptr(),
          _ptr(residual), _ptr(weight), rstd.data_ptr(), dx.data_ptr(), _ptr(dw), _ptr(space), size)
    return dx, dw


class _RmsNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, eps, out_dtype):
        y, _, rstd, ctx.norm = _rms_forward(x, None, weight, eps, out_dtype, True)
        ctx.save_for_backward(x, weight, rstd)
        return y

    @staticmethod
    def backward(ctx, dy):
        _first_order_only()
        x, weight, rstd = ctx.saved_tensors
        need = ctx.needs_input_grad
        dx, dw = _rms_backward(ctx.norm, dy, None, x, None, weight, rstd, need[1])
        return dx if need[0] else None, dw, None, None


class _RmsNormAdd(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, weight, eps, out_dtype):
        y, total, rstd, ctx.norm = _rms_forward(x, residual, weight, eps, out_dtype, True)
        if x.dtype == torch.float32:
            ctx.norm.x_stride = ctx.norm.channels
            ctx.save_for_backward(total, None, weight, rstd)
        else:       # the sum of 16-bit numbers, rounded, would take its 2^-9 into the weight's gradient
            ctx.save_for_backward(x, residual, weight, rstd)
        ctx.set_materialize_grads(False)
        return y, total

    @staticmethod
    def backward(ctx, dy, dtotal):
        _first_order_only()
        x, residual, weight, rstd = ctx.saved_tensors
        need = ctx.needs_input_grad
        if dy is None:          # y was not used: the gradient of a sum
            return dtotal, dtotal, torch.zeros_like(weight) if need[2] else None, None, None
        dx, dw = _rms_backward(ctx.norm, dy, dtotal, x, residual, weight, rstd, need[2])
        return dx if need[0] else None, dx if need[1] else None, dw, None, None


def rms_norm(x, weight=None, eps=1e-6, out_dtype=None):
    """Root-mean-square norm of every row: x [...][C] (fp32, bf16 or fp16),
    contiguous or with evenly spaced rows; returns a contiguous tensor of
    out_dtype (x's by default): weight * x / sqrt(mean(x^2) + eps) over the
    last dimension.

    weight: [C] of any of the types, or None for ones. Squares are summed in
    fp32 at any size of x, y is rounded once. Differentiable in x and weight,
    bitwise reproducible."""
    if _learns(x, weight):
        return _RmsNorm.apply(x, weight, eps, out_dtype)
    return _rms_forward(x, None, weight, eps, out_dtype, False)[0]


def rms_norm_add(x, residual, weight=None, eps=1e-6, out_dtype=None):
    """The norm of x + residual, and that sum: (y, total), both contiguous.

    residual: of x's shape and dtype. total has x's dtype; y (see ``rms_norm``)
    is formed from the sum before it is rounded to that. Differentiable in x,
    residual and weight, through either result or both."""
    if _learns(x, residual, weight):
        return _RmsNormAdd.apply(x, residual, weight, eps, out_dtype)
    return _rms_forward(x, residual, weight, eps, out_dtype, False)[:2]


def _rms_int8(x, residual, weight, eps):
    index, norm = _rms_of(x, residual, weight, eps, None)
    held = x.new_empty(x.shape, dtype=torch.int8)
    scale = x.new_empty(x.shape[:-1], dtype=torch.float32)
    total = None if residual is None else _empty_like(x)
    _call(_map_binding.bevmap_rms_norm_int8, index, norm, x.data_ptr(), _ptr(residual), _ptr(weight), _ptr(total),
          held.data_ptr(), scale.data_ptr())
    return held, scale, total


def rms_norm_int8(x, weight=None, eps=1e-6):
    """``rms_norm`` with its result in 8 bits: (held int8 [...][C], scale fp32
    [...]), held * scale being the norm to within half a scale, which is the
    row's largest magnitude over 127. Rows with an infinity or a NaN have scale
    NaN. For ``linear_int8``; has no gradient."""
    _no_gradient("rms_norm_int8", x, weight)
    return _rms_int8(x, None, weight, eps)[:2]


def rms_norm_add_int8(x, residual, weight=None, eps=1e-6):
    """``rms_norm_add`` with its result in 8 bits: (held, scale, total), see
    ``rms_norm_int8``. Has no gradient."""
    _no_gradient("rms_norm_add_int8", x, residual, weight)
    return _rms_int8(x, residual, weight, eps)


def quantize_int8(x):
    """Rows in 8 bits: x [...][C] (fp32, bf16 or fp16; evenly spaced rows) gives
    (held int8 [...][C], scale fp32 [...]): scale the row's largest magnitude
    over 127, held = round(x / scale), halves to the even neighbour. A row of
    zeros has scale 0, one with an infinity or a NaN scale NaN. For weights
    (a row is an output channel) and activations of ``linear_int8``. Has no
    gradient."""
    _no_gradient("quantize_int8", x)
    index = _device(x)
    rows, columns, stride = _rows(x, "x")
    held = x.new_empty(x.shape, dtype=torch.int8)
    scale = x.new_empty(x.shape[:-1], dtype=torch.float32)
    _call(_map_binding.bevmap_quantize_int8, index, x.data_ptr(), stride, held.data_ptr(), scale.data_ptr(), rows,
          columns, _code(x.dtype))
    return held, scale


def linear_int8(x, x_scale, weight, weight_scale, bias=None, out_dtype=None):
    """Product of 8-bit integers: x int8 [...][K], weight int8 [N][K] (both with
    evenly spaced rows), x_scale fp32 [...] and weight_scale fp32 [N] give
    x_scale * weight_scale * (x @ weight^T) + bias as [...][N] of out_dtype
    (fp32, bf16 or fp16; bf16 by default), contiguous. bias: fp32 [N] or None.

    The integers' sums are exact (K at most 131071); fp32 and one rounding
    follow. A scale of NaN reaches its row or channel. Has no gradient."""
    _no_gradient("linear_int8", x_scale, weight_scale, bias)
    index = _device(x, x_scale, weight, weight_scale, bias)
    if x.dtype != torch.int8 or weight.dtype != torch.int8:
        _refuse(f"x and weight must be int8, not {x.dtype} and {weight.dtype}", _binding.BEVPOOL_ERR_UNSUPPORTED_DTYPE)
    rows, channels, stride = _rows(x, "x")
    if weight.dim() != 2 or weight.shape[1] != channels:
        _refuse(f"weight must be [N][{channels}], not {tuple(weight.shape)}", _binding.BEVPOOL_ERR_SHAPE_MISMATCH)
    features, _, weight_stride = _rows(weight, "weight")
    if x_scale.shape != x.shape[:-1] or not x_scale.is_contiguous():
        _refuse(f"x_scale must be a contiguous tensor {tuple(x.shape[:-1])}", _binding.BEVPOOL_ERR_SHAPE_MISMATCH)
    _vector(weight_scale, features, "weight_scale")
    _vector(bias, features, "bias")
    for t, name in ((x_scale, "x_scale"), (weight_scale, "weight_scale"), (bias, "bias")):
        if t is not None and t.dtype != torch.float32:
            _refuse(f"{name} must be fp32, not {t.dtype}", _binding.BEVPOOL_ERR_UNSUPPORTED_DTYPE)
    out_dtype = out_dtype or torch.bfloat16
    linear = _map_binding.bevmap_linear(rows, channels, features, stride, weight_stride, _code(out_dtype))
    y = x_scale.new_empty((*x.shape[:-1], features), dtype=out_dtype)
    _call(_map_binding.bevmap_linear_int8, index, linear, x.data_ptr(), x_scale.data_ptr(), weight.data_ptr(),
          weight_scale.data_ptr(), _ptr(bias), y.data_ptr())
    return y


def _rotary_of(x, positions, frequencies, interleaved, amplitude):
    """The device and the description of a turn; x [B][N][H][D] in any strides but for adjacent channels."""
    index = _device(x, positions, frequencies)
    if x.dim() != 4:
        _refuse("x must be [B][N][H][D]", _binding.BEVPOOL_ERR_SHAPE_MISMATCH)
    B, N, H, D = x.shape
    if frequencies.dim() != 1 or not frequencies.is_contiguous():
        _refuse("frequencies must be a contiguous vector", _binding.BEVPOOL_ERR_SHAPE_MISMATCH)
    if frequencies.dtype != torch.float64:
        _refuse(f"frequencies must be fp64, not {frequencies.dtype}", _binding.BEVPOOL_ERR_UNSUPPORTED_DTYPE)
    kind = _POSITIONS.get(positions.dtype)
    if kind is None:
        _refuse(f"positions must be int32, int64 or fp32, not {positions.dtype}",
                _binding.BEVPOOL_ERR_UNSUPPORTED_DTYPE)
    shape = tuple(positions.shape)
    if len(shape) not in (2, 3) or shape[:2] != (B, N) or not positions.is_contiguous():
        _refuse(f"positions must be a contiguous tensor [{B}][{N}] or [{B}][{N}][axes], not {shape}",
                _binding.BEVPOOL_ERR_SHAPE_MISMATCH)
    axes, pairs = shape[2] if len(shape) == 3 else 1, frequencies.shape[0]
    if max(B, N, H, D, axes, pairs) > _MOST:
        _refuse(f"x {tuple(x.shape)}: too large", _binding.BEVPOOL_ERR_OVERFLOW)
    strides = x.stride()
    if D > 1 and strides[3] != 1:
        _refuse("the channels of x must be adjacent")
    return index, _map_binding.bevmap_turn(B, N, H, D, pairs, axes, bool(interleaved), kind, _code(x.dtype),
                                           amplitude, *strides[:3])


def _turn(index, turn, x, positions, frequencies, backward):
    out = _empty_like(x)
    _call(_map_binding.bevmap_rotary, index, turn, x.data_ptr(), positions.data_ptr(), frequencies.data_ptr(),
          out.data_ptr(), backward)
    return out


class _Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, positions, frequencies, interleaved, amplitude):
        index, ctx.turn = _rotary_of(x, positions, frequencies, interleaved, amplitude)
        ctx.save_for_backward(positions, frequencies)
        return _turn(index, ctx.turn, x, positions, frequencies, False)

    @staticmethod
    def backward(ctx, dy):
        _first_order_only()
        positions, frequencies = ctx.saved_tensors
        if dy.stride(3) != 1:
            dy = dy.contiguous()
        back = _map_binding.bevmap_turn.from_buffer_copy(ctx.turn)
        back.x_batch, back.x_row, back.x_head = dy.stride()[:3]
        return _turn(dy.get_device(), back, dy, positions, frequencies, True), None, None, None, None


def rotary(x, positions, frequencies, interleaved=False, amplitude=1.0):
    """Rotary positions: pairs of channels of every head turned by angles that go
    with the token's position. Returns a contiguous tensor of x's shape and dtype.

    x [B][N][H][D] (fp32, bf16 or fp16; any strides but for adjacent channels, so
    views of a packed projection do). frequencies: fp64 [P], radians to a unit of
    position (``rotary_frequencies``); the first 2 P channels turn, pair p being
    channels (2 p, 2 p + 1) if interleaved and (p, p + P) otherwise, and the
    others keep their values. positions: int32, int64 or fp32, [B][N], or
    [B][N][axes] for places along several axes (a cell's, in a map): P is a
    multiple of axes, and each P / axes neighbouring pairs turn with one axis.

    Angles are formed and reduced in 64 bits, so far positions are as exact as
    near ones; the turn, times amplitude, is fp32 and rounded once. An infinite
    position gives NaN. Differentiable in x."""
    if _learns(positions, frequencies) and (positions.requires_grad or frequencies.requires_grad):
        _refuse("positions and frequencies have no gradient")
    if _learns(x, positions, frequencies):
        return _Rotary.apply(x, positions, frequencies, interleaved, amplitude)
    index, turn = _rotary_of(x, positions, frequencies, interleaved, amplitude)
    return _turn(index, turn, x, positions, frequencies, False)


def rotary_frequencies(pairs, base=10000.0, axes=1, scaling=None, factor=1.0, context=None, fast=32.0, slow=1.0,
                       device=None):
    """Frequencies (fp64 [pairs]) for ``rotary``: base ** (-i / n) for the n =
    pairs / axes pairs i of each axis, scaled for contexts ``factor`` times as
    long as those that a model learned:

    None      as they are
    "linear"  all divided by factor: positions are interpolated
    "base"    a base that divides the slowest by factor and leaves the fastest
              (of at least two pairs to an axis)
    "parts"   pairs that turn ``fast`` times or more within ``context`` positions
              (the length learned) stay, those that turn ``slow`` times or less
              are divided by factor, and between the two the share goes linearly
              with the number of turns. (With this scaling an amplitude of
              0.1 log(factor) + 1 for queries and keys is customary.)"""
    if pairs < 1 or axes < 1 or pairs % axes:
        _refuse(f"pairs={pairs} must be a multiple of axes={axes}")
    if not (base > 0 and math.isfinite(base) and factor >= 1 and math.isfinite(factor)):
        _refuse(f"base={base} must be positive and factor={factor} at least 1, both finite")
    n = pairs // axes
    if scaling == "base":
        if n < 2:
            _refuse("scaling by the base needs two pairs to an axis")
        base = base * factor ** (n / (n - 1))
    f = base ** (-torch.arange(n, dtype=torch.float64) / n)
    if scaling == "linear":
        f = f / factor
    elif scaling == "parts":
        if context is None or not (context > 0 and 0 <= slow < fast):
            _refuse(f"scaling by parts needs a context above 0 and 0 <= slow < fast, not {context}, {slow}, {fast}")
        stays = ((f * context / (2 * math.pi) - slow) / (fast - slow)).clamp(0, 1)
        f = f * (stays + (1 - stays) / factor)
    elif scaling not in (None, "base"):
        _refuse(f"scaling must be None, linear, base or parts, not {scaling}")
    return f.repeat(axes).to(device)


def _gate_of(x, act):
    index = _device(x)
    code = _ACTS.get(act)
    if code is None:
        _refuse(f"act must be one of {', '.join(_ACTS)}")
    rows, columns, stride = _rows(x, "x")
    if columns % 2 or not columns:
        _refuse(f"x must have two halves, not {columns} channels", _binding.BEVPOOL_ERR_SHAPE_MISMATCH)
    return index, _map_binding.bevmap_gate(rows, columns // 2, code, _code(x.dtype), stride)


def _gate_forward(x, act, hold):
    """y, what is held of x in 8 bits (or None twice), and the description."""
    index, gate = _gate_of(x, act)
    y = x.new_empty((*x.shape[:-1], gate.features))
    held = exponents = None
    if hold:
        held = x.new_empty((gate.rows, 2, gate.features), dtype=torch.int8)
        exponents = x.new_empty((gate.rows, 2, -(-gate.features // _HELD_BLOCK)), dtype=torch.uint8)
    _call(_map_binding.bevmap_gated_act, index, gate, x.data_ptr(), y.data_ptr(), _ptr(held), _ptr(exponents))
    return y, held, exponents, gate


class _GatedAct(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, act, hold):
        y, held, exponents, ctx.gate = _gate_forward(x, act, hold)
        if hold:
            ctx.save_for_backward(held, exponents)
        else:
            ctx.save_for_backward(x)
        return y

    @staticmethod
    def backward(ctx, dy):
        _first_order_only()
        x = held = exponents = None
        if len(ctx.saved_tensors) == 1:
            x, = ctx.saved_tensors
        else:
            held, exponents = ctx.saved_tensors
        dy = dy.contiguous()
        gate = ctx.gate
        dx = dy.new_empty((*dy.shape[:-1], 2 * gate.features))
        _call(_map_binding.bevmap_gated_act_backward, dy.get_device(), gate, dy.data_ptr(),
              _ptr(x), _ptr(held), _ptr(exponents), dx.data_ptr())
        return dx, None, None


def gated_act(x, act="silu", checkpoint=None):
    """Gated activation: act(gate) * value, the halves of every row of x [...][2 F]
    (fp32, bf16 or fp16; contiguous or with evenly spaced rows). Returns [...][F],
    contiguous, rounded once; act "none", "relu", "silu" or "gelu" (through erf).

    checkpoint: what the backward reads. None keeps x; "int8" keeps a copy in 8.25
    bits an element (32 neighbouring channels of a half share a power of two, and
    each is off by at most 1 / 127 of the largest magnitude among them), so that x can
    be freed. The result is the same; the gradient is that at the copy.
    Differentiable in x, bitwise reproducible."""
    if checkpoint not in (None, "int8"):
        _refuse(f"checkpoint must be None or int8, not {checkpoint}")
    if _learns(x):
        return _GatedAct.apply(x, act, checkpoint is not None)
    return _gate_forward(x, act, False)[0]
