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
with a BevpoolError. Checks, allocations and autograd nodes are native too
(csrc/layer_torch.cpp): a call on a few rows costs its host time.

A call that is being traced (torch.jit.trace, make_fx) is refused too: a tracer
cannot see it and would record its result as a constant.

All of them may be captured into a graph. Before a training step is, let go of what
earlier eager steps on the same leaves returned: while such a result lives, torch
forms the leaves' gradients on that step's stream, which a capture must not enter.
"""
from __future__ import annotations

import math

import torch

from . import _binding, _map_binding
from .map_ops import _ACTS, _refuse

_map_binding.load()         # the library that the native module calls, built if this package was
try:
    from . import _layer_native as _native
except ImportError as missing:
    raise ImportError(f"{missing}: build it with python -m paper_2205_13542_amd.build") from missing
_native.set_error(_binding.BevpoolError)


def _given(t, name):
    if t is None:
        _refuse(f"{name} must be a tensor")
    return t


def rms_norm(x, weight=None, eps=1e-6, out_dtype=None):
    """Root-mean-square norm of every row: x [...][C] (fp32, bf16 or fp16),
    contiguous or with evenly spaced rows; returns a contiguous tensor of
    out_dtype (x's by default): weight * x / sqrt(mean(x^2) + eps) over the
    last dimension.

    weight: [C] of any of the types, or None for ones. Squares are summed in
    fp32 at any size of x, y is rounded once. Differentiable in x and weight,
    bitwise reproducible."""
    return _native.rms_norm(x, None, weight, eps, out_dtype)


def rms_norm_add(x, residual, weight=None, eps=1e-6, out_dtype=None):
    """The norm of x + residual, and that sum: (y, total), both contiguous.

    residual: of x's shape and dtype. total has x's dtype; y (see ``rms_norm``)
    is formed from the sum before it is rounded to that. Differentiable in x,
    residual and weight, through either result or both."""
    return _native.rms_norm(x, _given(residual, "residual"), weight, eps, out_dtype)


def rms_norm_int8(x, weight=None, eps=1e-6):
    """``rms_norm`` with its result in 8 bits: (held int8 [...][C], scale fp32
    [...]), held * scale being the norm to within half a scale, which is the
    row's largest magnitude over 127. Rows with an infinity or a NaN have scale
    NaN. For ``linear_int8``; has no gradient."""
    return _native.rms_norm_int8(x, None, weight, eps)


def rms_norm_add_int8(x, residual, weight=None, eps=1e-6):
    """``rms_norm_add`` with its result in 8 bits: (held, scale, total), see
    ``rms_norm_int8``. Has no gradient."""
    return _native.rms_norm_int8(x, _given(residual, "residual"), weight, eps)


def quantize_int8(x):
    """Rows in 8 bits: x [...][C] (fp32, bf16 or fp16; evenly spaced rows) gives
    (held int8 [...][C], scale fp32 [...]): scale the row's largest magnitude
    over 127, held = round(x * (127 / that magnitude)), halves to the even neighbour. A row of
    zeros has scale 0, one with an infinity or a NaN scale NaN. For weights
    (a row is an output channel) and activations of ``linear_int8``. Has no
    gradient."""
    return _native.quantize_int8(x)


def linear_int8(x, x_scale, weight, weight_scale, bias=None, out_dtype=None):
    """Product of 8-bit integers: x int8 [...][K], weight int8 [N][K] (both with
    evenly spaced rows), x_scale fp32 [...] and weight_scale fp32 [N] give
    x_scale * weight_scale * (x @ weight^T) + bias as [...][N] of out_dtype
    (fp32, bf16 or fp16; bf16 by default), contiguous. bias: fp32 [N] or None.

    The integers' sums are exact (K at most 131071); fp32 and one rounding
    follow. A scale of NaN reaches its row or channel. Has no gradient."""
    return _native.linear_int8(x, x_scale, weight, weight_scale, bias, out_dtype)


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

    Angles are formed and reduced in 64 bits, so far positions, up to 2^53 in
    magnitude, are as exact as near ones; the turn, times amplitude, is fp32 and rounded once. An infinite
    position gives NaN. Differentiable in x."""
    return _native.rotary(x, positions, frequencies, interleaved, amplitude)


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


def gated_act(x, act="silu", checkpoint=None):
    """Gated activation: act(gate) * value, the halves of every row of x [...][2 F]
    (fp32, bf16 or fp16; contiguous or with evenly spaced rows). Returns [...][F],
    contiguous; act "none", "relu", "silu" or "gelu" (through erf), in fp32 to within
    2^-15 of its value in the tail far below 0 and some 2^-22 elsewhere, and the product
    rounded once.

    checkpoint: what the backward reads. None keeps x; "int8" keeps a copy in 8.25
    bits an element (32 neighbouring channels of a half share a power of two, and
    each is off by at most 1 / 127 of the largest magnitude among them), so that x can
    be freed. The result is the same; the gradient is that at the copy.
    Differentiable in x, bitwise reproducible."""
    code = _ACTS.get(act)
    if code is None:
        _refuse(f"act must be one of {', '.join(_ACTS)}")
    if checkpoint not in (None, "int8"):
        _refuse(f"checkpoint must be None or int8, not {checkpoint}")
    return _native.gated_act(x, code, checkpoint is not None)
