"""Operators of the model that reads a pooled map, channels last, with gradients.

    normed = group_norm_act(bev, groups=8, weight=w, bias=b, act="silu", out_dtype=torch.bfloat16)
    heard  = cross_attention(q, k, v, key_mask=seen)       # queries ask the map's cells
    tokens = dropout_add(heard, 0.1, seed, step, residual=tokens)

Each runs in libbevpool.so (include/bevmap.h) on the current stream of its
inputs' device, and is differentiable (backwards; inputs with a tangent of
torch.autograd.forward_ad are refused). Calls that are being traced by make_fx, or
without gradients by torch.jit.trace, are refused: their results would be recorded
as empty tensors. Temporaries come from torch's allocator.
There is no CPU form: tensors elsewhere are refused with a BevpoolError, as
are types and layouts that a call does not take (nothing is copied silently).
"""
from __future__ import annotations

import math

import torch
from torch.autograd import forward_ad

from . import _binding, _map_binding
from ._binding import BevpoolError

try:
    from . import _layer_native as _native
    _native.set_error(BevpoolError)
except ImportError:             # a build without it
    _native = None

_ACTS = {"none": _map_binding.BEVMAP_ACT_NONE, "relu": _map_binding.BEVMAP_ACT_RELU,
         "silu": _map_binding.BEVMAP_ACT_SILU, "gelu": _map_binding.BEVMAP_ACT_GELU}
_CODES = {torch.float32: _binding.BEVPOOL_F32, torch.bfloat16: _binding.BEVPOOL_BF16,
          torch.float16: _binding.BEVPOOL_F16}
_DTYPES = {code: dtype for dtype, code in _CODES.items()}

_MOST = (1 << 31) - 1       # of a size in the C descriptions, where ctypes would wrap it round


def _refuse(message, code=_binding.BEVPOOL_ERR_INVALID_ARG):
    raise BevpoolError(code, message)


def _code(dtype) -> int:
    code = _CODES.get(dtype)
    if code is None:
        _refuse(f"dtype {dtype}", _binding.BEVPOOL_ERR_UNSUPPORTED_DTYPE)
    return code


def _row_stride(t):
    """Elements from row to row (of the last dimension) if rows are evenly
    spaced and their elements adjacent, else None."""
    if t.is_contiguous():
        return t.shape[-1] if t.dim() else 1
    shape, strides = t.shape, t.stride()
    if strides[-1] != 1 and shape[-1] > 1:
        return None
    step = expect = None
    for size, stride in zip(reversed(shape[:-1]), reversed(strides[:-1])):
        if size == 1:
            continue
        if step is None:
            step = stride
        elif stride != expect:
            return None
        expect = stride * size
    return shape[-1] if step is None else step if step >= shape[-1] else None


def _device(first, *others) -> int:
    """The index of the GPU that holds all tensors (None among them is skipped)."""
    if not first.is_cuda:
        _refuse("inputs must be device tensors")
    index = first.get_device()
    for t in others:
        if t is not None and t.get_device() != index:
            _refuse("all tensors must be on one device")
    return index


def _jit_not_traced(jit=True):
    if jit and torch.jit.is_tracing():
        _refuse("the operators cannot be traced: their results would be recorded as empty tensors")


# Refuses a call that is being traced (torch.jit.trace, make_fx), which sees the allocation of a
# result but not what fills it. An autograd function is called again by what torch.jit.trace makes
# of it: _not_traced(False) lets that pass.
_not_traced = _jit_not_traced if _native is None else _native.not_traced


def _call(function, index, *args):
    """function(*args, stream) with the device current and its current stream."""
    # the C function behind torch.cuda.current_stream: calls here cost as little as their host time
    if torch.cuda.current_device() == index:
        return function(*args, torch._C._cuda_getCurrentRawStream(index))
    with torch.cuda.device(index):
        return function(*args, torch._C._cuda_getCurrentRawStream(index))


def _empty_like(t):
    return torch.empty_like(t, memory_format=torch.contiguous_format)


def _ptr(t) -> int:
    return 0 if t is None else t.data_ptr()


def _first_order_only():
    """Backward passes run with gradients enabled only where a graph of them is asked for."""
    if torch.is_grad_enabled():
        raise RuntimeError("the map operators have no second derivatives")


def _norm_forward(x, groups, weight, bias, eps, act, out_dtype):
    """y, mean and rstd [2][B][groups], and the description."""
    if x.dim() < 2:
        _refuse("x must have a batch and a channel dimension")
    index = _device(x, weight, bias)
    act = _ACTS.get(act)
    if act is None:
        _refuse(f"act must be one of {', '.join(_ACTS)}")
    shape = x.shape
    B, C = shape[0], shape[-1]
    pixels = math.prod(shape[1:-1])
    if B > _MOST or pixels > _MOST or C > _MOST or not -_MOST <= groups <= _MOST:
        _refuse(f"x {tuple(shape)}, groups={groups}: too large", _binding.BEVPOOL_ERR_OVERFLOW)
    for t, name in ((weight, "weight"), (bias, "bias")):
        if t is not None and (t.dim() != 1 or t.shape[0] != C or not t.is_contiguous()):
            _refuse(f"{name} must be a contiguous tensor of {C} elements", _binding.BEVPOOL_ERR_SHAPE_MISMATCH)
    if weight is not None and bias is not None and weight.dtype != bias.dtype:
        _refuse("weight and bias must share a dtype", _binding.BEVPOOL_ERR_UNSUPPORTED_DTYPE)
    stride = _row_stride(x)
    if stride is None:
        _refuse("rows of x must be evenly spaced, their channels adjacent")
    w_like = weight if weight is not None else bias
    out_dtype = out_dtype or x.dtype
    norm = _map_binding.bevmap_norm(B, pixels, C, groups, stride, eps, act, _code(x.dtype),
                                    _code(out_dtype),
                                    _binding.BEVPOOL_F32 if w_like is None else _code(w_like.dtype))
    size = _map_binding.bevmap_group_norm_workspace(norm, False)
    y = x.new_empty(shape, dtype=out_dtype)
    # kept for the backward, which has no use for the workspace
    stats = x.new_empty((2, B, groups), dtype=torch.float32)
    space = x.new_empty(size, dtype=torch.uint8) if size else None
    mean = stats.data_ptr()
    _call(_map_binding.bevmap_group_norm, index, norm, x.data_ptr(), _ptr(weight), _ptr(bias), y.data_ptr(), mean,
          mean + 4 * B * groups, _ptr(space), size)
    return y, stats, norm


def _layout_of(*tensors):
    return [None if t is None else (t.shape, t.stride(), t.dtype, t.device, t.is_neg()) for t in tensors]


# How tensors lie, to compare with how others do; native for its host time
_layout = _layout_of if _native is None else _native.layout


def _check_saved(index, *expected):
    """What a forward saved, as a hook on saved tensors brought it back: other strides are looked at by the
    callers, anything else is refused."""
    for t, shape, dtype in expected:
        if t is not None and (t.shape != shape or t.dtype != dtype or t.get_device() != index or t.is_neg()):
            _refuse("a saved tensor came back with another size, dtype or device",
                    _binding.BEVPOOL_ERR_SHAPE_MISMATCH)


def _whole(t):
    return t if t is None or t.is_contiguous() else t.contiguous()


def _norm_brought_back(norm, index, shape, x, weight, bias, stats):
    C, w_dtype = norm.channels, _DTYPES[norm.weight_dtype]
    _check_saved(index, (x, shape, _DTYPES[norm.x_dtype]), (weight, (C,), w_dtype), (bias, (C,), w_dtype),
                 (stats, (2, norm.batch, norm.groups), torch.float32))
    norm = type(norm).from_buffer_copy(norm)
    norm.row_stride = _row_stride(x)
    if norm.row_stride is None:
        x, norm.row_stride = x.contiguous(), C
    return norm, x, _whole(weight), _whole(bias), _whole(stats)


def _norm_backward(norm, layout, stats, dy, x, weight, bias, want_weight, want_bias):
    if _layout(x, weight, bias, stats) != layout:
        norm, x, weight, bias, stats = _norm_brought_back(norm, dy.get_device(), dy.shape, x, weight, bias, stats)
    dy = dy.contiguous()
    size = _map_binding.bevmap_group_norm_workspace(norm, True)
    dx = _empty_like(x)
    dw = torch.empty_like(weight) if want_weight else None
    db = torch.empty_like(bias) if want_bias else None
    temp = stats.new_empty(size, dtype=torch.uint8) if size else None
    mean = stats.data_ptr()
    _call(_map_binding.bevmap_group_norm_backward, x.get_device(), norm, dy.data_ptr(), x.data_ptr(), _ptr(weight),
          _ptr(bias), mean, mean + 4 * norm.batch * norm.groups, dx.data_ptr(), _ptr(dw), _ptr(db), _ptr(temp), size)
    return dx, dw, db


def _attend_forward(q, k, v, scale, key_lengths, key_mask, train):
    """out, what its rounding left over, lse (both for the backward), the description and the
    backward's bytes of workspace: what the backward would refuse is refused here."""
    index = _device(q, k, v, key_lengths, key_mask)
    if q.dim() != 4 or k.dim() != 4 or v.dim() != 4:
        _refuse("q, k and v must be 4-D", _binding.BEVPOOL_ERR_SHAPE_MISMATCH)
    B, N, H, D = shape = q.shape
    _, M, K, _ = k.shape
    if k.shape != v.shape or k.shape[0] != B or k.shape[3] != D:
        _refuse(f"q {tuple(shape)}, k {tuple(k.shape)} and v {tuple(v.shape)} do not fit",
                _binding.BEVPOOL_ERR_SHAPE_MISMATCH)
    if B > _MOST or N > _MOST or M > _MOST or H > _MOST or K > _MOST or D > _MOST:
        _refuse(f"q {tuple(shape)}, k {tuple(k.shape)}: too large", _binding.BEVPOOL_ERR_OVERFLOW)
    dtype = q.dtype
    if k.dtype != dtype or v.dtype != dtype:
        _refuse("q, k and v must share a dtype", _binding.BEVPOOL_ERR_UNSUPPORTED_DTYPE)
    qs, ks, vs = q.stride(), k.stride(), v.stride()
    if D > 1 and (qs[3] != 1 or ks[3] != 1 or vs[3] != 1):
        _refuse("the channels of q, k and v must be adjacent")
    if key_lengths is not None:
        if key_lengths.dim() != 1 or key_lengths.shape[0] != B or not key_lengths.is_contiguous():
            _refuse(f"key_lengths must be a contiguous tensor of {B} elements", _binding.BEVPOOL_ERR_SHAPE_MISMATCH)
        if key_lengths.dtype != torch.int32:
            _refuse("key_lengths must be int32", _binding.BEVPOOL_ERR_UNSUPPORTED_DTYPE)
    mask_batch = 0
    if key_mask is not None:
        if tuple(key_mask.shape) != (B, M) or (M > 1 and key_mask.stride(1) != 1):
            _refuse(f"key_mask must be [{B}][{M}] with adjacent elements", _binding.BEVPOOL_ERR_SHAPE_MISMATCH)
        if key_mask.dtype != torch.bool:
            _refuse("key_mask must be bool", _binding.BEVPOOL_ERR_UNSUPPORTED_DTYPE)
        mask_batch = key_mask.stride(0)
    if scale is None:
        scale = D ** -0.5 if D else 1.0
    attend = _map_binding.bevmap_attend(B, N, M, H, K, D, _code(dtype), scale, qs[0], qs[1], qs[2], ks[0], ks[1],
                                        ks[2], vs[0], vs[1], vs[2], mask_batch)
    size = _map_binding.bevmap_attention_workspace(attend, False)
    back_size = _map_binding.bevmap_attention_workspace(attend, True) if train else 0
    out = _empty_like(q)
    low = _empty_like(q) if train and dtype != torch.float32 else None
    lse = q.new_empty((B, H, N), dtype=torch.float32) if train else None
    space = q.new_empty(size, dtype=torch.uint8) if size else None
    _call(_map_binding.bevmap_attention, index, attend, q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(key_lengths),
          _ptr(key_mask), out.data_ptr(), _ptr(low), _ptr(lse), _ptr(space), size)
    return out, low, lse, attend, back_size


def _attend_brought_back(attend, index, q, k, v, key_lengths, key_mask, out, low, lse):
    B, N, M, H, K, D = attend.batch, attend.queries, attend.keys, attend.heads, attend.key_heads, attend.dim
    dtype, asked, states = _DTYPES[attend.dtype], (B, N, H, D), (B, M, K, D)
    _check_saved(index, (q, asked, dtype), (k, states, dtype), (v, states, dtype), (out, asked, dtype),
                 (low, asked, dtype), (lse, (B, H, N), torch.float32), (key_lengths, (B,), torch.int32),
                 (key_mask, (B, M), torch.bool))
    attend = type(attend).from_buffer_copy(attend)
    heads = []
    for name, t in (("q", q), ("k", k), ("v", v)):
        heads.append(t if D <= 1 or t.stride(3) == 1 else t.contiguous())
        for dim, part in enumerate(("batch", "row", "head")):
            setattr(attend, f"{name}_{part}", heads[-1].stride(dim))
    if key_mask is not None:
        key_mask = key_mask if M <= 1 or key_mask.stride(1) == 1 else key_mask.contiguous()
        attend.mask_batch = key_mask.stride(0)
    size = _map_binding.bevmap_attention_workspace(attend, True)
    return attend, size, *heads, _whole(key_lengths), key_mask, _whole(out), _whole(low), _whole(lse)


def _attend_backward(attend, size, layout, dout, q, k, v, key_lengths, key_mask, out, low, lse):
    if _layout(q, k, v, key_lengths, key_mask, out, low, lse) != layout:
        attend, size, q, k, v, key_lengths, key_mask, out, low, lse = _attend_brought_back(
            attend, dout.get_device(), q, k, v, key_lengths, key_mask, out, low, lse)
    dout = dout.contiguous()
    dq, dk, dv = _empty_like(q), _empty_like(k), _empty_like(v)
    temp = q.new_empty(size, dtype=torch.uint8)
    _call(_map_binding.bevmap_attention_backward, q.get_device(), attend, dout.data_ptr(), q.data_ptr(),
          k.data_ptr(), v.data_ptr(), _ptr(key_lengths), _ptr(key_mask), out.data_ptr(), _ptr(low), lse.data_ptr(),
          dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), temp.data_ptr(), size)
    return dq, dk, dv


def _dropout(x, threshold, seed, offset, residual):
    index = _device(x, residual)
    stride = _row_stride(x)
    residual_stride = 0
    if residual is not None:
        residual_stride = _row_stride(residual)
        if residual.shape != x.shape or residual.dtype != x.dtype:
            _refuse("residual must have the shape and dtype of x", _binding.BEVPOOL_ERR_SHAPE_MISMATCH)
    if stride is None or residual_stride is None:
        _refuse("rows of x and residual must be evenly spaced, their elements adjacent")
    y = _empty_like(x)
    columns = x.shape[-1] if x.dim() else 1
    rows = x.numel() // columns if columns else 0
    _call(_map_binding.bevmap_dropout, index, x.data_ptr(), stride, _ptr(residual), residual_stride, y.data_ptr(),
          rows, columns, _code(x.dtype), threshold, seed, offset)
    return y


class _GroupNormAct(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, groups, eps, act, out_dtype):
        _not_traced(False)
        y, stats, norm = _norm_forward(x, groups, weight, bias, eps, act, out_dtype)
        ctx.norm = norm, _layout(x, weight, bias, stats)
        ctx.save_for_backward(x, weight, bias, stats)
        return y

    @staticmethod
    def backward(ctx, dy):
        _first_order_only()
        x, weight, bias, stats = ctx.saved_tensors
        need = ctx.needs_input_grad
        dx, dw, db = _norm_backward(*ctx.norm, stats, dy, x, weight, bias, need[1], need[2])
        return dx if need[0] else None, dw, db, None, None, None, None


class _CrossAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, scale, key_lengths, key_mask):
        _not_traced(False)
        out, low, lse, attend, size = _attend_forward(q, k, v, scale, key_lengths, key_mask, True)
        ctx.attend = attend, size, _layout(q, k, v, key_lengths, key_mask, out, low, lse)
        ctx.save_for_backward(q, k, v, key_lengths, key_mask, out, low, lse)
        return out

    @staticmethod
    def backward(ctx, dout):
        _first_order_only()
        q, k, v, key_lengths, key_mask, out, low, lse = ctx.saved_tensors
        need = ctx.needs_input_grad
        dq, dk, dv = _attend_backward(*ctx.attend, dout, q, k, v, key_lengths, key_mask, out, low, lse)
        return dq if need[0] else None, dk if need[1] else None, dv if need[2] else None, None, None, None


class _DropoutAdd(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, threshold, seed, offset):
        _not_traced(False)
        ctx.draw = threshold, seed, offset
        return _dropout(x, threshold, seed, offset, residual)

    @staticmethod
    def backward(ctx, dy):
        _first_order_only()
        need = ctx.needs_input_grad
        dx = None
        if need[0]:
            dx = _dropout(dy if _row_stride(dy) is not None else dy.contiguous(), *ctx.draw, None)
        return dx, dy if need[1] else None, None, None, None


def _learns(*tensors) -> bool:
    """Whether a call has to go through its autograd function: where a gradient is asked for,
    and while a level of forward-mode differentiation is open, so that a tangent among the
    inputs is refused there (the operators have no forward-mode form) and not dropped."""
    if forward_ad._current_level >= 0:
        return True
    if torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                return True
    return False


def group_norm_act(x, groups, weight=None, bias=None, eps=1e-5, act="none", out_dtype=None):
    """Group norm over a map with an activation, channels last: x [B][...][C]
    (fp32, bf16 or fp16), contiguous or a channel slice of a wider map; returns
    a contiguous map of out_dtype (x's by default).

    Channel c belongs to group c // (C // groups); mean and biased variance are
    those of a sample's group over all its cells; y = act(weight * (x - mean) /
    sqrt(variance + eps) + bias), act "none", "relu", "silu" or "gelu" (through
    erf). weight, bias: [C] of one dtype, or None. Statistics are fp32, y is
    rounded once. Differentiable in x, weight and bias."""
    if _learns(x, weight, bias):
        return _GroupNormAct.apply(x, weight, bias, groups, eps, act, out_dtype)
    _not_traced()
    return _norm_forward(x, groups, weight, bias, eps, act, out_dtype)[0]


def cross_attention(q, k, v, scale=None, key_lengths=None, key_mask=None):
    """Attention of queries to an encoder's states of another length.

    q [B][N][H][D], k and v [B][M][K][D] (fp32, bf16 or fp16, one dtype; any
    strides but for adjacent channels, so views of a packed projection do); H
    is a multiple of K, and head h reads key head h // (H // K); D at most 128.
    Returns [B][N][H][D], contiguous: softmax(scale * q k^T) v, scale by default
    1 / sqrt(D).

    key_lengths: int32 [B], states j >= key_lengths[b] are not in use (values
    are clamped to [0, M]). key_mask: bool [B][M], states with False are not in
    use. States not in use may hold anything, NaN too; they do not reach the
    output, and their gradients are 0. A query without a state in use gets 0.
    Queries and states in use must be finite.
    Scores, statistics and sums are fp32. With bf16 and fp16 the probabilities of
    more than 32 queries to a key head (N * H // K) are rounded to the type for
    their product with v; with fewer, in the backward and with fp32 they are not.
    Few queries over many states (one token in serving) are split over the
    states. Differentiable in q, k and v, bitwise reproducible."""
    if _learns(q, k, v):
        return _CrossAttention.apply(q, k, v, scale, key_lengths, key_mask)
    _not_traced()
    return _attend_forward(q, k, v, scale, key_lengths, key_mask, False)[0]


def dropout_add(x, p, seed, offset=0, residual=None):
    """residual + dropout(x), the mask drawn from (seed, offset) and the element's
    index in x and never stored.

    x (fp32, bf16 or fp16), contiguous or with evenly spaced rows; residual alike
    or None. p in [0, 1] is placed to the nearest 1 / 65536, and kept elements
    are scaled by one over the placed keep probability. seed, offset: integers
    in [0, 2^64); a step that needs another mask takes another offset (a HIP
    graph that captured the call draws the same mask in each replay).
    Differentiable in x and residual: the backward draws the mask again."""
    if not 0.0 <= p <= 1.0:
        _refuse(f"p={p} is outside [0, 1]")
    if not (0 <= seed < 1 << 64 and 0 <= offset < 1 << 64):
        _refuse("seed and offset must be in [0, 2^64)")
    threshold = int(65536 * p + 0.5)
    if _learns(x, residual):
        return _DropoutAdd.apply(x, residual, threshold, seed, offset)
    _not_traced()
    return _dropout(x, threshold, seed, offset, residual)
