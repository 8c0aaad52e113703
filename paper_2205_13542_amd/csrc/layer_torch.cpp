// The operators around attention as calls from Python on torch tensors: the module
// _layer_native, which layer_ops.py documents and wraps. Argument checks, allocations,
// the C ABI's calls and the autograd nodes are here and not in Python because a call on a
// few rows costs its host time: one token's rotary positions take 4.9 us a call here, 8.7
// through ctypes; a training step of the norm of 600 rows 66 instead of 110.
//
// Everything runs on the current stream of its inputs' device, with temporaries from
// torch's allocator. A refusal is a BevpoolError (its class comes from Python), an input
// with a tangent of torch.autograd.forward_ad a NotImplementedError.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/DynamicTypes.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/jit/frontend/tracer.h>

#include <algorithm>
#include <optional>
#include <string>

#include "bevmap.h"

namespace {

using at::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

constexpr int kShapeMismatch = -2;
static_assert(BEVPOOL_ERR_SHAPE_MISMATCH == kShapeMismatch, "");
constexpr int64_t kMost = (int64_t(1) << 31) - 1;   // of a size in the C descriptions
constexpr int64_t kHeldBlock = 32;                  // channels that share an exponent in a checkpoint

struct Refused {
    int code;
    std::string message;
};

[[noreturn]] void refuse(const std::string &message, int code = BEVPOOL_ERR_INVALID_ARG) { throw Refused{code, message}; }

struct Tangent {};

// torch's dispatcher sees nothing of these calls, so that a tracer would keep the result of
// the inputs that it traces with as a constant (of the map operators, an empty tensor that
// nothing fills): refused, under torch.jit.trace, and under make_fx (whose mode is on the dispatcher's stack, or on one of its own ahead of autograd,
// which this key stands for).
void not_traced(bool jit = true) {
    using c10::impl::TorchDispatchModeKey;
    using c10::impl::TorchDispatchModeTLS;
    if ((jit && torch::jit::tracer::isTracing()) ||
        (TorchDispatchModeTLS::any_modes_set() && TorchDispatchModeTLS::get_mode(TorchDispatchModeKey::PROXY)) ||
        c10::impl::tls_local_dispatch_key_set().included_.has(c10::DispatchKey::PreDispatch))
        refuse("the operators cannot be traced: their results would be recorded as constants, or as empty tensors");
}

std::string shape_of(const Tensor &t) { return c10::str("[", c10::Join(", ", t.sizes()), "]"); }

int code_of(at::ScalarType type) {
    if (type == at::kFloat) return BEVPOOL_F32;
    if (type == at::kBFloat16) return BEVPOOL_BF16;
    if (type == at::kHalf) return BEVPOOL_F16;
    refuse(c10::str("dtype ", type), BEVPOOL_ERR_UNSUPPORTED_DTYPE);
}

at::ScalarType type_of(int32_t code) {
    return code == BEVPOOL_F32 ? at::kFloat : code == BEVPOOL_BF16 ? at::kBFloat16 : at::kHalf;
}

void done(int64_t rc) {
    if (rc < 0) throw Refused{int(rc), bevpool_last_error()};
}

const void *ptr(const Tensor &t) { return t.defined() ? t.const_data_ptr() : nullptr; }
void *out(const Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }

template <class... Ts>
void one_device(const Tensor &first, const Ts &...others) {
    if (!first.is_cuda()) refuse("inputs must be device tensors");
    for (const Tensor *t : {&others..., &first})
        if (t->defined()) {
            if (t->device() != first.device()) refuse("all tensors must be on one device");
            if (t->is_neg()) refuse("a view that negates what lies in memory: resolve_neg() first");
        }
}

// Whether a gradient is asked for through a call on these; a tangent among them ends it.
template <class... Ts>
bool learns(const Ts &...tensors) {
    bool any = false;
    for (const Tensor *t : {&tensors...})
        if (t->defined()) {
            if (t->_fw_grad(0).defined()) throw Tangent{};
            any = any || t->requires_grad();
        }
    return any && c10::GradMode::is_enabled();
}

template <class... Ts>
void no_gradient(const char *call, const Ts &...tensors) {
    if (learns(tensors...)) refuse(c10::str(call, " has no gradient: call it under torch.no_grad()"));
}

// The device current, for a call and its allocations, and its current stream.
struct On {
    std::optional<c10::DeviceGuard> guard;
    void *stream;
    explicit On(const Tensor &t) {
        const auto index = t.device().index();
        if (c10::hip::current_device() != index) guard.emplace(t.device());
        stream = c10::hip::getCurrentHIPStream(index).stream();
    }
};

Tensor empty(at::IntArrayRef sizes, at::ScalarType type, const Tensor &like) {
    return at::detail::empty_cuda(sizes, type, like.device(), std::nullopt);
}

struct Rows {
    int64_t rows, columns, stride;
};

// Rows, columns and the row stride of t, its last dimension the columns; whether rows are
// evenly spaced and their elements adjacent.
bool even_rows(const Tensor &t, Rows &r) {
    const int64_t dims = t.dim();
    r = {1, t.size(-1), t.size(-1)};
    for (int64_t i = 0; i + 1 < dims; ++i) r.rows *= t.size(i);
    if (t.is_contiguous()) return true;
    bool even = t.stride(-1) == 1 || r.columns <= 1;
    int64_t step = -1, expect = 0;
    for (int64_t i = dims - 2; even && i >= 0; --i) {
        if (t.size(i) == 1) continue;
        if (step < 0) step = t.stride(i);
        else even = t.stride(i) == expect;
        expect = t.stride(i) * t.size(i);
    }
    if (step >= 0) {
        even = even && step >= r.columns;
        r.stride = step;
    }
    return even;
}
Rows rows_of(const Tensor &t, const char *name) {
    if (t.dim() < 1) refuse(c10::str(name, " must have a channel dimension"), BEVPOOL_ERR_SHAPE_MISMATCH);
    Rows r;
    if (!even_rows(t, r)) refuse(c10::str("rows of ", name, " must be evenly spaced, their channels adjacent"));
    if (r.rows > kMost || r.columns > kMost) refuse(c10::str(name, " ", shape_of(t), ": too large"), BEVPOOL_ERR_OVERFLOW);
    return r;
}

void check_vector(const Tensor &t, int64_t n, const char *name) {
    if (t.defined() && (t.dim() != 1 || t.size(0) != n || !t.is_contiguous()))
        refuse(c10::str(name, " must be a contiguous tensor of ", n, " elements"), BEVPOOL_ERR_SHAPE_MISMATCH);
}

void first_order_only() {
    if (c10::GradMode::is_enabled()) throw std::runtime_error("the map operators have no second derivatives");
}

// t, contiguous and as its memory says.
Tensor whole(const Tensor &t) { return t.is_contiguous() && !t.is_neg() ? t : t.resolve_neg().contiguous(); }

// A description kept from a forward for its backward.
template <class T>
void keep(AutogradContext *ctx, const T &description) {
    ctx->saved_data["d"] = std::string(reinterpret_cast<const char *>(&description), sizeof(T));
}
template <class T>
T kept(AutogradContext *ctx) {
    T description;
    const std::string &bytes = ctx->saved_data["d"].toStringRef();
    memcpy(&description, bytes.data(), sizeof(T));
    return description;
}

// What a forward saved, as the backward gets it: a hook on saved tensors may have brought it
// back with other strides, or as something else.
[[noreturn]] void changed() { refuse("a saved tensor came back with another size, dtype or device", BEVPOOL_ERR_SHAPE_MISMATCH); }
Tensor saved_whole(const Tensor &t, int64_t numel, at::ScalarType type, const Tensor &gradient) {
    if (!t.defined()) return t;
    if (t.numel() != numel || t.scalar_type() != type || t.device() != gradient.device()) changed();
    return whole(t);
}
Tensor saved_rows(const Tensor &t, int64_t rows, int64_t columns, int32_t dtype, const Tensor &gradient, int64_t *stride) {
    if (!t.defined()) return t;
    Rows r;
    if (t.dim() < 1 || t.device() != gradient.device() || code_of(t.scalar_type()) != dtype) changed();
    const bool even = even_rows(t, r) && !t.is_neg();
    if (r.rows != rows || r.columns != columns) changed();
    *stride = even ? r.stride : columns;
    return even ? t : whole(t);
}

// A refusal inside a backward, where no caller of ours catches it.
template <class F>
variable_list in_backward(F body) {
    first_order_only();
    try {
        return body();
    } catch (const Refused &r) {
        throw std::runtime_error(r.message);
    }
}

// ------------------------------------------------------------------ RMS norm

bevmap_rms describe_rms(const Tensor &x, const Tensor &residual, const Tensor &weight, double eps, at::ScalarType out_type) {
    one_device(x, residual, weight);
    const Rows r = rows_of(x, "x");
    bevmap_rms n{};
    n.rows = r.rows;
    n.channels = int32_t(r.columns);
    n.x_stride = r.stride;
    n.residual_stride = r.columns;
    if (residual.defined()) {
        if (residual.sizes() != x.sizes() || residual.scalar_type() != x.scalar_type())
            refuse("residual must have the shape and dtype of x", BEVPOOL_ERR_SHAPE_MISMATCH);
        n.residual_stride = rows_of(residual, "residual").stride;
    }
    check_vector(weight, r.columns, "weight");
    n.x_dtype = code_of(x.scalar_type());
    n.y_dtype = code_of(out_type);
    n.weight_dtype = weight.defined() ? code_of(weight.scalar_type()) : BEVPOOL_F32;
    n.eps = float(eps);
    return n;
}

struct Normed {
    Tensor y, total, rstd;
};
Normed rms_forward(const bevmap_rms &n, const Tensor &x, const Tensor &residual, const Tensor &weight,
                   at::ScalarType out_type, bool train) {
    const On on(x);
    Normed r;
    r.y = empty(x.sizes(), out_type, x);
    if (residual.defined()) r.total = empty(x.sizes(), x.scalar_type(), x);
    if (train) r.rstd = empty({n.rows}, at::kFloat, x);
    done(bevmap_rms_norm(&n, ptr(x), ptr(residual), ptr(weight), out(r.total), out(r.y),
                         static_cast<float *>(out(r.rstd)), on.stream));
    return r;
}

struct RmsNorm : torch::autograd::Function<RmsNorm> {
    // (an undefined tensor is not taken for an argument of a node, an empty optional is)
    static variable_list forward(AutogradContext *ctx, const Tensor &x, const std::optional<Tensor> &maybe_residual,
                                 const std::optional<Tensor> &maybe_weight, double eps, int64_t out_type) {
        const Tensor residual = maybe_residual.value_or(Tensor()), weight = maybe_weight.value_or(Tensor());
        const bevmap_rms n = describe_rms(x, residual, weight, eps, at::ScalarType(out_type));
        const Normed r = rms_forward(n, x, residual, weight, at::ScalarType(out_type), true);
        ctx->set_materialize_grads(false);
        ctx->saved_data["w"] = weight.defined() && weight.requires_grad();
        if (!residual.defined()) {
            ctx->save_for_backward({x, Tensor(), weight, r.rstd});
            keep(ctx, n);
            return {r.y};
        }
        if (x.scalar_type() == at::kFloat) {
            ctx->save_for_backward({r.total, Tensor(), weight, r.rstd});
        } else {
            // the sum of 16-bit numbers, rounded, would take its rounding into the weight's gradient
            ctx->save_for_backward({x, residual, weight, r.rstd});
        }
        keep(ctx, n);
        return {r.y, r.total};
    }

    static variable_list backward(AutogradContext *ctx, variable_list grads) {
        return in_backward([&]() -> variable_list {
            const variable_list saved = ctx->get_saved_variables();
            const bool want = ctx->saved_data["w"].toBool(), added = grads.size() > 1;
            const Tensor dtotal = added && grads[1].defined() ? whole(grads[1]) : Tensor();
            if (!grads[0].defined())        // y was not used: the gradient of a sum
                return {dtotal, dtotal, want ? at::zeros_like(saved[2]) : Tensor(), Tensor(), Tensor()};
            bevmap_rms n = kept<bevmap_rms>(ctx);
            const Tensor dy = whole(grads[0]);
            const On on(dy);
            const Tensor x = saved_rows(saved[0], n.rows, n.channels, n.x_dtype, dy, &n.x_stride);
            const Tensor residual = saved_rows(saved[1], n.rows, n.channels, n.x_dtype, dy, &n.residual_stride);
            const Tensor weight = saved_whole(saved[2], n.channels, type_of(n.weight_dtype), dy);
            const Tensor rstd = saved_whole(saved[3], n.rows, at::kFloat, dy);
            const Tensor dx = empty(x.sizes(), x.scalar_type(), x);
            Tensor dw, space;
            int64_t size = 0;
            if (want) {
                dw = empty(weight.sizes(), weight.scalar_type(), x);
                done(size = bevmap_rms_norm_backward_workspace(&n));
                if (size) space = empty({size}, at::kByte, x);
            }
            done(bevmap_rms_norm_backward(&n, ptr(dy), ptr(dtotal), ptr(x), ptr(residual), ptr(weight),
                                          static_cast<const float *>(ptr(rstd)), out(dx), out(dw), out(space), size,
                                          on.stream));
            return {dx, added ? dx : Tensor(), dw, Tensor(), Tensor()};
        });
    }
};

variable_list rms_norm(const Tensor &x, const Tensor &residual, const Tensor &weight, double eps,
                       std::optional<at::ScalarType> out_type) {
    const at::ScalarType type = out_type.value_or(x.scalar_type());
    auto maybe = [](const Tensor &t) { return t.defined() ? std::optional<Tensor>(t) : std::nullopt; };
    if (learns(x, residual, weight)) return RmsNorm::apply(x, maybe(residual), maybe(weight), eps, int64_t(type));
    const Normed r = rms_forward(describe_rms(x, residual, weight, eps, type), x, residual, weight, type, false);
    if (residual.defined()) return {r.y, r.total};
    return {r.y};
}

variable_list rms_norm_int8(const Tensor &x, const Tensor &residual, const Tensor &weight, double eps) {
    no_gradient(residual.defined() ? "rms_norm_add_int8" : "rms_norm_int8", x, residual, weight);
    const bevmap_rms n = describe_rms(x, residual, weight, eps, x.scalar_type());
    const On on(x);
    const Tensor held = empty(x.sizes(), at::kChar, x);
    const Tensor scale = empty(x.sizes().slice(0, x.dim() - 1), at::kFloat, x);
    const Tensor total = residual.defined() ? empty(x.sizes(), x.scalar_type(), x) : Tensor();
    done(bevmap_rms_norm_int8(&n, ptr(x), ptr(residual), ptr(weight), out(total), static_cast<int8_t *>(out(held)),
                              static_cast<float *>(out(scale)), on.stream));
    if (total.defined()) return {held, scale, total};
    return {held, scale};
}

// ------------------------------------------------------------------ 8-bit integers

variable_list quantize_int8(const Tensor &x) {
    no_gradient("quantize_int8", x);
    one_device(x);
    const Rows r = rows_of(x, "x");
    const int dtype = code_of(x.scalar_type());
    const On on(x);
    const Tensor held = empty(x.sizes(), at::kChar, x);
    const Tensor scale = empty(x.sizes().slice(0, x.dim() - 1), at::kFloat, x);
    done(bevmap_quantize_int8(ptr(x), r.stride, static_cast<int8_t *>(out(held)), static_cast<float *>(out(scale)),
                              r.rows, int32_t(r.columns), dtype, on.stream));
    return {held, scale};
}

Tensor linear_int8(const Tensor &x, const Tensor &x_scale, const Tensor &weight, const Tensor &weight_scale,
                   const Tensor &bias, std::optional<at::ScalarType> out_type) {
    no_gradient("linear_int8", x_scale, weight_scale, bias);
    one_device(x, x_scale, weight, weight_scale, bias);
    if (x.scalar_type() != at::kChar || weight.scalar_type() != at::kChar)
        refuse(c10::str("x and weight must be int8, not ", x.scalar_type(), " and ", weight.scalar_type()),
               BEVPOOL_ERR_UNSUPPORTED_DTYPE);
    const Rows r = rows_of(x, "x");
    if (weight.dim() != 2 || weight.size(1) != r.columns)
        refuse(c10::str("weight must be [N][", r.columns, "], not ", shape_of(weight)), BEVPOOL_ERR_SHAPE_MISMATCH);
    const Rows w = rows_of(weight, "weight");
    if (x_scale.sizes() != x.sizes().slice(0, x.dim() - 1) || !x_scale.is_contiguous())
        refuse("x_scale must be a contiguous tensor of x's shape without its last dimension",
               BEVPOOL_ERR_SHAPE_MISMATCH);
    check_vector(weight_scale, w.rows, "weight_scale");
    check_vector(bias, w.rows, "bias");
    if (x_scale.scalar_type() != at::kFloat || weight_scale.scalar_type() != at::kFloat ||
        (bias.defined() && bias.scalar_type() != at::kFloat))
        refuse("x_scale, weight_scale and bias must be fp32", BEVPOOL_ERR_UNSUPPORTED_DTYPE);
    const at::ScalarType type = out_type.value_or(at::kBFloat16);
    bevmap_linear n{};
    n.rows = r.rows;
    n.channels = int32_t(r.columns);
    n.features = int32_t(w.rows);
    n.x_stride = r.stride;
    n.w_stride = w.stride;
    n.y_dtype = code_of(type);
    const On on(x);
    at::DimVector sizes(x.sizes());
    sizes.back() = w.rows;
    const Tensor y = empty(sizes, type, x);
    done(bevmap_linear_int8(&n, static_cast<const int8_t *>(ptr(x)), static_cast<const float *>(ptr(x_scale)),
                            static_cast<const int8_t *>(ptr(weight)), static_cast<const float *>(ptr(weight_scale)),
                            static_cast<const float *>(ptr(bias)), out(y), on.stream));
    return y;
}

// ------------------------------------------------------------------ rotary positions

bevmap_turn describe_turn(const Tensor &x, const Tensor &positions, const Tensor &frequencies, bool interleaved,
                          double amplitude) {
    one_device(x, positions, frequencies);
    if (x.dim() != 4) refuse("x must be [B][N][H][D]", BEVPOOL_ERR_SHAPE_MISMATCH);
    if (frequencies.dim() != 1 || !frequencies.is_contiguous())
        refuse("frequencies must be a contiguous vector", BEVPOOL_ERR_SHAPE_MISMATCH);
    if (frequencies.scalar_type() != at::kDouble)
        refuse(c10::str("frequencies must be fp64, not ", frequencies.scalar_type()), BEVPOOL_ERR_UNSUPPORTED_DTYPE);
    bevmap_turn n{};
    const at::ScalarType type = positions.scalar_type();
    if (type == at::kInt) n.positions_type = BEVMAP_POSITION_I32;
    else if (type == at::kLong) n.positions_type = BEVMAP_POSITION_I64;
    else if (type == at::kFloat) n.positions_type = BEVMAP_POSITION_F32;
    else refuse(c10::str("positions must be int32, int64 or fp32, not ", type), BEVPOOL_ERR_UNSUPPORTED_DTYPE);
    if (positions.dim() < 2 || positions.dim() > 3 || positions.size(0) != x.size(0) ||
        positions.size(1) != x.size(1) || !positions.is_contiguous())
        refuse(c10::str("positions must be a contiguous tensor [", x.size(0), "][", x.size(1), "] or [", x.size(0),
                        "][", x.size(1), "][axes], not ", shape_of(positions)), BEVPOOL_ERR_SHAPE_MISMATCH);
    const int64_t axes = positions.dim() == 3 ? positions.size(2) : 1, pairs = frequencies.size(0);
    if (std::max({x.size(0), x.size(1), x.size(2), x.size(3), axes, pairs}) > kMost)
        refuse(c10::str("x ", shape_of(x), ": too large"), BEVPOOL_ERR_OVERFLOW);
    if (x.size(3) > 1 && x.stride(3) != 1) refuse("the channels of x must be adjacent");
    n.batch = int32_t(x.size(0));
    n.tokens = int32_t(x.size(1));
    n.heads = int32_t(x.size(2));
    n.dim = int32_t(x.size(3));
    n.pairs = int32_t(pairs);
    n.axes = int32_t(axes);
    n.interleaved = interleaved;
    n.dtype = code_of(x.scalar_type());
    n.amplitude = float(amplitude);
    return n;
}

Tensor turn(bevmap_turn n, const Tensor &x, const Tensor &positions, const Tensor &frequencies, bool backward) {
    const On on(x);
    n.x_batch = x.stride(0);
    n.x_row = x.stride(1);
    n.x_head = x.stride(2);
    const Tensor y = empty(x.sizes(), x.scalar_type(), x);
    done(bevmap_rotary(&n, ptr(x), ptr(positions), static_cast<const double *>(ptr(frequencies)), out(y), backward,
                       on.stream));
    return y;
}

struct Rotary : torch::autograd::Function<Rotary> {
    static Tensor forward(AutogradContext *ctx, const Tensor &x, const Tensor &positions, const Tensor &frequencies,
                          bool interleaved, double amplitude) {
        const bevmap_turn n = describe_turn(x, positions, frequencies, interleaved, amplitude);
        ctx->save_for_backward({positions, frequencies});
        keep(ctx, n);
        return turn(n, x, positions, frequencies, false);
    }
    static variable_list backward(AutogradContext *ctx, variable_list grads) {
        return in_backward([&]() -> variable_list {
            const variable_list saved = ctx->get_saved_variables();
            const Tensor dy = grads[0].stride(3) == 1 ? grads[0].resolve_neg() : whole(grads[0]);
            const bevmap_turn n = kept<bevmap_turn>(ctx);
            const at::ScalarType type = n.positions_type == BEVMAP_POSITION_I32   ? at::kInt
                                        : n.positions_type == BEVMAP_POSITION_I64 ? at::kLong
                                                                                  : at::kFloat;
            const Tensor positions = saved_whole(saved[0], int64_t(n.batch) * n.tokens * n.axes, type, dy);
            const Tensor frequencies = saved_whole(saved[1], n.pairs, at::kDouble, dy);
            return {turn(n, dy, positions, frequencies, true), Tensor(), Tensor(), Tensor(), Tensor()};
        });
    }
};

Tensor rotary(const Tensor &x, const Tensor &positions, const Tensor &frequencies, bool interleaved, double amplitude) {
    if (learns(positions, frequencies)) refuse("positions and frequencies have no gradient");
    if (learns(x)) return Rotary::apply(x, positions, frequencies, interleaved, amplitude);
    return turn(describe_turn(x, positions, frequencies, interleaved, amplitude), x, positions, frequencies, false);
}

// ------------------------------------------------------------------ gated activation

bevmap_gate describe_gate(const Tensor &x, int64_t act) {
    one_device(x);
    const Rows r = rows_of(x, "x");
    if (r.columns < 2 || r.columns % 2)
        refuse(c10::str("x must have two halves, not ", r.columns, " channels"), BEVPOOL_ERR_SHAPE_MISMATCH);
    bevmap_gate n{};
    n.rows = r.rows;
    n.features = int32_t(r.columns / 2);
    n.act = int32_t(act);
    n.dtype = code_of(x.scalar_type());
    n.x_stride = r.stride;
    return n;
}

// y, and what is held of x in 8 bits if asked
variable_list gate_forward(const bevmap_gate &n, const Tensor &x, bool hold) {
    const On on(x);
    at::DimVector sizes(x.sizes());
    sizes.back() = n.features;
    const Tensor y = empty(sizes, x.scalar_type(), x);
    Tensor held, exponents;
    if (hold) {
        held = empty({n.rows, 2, n.features}, at::kChar, x);
        exponents = empty({n.rows, 2, (n.features + kHeldBlock - 1) / kHeldBlock}, at::kByte, x);
    }
    done(bevmap_gated_act(&n, ptr(x), out(y), static_cast<int8_t *>(out(held)), static_cast<uint8_t *>(out(exponents)),
                          on.stream));
    return {y, held, exponents};
}

struct GatedAct : torch::autograd::Function<GatedAct> {
    static Tensor forward(AutogradContext *ctx, const Tensor &x, int64_t act, bool hold) {
        const bevmap_gate n = describe_gate(x, act);
        const variable_list r = gate_forward(n, x, hold);
        ctx->save_for_backward({hold ? Tensor() : x, r[1], r[2]});
        keep(ctx, n);
        return r[0];
    }
    static variable_list backward(AutogradContext *ctx, variable_list grads) {
        return in_backward([&]() -> variable_list {
            const variable_list saved = ctx->get_saved_variables();
            bevmap_gate n = kept<bevmap_gate>(ctx);
            const Tensor dy = whole(grads[0]);
            const On on(dy);
            const int64_t halves = n.rows * 2, blocks = (n.features + kHeldBlock - 1) / kHeldBlock;
            const Tensor x = saved_rows(saved[0], n.rows, 2 * int64_t(n.features), n.dtype, dy, &n.x_stride);
            const Tensor held = saved_whole(saved[1], halves * n.features, at::kChar, dy);
            const Tensor exponents = saved_whole(saved[2], halves * blocks, at::kByte, dy);
            at::DimVector sizes(dy.sizes());
            sizes.back() = 2 * int64_t(n.features);
            const Tensor dx = empty(sizes, dy.scalar_type(), dy);
            done(bevmap_gated_act_backward(&n, ptr(dy), ptr(x), static_cast<const int8_t *>(ptr(held)),
                                           static_cast<const uint8_t *>(ptr(exponents)), out(dx), on.stream));
            return {dx, Tensor(), Tensor()};
        });
    }
};

Tensor gated_act(const Tensor &x, int64_t act, bool hold) {
    if (learns(x)) return GatedAct::apply(x, act, hold);
    return gate_forward(describe_gate(x, act), x, false)[0];
}

// ------------------------------------------------------------------ from Python

PyObject *g_error = nullptr;    // BevpoolError

// While one lives, other Python threads run: a launch may wait for a place in the queue, an
// allocation for the driver.
struct Released {
    PyThreadState *const state = PyEval_SaveThread();
    ~Released() { PyEval_RestoreThread(state); }
};
// body's result, formed without the interpreter's lock
template <class F>
auto released(F body) {
    const Released r;
    return body();
}

// body's result, what it throws as a Python exception
template <class F>
PyObject *guarded(F body) {
    try {
        return body();
    } catch (const Refused &r) {
        PyObject *e = PyObject_CallFunction(g_error ? g_error : PyExc_RuntimeError, "is", r.code, r.message.c_str());
        if (e) {
            PyErr_SetObject(reinterpret_cast<PyObject *>(Py_TYPE(e)), e);
            Py_DECREF(e);
        }
    } catch (const Tangent &) {
        PyErr_SetString(PyExc_NotImplementedError, "the operators around attention have no forward mode");
    } catch (python_error &e) {
        e.restore();
    } catch (const c10::Error &e) {
        PyErr_SetString(std::string(e.what()).find("out of memory") != std::string::npos ? PyExc_MemoryError
                                                                                         : PyExc_RuntimeError,
                        e.what_without_backtrace());
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

Tensor tensor_of(PyObject *o, const char *name) {
    if (!THPVariable_Check(o)) refuse(c10::str(name, " must be a tensor, not ", Py_TYPE(o)->tp_name));
    return THPVariable_Unpack(o);
}
Tensor maybe_tensor(PyObject *o, const char *name) { return o == Py_None ? Tensor() : tensor_of(o, name); }

double number_of(PyObject *o, const char *name) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) {
        PyErr_Clear();
        refuse(c10::str(name, " must be a number, not ", Py_TYPE(o)->tp_name));
    }
    return v;
}

bool truth_of(PyObject *o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw python_error();
    return v != 0;
}

std::optional<at::ScalarType> maybe_type(PyObject *o) {
    if (o == Py_None) return std::nullopt;
    if (!THPDtype_Check(o)) refuse(c10::str("out_dtype must be a dtype, not ", Py_TYPE(o)->tp_name));
    return reinterpret_cast<THPDtype *>(o)->scalar_type;
}

PyObject *wrap(const variable_list &list) {
    PyObject *tuple = PyTuple_New(Py_ssize_t(list.size()));
    if (!tuple) throw python_error();
    for (size_t i = 0; i < list.size(); ++i) PyTuple_SET_ITEM(tuple, Py_ssize_t(i), THPVariable_Wrap(list[i]));
    return tuple;
}

void expect(Py_ssize_t got, Py_ssize_t want) {
    if (got != want) refuse(c10::str("takes ", want, " arguments, not ", got));
}

PyObject *py_rms_norm(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&] {
        not_traced();
        expect(n, 5);
        const Tensor x = tensor_of(a[0], "x"), residual = maybe_tensor(a[1], "residual"), weight = maybe_tensor(a[2], "weight");
        const double eps = number_of(a[3], "eps");
        const auto type = maybe_type(a[4]);
        const variable_list r = released([&] { return rms_norm(x, residual, weight, eps, type); });
        return r.size() == 1 ? THPVariable_Wrap(r[0]) : wrap(r);
    });
}
PyObject *py_rms_norm_int8(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&] {
        not_traced();
        expect(n, 4);
        const Tensor x = tensor_of(a[0], "x"), residual = maybe_tensor(a[1], "residual"), weight = maybe_tensor(a[2], "weight");
        const double eps = number_of(a[3], "eps");
        return wrap(released([&] { return rms_norm_int8(x, residual, weight, eps); }));
    });
}
PyObject *py_quantize_int8(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&] {
        not_traced();
        expect(n, 1);
        const Tensor x = tensor_of(a[0], "x");
        return wrap(released([&] { return quantize_int8(x); }));
    });
}
PyObject *py_linear_int8(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&] {
        not_traced();
        expect(n, 6);
        const Tensor x = tensor_of(a[0], "x"), x_scale = tensor_of(a[1], "x_scale"), weight = tensor_of(a[2], "weight"),
                     weight_scale = tensor_of(a[3], "weight_scale"), bias = maybe_tensor(a[4], "bias");
        const auto type = maybe_type(a[5]);
        return THPVariable_Wrap(released([&] { return linear_int8(x, x_scale, weight, weight_scale, bias, type); }));
    });
}
PyObject *py_rotary(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&] {
        not_traced();
        expect(n, 5);
        const Tensor x = tensor_of(a[0], "x"), positions = tensor_of(a[1], "positions"),
                     frequencies = tensor_of(a[2], "frequencies");
        const bool interleaved = truth_of(a[3]);
        const double amplitude = number_of(a[4], "amplitude");
        return THPVariable_Wrap(released([&] { return rotary(x, positions, frequencies, interleaved, amplitude); }));
    });
}
PyObject *py_gated_act(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&] {
        not_traced();
        expect(n, 3);
        const Tensor x = tensor_of(a[0], "x");
        const int64_t act = int64_t(number_of(a[1], "act"));
        const bool hold = truth_of(a[2]);
        return THPVariable_Wrap(released([&] { return gated_act(x, act, hold); }));
    });
}
// y and the copy in 8 bits, as a training step keeps it
PyObject *py_gated_act_held(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&] {
        not_traced();
        expect(n, 2);
        const Tensor x = tensor_of(a[0], "x");
        no_gradient("gated_act_held", x);
        const int64_t act = int64_t(number_of(a[1], "act"));
        return wrap(released([&] { return gate_forward(describe_gate(x, act), x, true); }));
    });
}
// How tensors (or None) lie: sizes, strides, types and devices as bytes, to compare with others
PyObject *py_layout(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&] {
        c10::SmallVector<int64_t, 96> lie;
        for (Py_ssize_t i = 0; i < n; ++i) {
            if (a[i] == Py_None) {
                lie.push_back(-1);
                continue;
            }
            const Tensor t = tensor_of(a[i], "a tensor");
            lie.append({t.dim(), int64_t(t.scalar_type()), int64_t(t.device().type()), t.device().index(), t.is_neg()});
            lie.append(t.sizes().begin(), t.sizes().end());
            lie.append(t.strides().begin(), t.strides().end());
        }
        return PyBytes_FromStringAndSize(reinterpret_cast<const char *>(lie.data()), Py_ssize_t(lie.size() * sizeof(int64_t)));
    });
}
// not_traced(False): by torch.jit.trace the call may be
PyObject *py_not_traced(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        not_traced(n < 1 || truth_of(a[0]));
        Py_RETURN_NONE;
    });
}
PyObject *py_set_error(PyObject *, PyObject *type) {
    Py_XDECREF(g_error);
    Py_INCREF(type);
    g_error = type;
    Py_RETURN_NONE;
}

#define FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_##name)), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {FAST(rms_norm),    FAST(rms_norm_int8), FAST(quantize_int8),    FAST(linear_int8),
                           FAST(rotary),      FAST(gated_act),     FAST(gated_act_held), FAST(layout),
                           FAST(not_traced),
                           {"set_error", py_set_error, METH_O, nullptr},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_layer_native", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__layer_native() { return PyModule_Create(&g_module); }
