// What a training step has beside its layers (layers.py and optim.py hold the Python side): root-mean-square norm with the
// residual's addition and the cross entropy of a linear layer, each forward and backward one C++ function with one autograd
// node, and the orthogonalised update.
//
// No device code here; all work goes through the C ABI of include/da_training.h.
#include "native_operands.h"

#include "da_training.h"

namespace da_native {
namespace {

int64_t rows_of(const Tensor& x) {
    int64_t rows = 1;
    for (int64_t i = 0; i + 1 < x.dim(); ++i) rows *= x.size(i);
    return rows;
}
int64_t row_pitch(const Tensor& t, const Tensor& m) { return t.dim() == 1 ? t.size(0) : pitch(m); }

int param_dtype(const Tensor& w, const char* what) { return w.defined() ? dtype_of(w, what) : DA_F32; }
Tensor whole(const Tensor& t) { return t.defined() ? t.resolve_neg().contiguous() : t; }

// ------------------------------------------------------------------------------------------
// root-mean-square norm
// ------------------------------------------------------------------------------------------
void rms_check(const Tensor& x, const Tensor& w, const Tensor& residual) {
    on_gpu(x, "x");
    dtype_of(x, "x");
    if (x.dim() < 1) throw py::value_error("x must have a last axis of channels");
    if (w.defined()) {
        on_device_of(x, w, "weight");
        dtype_of(w, "weight");
        if (w.dim() != 1 || w.size(0) != x.size(-1)) throw py::value_error("weight must hold one number a channel");
    }
    if (residual.defined()) {
        on_device_of(x, residual, "residual");
        if (residual.scalar_type() != x.scalar_type()) throw py::type_error("residual must have the type of x");
        if (!residual.sizes().equals(x.sizes())) throw py::value_error("residual must have the shape of x");
    }
}

struct RmsResult {
    Tensor y, sum, scale;        // scale: y is in e4m3
};

RmsResult rms_forward(const Tensor& x, const Tensor& weight, const Tensor& residual, double eps, bool eight) {
    rms_check(x, weight, residual);
    c10::DeviceGuard guard(x.device());
    const Tensor m = as_rows(x), r = residual.defined() ? as_rows(residual) : residual, w = whole(weight);
    const int dt = dtype_of(x, "x");
    const int64_t rows = rows_of(x), channels = x.size(-1);
    RmsResult out;
    out.y = at::empty(x.sizes(), eight ? x.options().dtype(at::kFloat8_e4m3fn) : x.options());
    if (r.defined()) out.sum = at::empty(x.sizes(), x.options());
    const int64_t ldr = r.defined() ? row_pitch(residual, r) : 0;
    if (eight) {
        out.scale = at::empty(x.sizes().slice(0, x.dim() - 1), x.options().dtype(at::kFloat));
        check(da_rms_norm_e4m3(dt, rows, channels, data<void>(m), row_pitch(x, m), data<void>(r), ldr, data<void>(w),
                               param_dtype(w, "weight"), (float)eps, data<void>(out.sum), data<void>(out.y), data<float>(out.scale),
                               stream_of(x)));
    } else {
        check(da_rms_norm(dt, rows, channels, data<void>(m), row_pitch(x, m), data<void>(r), ldr, data<void>(w), param_dtype(w, "weight"),
                          (float)eps, data<void>(out.sum), data<void>(out.y), stream_of(x)));
    }
    return out;
}

// (dx, dw); dy and dsum may be undefined
std::pair<Tensor, Tensor> rms_backward(const Tensor& dy, const Tensor& dsum, const Tensor& s, const Tensor& weight, double eps, bool need_x,
                                       bool need_w) {
    rms_check(s, weight, Tensor());
    for (const Tensor* t : {&dy, &dsum}) {
        if (!t->defined()) continue;
        on_device_of(s, *t, "a gradient");
        if (!t->sizes().equals(s.sizes()) || t->scalar_type() != s.scalar_type()) throw py::value_error("gradients must be like the results");
    }
    c10::DeviceGuard guard(s.device());
    const Tensor m = as_rows(s), d = dy.defined() ? as_rows(dy) : dy, e = dsum.defined() ? as_rows(dsum) : dsum, w = whole(weight);
    const int dt = dtype_of(s, "x");
    const int64_t rows = rows_of(s), channels = s.size(-1);
    Tensor dx, dw;
    if (need_x) dx = at::empty(s.sizes(), s.options());
    if (need_w) dw = at::empty(w.sizes(), w.options());
    size_t bytes = 0;
    if (need_w) check(da_rms_norm_workspace(dt, rows, channels, &bytes));
    const Tensor ws = scratch(bytes, s);
    check(da_rms_norm_backward(dt, rows, channels, data<void>(m), row_pitch(s, m), data<void>(d), d.defined() ? row_pitch(dy, d) : 0,
                               data<void>(e), e.defined() ? row_pitch(dsum, e) : 0, data<void>(w), param_dtype(w, "weight"), (float)eps,
                               data<void>(dx), data<void>(dw), data<void>(ws), bytes, stream_of(s)));
    return {dx, dw};
}

struct RmsNormBackward : torch::autograd::Node {
    SavedVariable s, w;          // s: the sum, which is this node's own result, or x
    double eps = 0.0;
    bool own_sum = false;

    void release_variables() override {
        std::lock_guard<std::mutex> lk(mutex_);
        s.reset_data();
        w.reset_data();
    }
    variable_list apply(variable_list&& grads) override {
        return in_backward([&] { return gradients(grads); });
    }
    // of x, the residual and the weight
    variable_list gradients(const variable_list& grads) {
        const Tensor dy = grads[0], dsum = own_sum ? grads[1] : Tensor();
        if (!dy.defined() && !dsum.defined()) return variable_list(3);
        Tensor S, W;
        {
            std::lock_guard<std::mutex> lk(mutex_);
            S = own_sum ? s.unpack(shared_from_this()) : s.unpack();
            W = w.unpack();
        }
        const bool x = task_should_compute_output(0), r = own_sum && task_should_compute_output(1);
        std::pair<Tensor, Tensor> got;
        {
            at::AutoDispatchBelowADInplaceOrView below;
            got = rms_backward(dy, dsum, S, W, eps, x || r, W.defined() && task_should_compute_output(2));
        }
        return once({x ? got.first : Tensor(), r ? got.first : Tensor(), got.second}, "rms_norm", {dy, dsum, S, W});
    }
    std::string name() const override { return "RmsNormBackward"; }
};

// (y, sum); sum is undefined without a residual
std::pair<Tensor, Tensor> rms_norm(const Tensor& x, const Tensor& w, const Tensor& residual, double eps) {
    const bool train = at::GradMode::is_enabled() && (wants_grad(x) || wants_grad(w) || wants_grad(residual));
    RmsResult out;
    {
        at::AutoDispatchBelowADInplaceOrView below;
        out = rms_forward(x, w, residual, eps, false);
    }
    if (train) {
        auto node = std::shared_ptr<RmsNormBackward>(new RmsNormBackward(), torch::autograd::deleteNode);
        node->eps = eps;
        node->own_sum = residual.defined();
        node->set_next_edges(torch::autograd::collect_next_edges(x, residual, w));
        torch::autograd::set_history(out.y, node);
        if (node->own_sum) torch::autograd::set_history(out.sum, node);
        node->s = node->own_sum ? SavedVariable(out.sum, true) : SavedVariable(x, false);
        node->w = SavedVariable(w, false);
    }
    return {out.y, out.sum};
}

// ------------------------------------------------------------------------------------------
// cross entropy of a linear layer
// ------------------------------------------------------------------------------------------
struct CeSizes {
    int64_t rows, d, classes;
};

CeSizes ce_check(const Tensor& x, const Tensor& w, const Tensor& bias) {
    on_gpu(x, "x");
    dtype_of(x, "x");
    if (x.dim() < 1) throw py::value_error("x must have a last axis");
    on_device_of(x, w, "weight");
    if (w.scalar_type() != x.scalar_type()) throw py::type_error("weight must have the type of x");
    if (w.dim() != 2 || w.size(0) != x.size(-1)) throw py::value_error("sizes do not match: x (..., d), weight (d, classes)");
    if (bias.defined()) {
        on_device_of(x, bias, "bias");
        dtype_of(bias, "bias");
        if (bias.dim() != 1 || bias.size(0) != w.size(1)) throw py::value_error("bias must hold one number a class");
    }
    return {rows_of(x), x.size(-1), w.size(1)};
}

// The loss, and what the backward pass reads
std::pair<Tensor, Tensor> ce_forward(const Tensor& x, const Tensor& weight, const Tensor& bias, const Tensor& target, int reduction) {
    const CeSizes n = ce_check(x, weight, bias);
    if (target.scalar_type() != at::kInt && target.scalar_type() != at::kLong) throw py::type_error("target must be int32 or int64");
    on_device_of(x, target, "target");
    if (!target.sizes().equals(x.sizes().slice(0, x.dim() - 1))) throw py::value_error("target must hold one class a row of x");
    c10::DeviceGuard guard(x.device());
    const Tensor m = as_rows(x), w = whole(weight), b = whole(bias), t = target.contiguous();
    const int dt = dtype_of(x, "x");
    size_t keep = 0, fwd = 0, bwd = 0;
    check(da_linear_cross_entropy_sizes(dt, n.rows, n.d, n.classes, &keep, &fwd, &bwd));
    const Tensor stats = scratch(keep, x), ws = scratch(fwd, x);
    const Tensor loss = reduction == DA_LOSS_ROWS ? at::empty(target.sizes(), x.options().dtype(at::kFloat))
                                                  : at::empty({}, x.options().dtype(at::kFloat));
    check(da_linear_cross_entropy(dt, n.rows, n.d, n.classes, data<void>(m), row_pitch(x, m), data<void>(w), data<void>(b),
                                  param_dtype(b, "bias"), data<void>(t), t.scalar_type() == at::kLong, reduction, data<float>(loss),
                                  data<void>(stats), data<void>(ws), fwd, stream_of(x)));
    return {loss, stats};
}

// of x, the weight and the bias
variable_list ce_backward(const Tensor& dloss, const Tensor& x, const Tensor& weight, const Tensor& bias, const Tensor& stats, int reduction,
                          bool need_x, bool need_w, bool need_b) {
    const CeSizes n = ce_check(x, weight, bias);
    const int64_t numbers = reduction == DA_LOSS_ROWS ? n.rows : 1;
    if (dloss.numel() != numbers || dloss.scalar_type() != at::kFloat) throw py::value_error("the loss's gradient must be float32 and like the loss");
    on_device_of(x, dloss, "the loss's gradient");
    c10::DeviceGuard guard(x.device());
    const Tensor m = as_rows(x), w = whole(weight), b = whole(bias), d = dloss.resolve_neg().reshape({numbers});
    const int dt = dtype_of(x, "x");
    size_t keep = 0, fwd = 0, bwd = 0;
    check(da_linear_cross_entropy_sizes(dt, n.rows, n.d, n.classes, &keep, &fwd, &bwd));
    if ((size_t)stats.numel() < keep) throw py::value_error("stats do not belong to these sizes");
    variable_list out(3);
    if (need_x) out[0] = at::empty(x.sizes(), x.options());
    if (need_w) out[1] = at::empty(w.sizes(), w.options());
    if (need_b) out[2] = at::empty(b.sizes(), b.options());
    const Tensor ws = scratch(bwd, x);
    check(da_linear_cross_entropy_backward(dt, n.rows, n.d, n.classes, data<void>(m), row_pitch(x, m), data<void>(w), data<void>(b),
                                           param_dtype(b, "bias"), reduction, data<void>(stats), data<float>(d),
                                           numbers > 1 ? d.stride(0) : 1, data<void>(out[0]), data<void>(out[1]), data<void>(out[2]),
                                           data<void>(ws), bwd, stream_of(x)));
    return out;
}

struct LinearCrossEntropyBackward : torch::autograd::Node {
    SavedVariable x, w, b, stats;
    int reduction = DA_LOSS_MEAN;

    void release_variables() override {
        std::lock_guard<std::mutex> lk(mutex_);
        x.reset_data();
        w.reset_data();
        b.reset_data();
        stats.reset_data();
    }
    variable_list apply(variable_list&& grads) override {
        return in_backward([&] { return gradients(grads); });
    }
    variable_list gradients(const variable_list& grads) {
        if (!grads[0].defined()) return variable_list(3);
        Tensor X, W, B, S;
        {
            std::lock_guard<std::mutex> lk(mutex_);
            X = x.unpack();
            W = w.unpack();
            B = b.unpack();
            S = stats.unpack();
        }
        variable_list result;
        {
            at::AutoDispatchBelowADInplaceOrView below;
            result = ce_backward(grads[0], X, W, B, S, reduction, task_should_compute_output(0), task_should_compute_output(1),
                                 B.defined() && task_should_compute_output(2));
        }
        return once(std::move(result), "linear_cross_entropy", {grads[0], X, W, B});
    }
    std::string name() const override { return "LinearCrossEntropyBackward"; }
};

Tensor linear_cross_entropy(const Tensor& x, const Tensor& w, const Tensor& b, const Tensor& target, int reduction) {
    const bool train = at::GradMode::is_enabled() && (wants_grad(x) || wants_grad(w) || wants_grad(b));
    std::pair<Tensor, Tensor> out;
    {
        at::AutoDispatchBelowADInplaceOrView below;
        out = ce_forward(x, w, b, target, reduction);
    }
    if (train) {
        auto node = std::shared_ptr<LinearCrossEntropyBackward>(new LinearCrossEntropyBackward(), torch::autograd::deleteNode);
        node->reduction = reduction;
        node->stats = SavedVariable(out.second, false);
        node->x = SavedVariable(x, false);
        node->w = SavedVariable(w, false);
        node->b = SavedVariable(b, false);
        node->set_next_edges(torch::autograd::collect_next_edges(x, w, b));
        torch::autograd::set_history(out.first, node);
    }
    return out.first;
}

// ------------------------------------------------------------------------------------------
// orthogonalised update
// ------------------------------------------------------------------------------------------
Tensor orthogonalise(const Tensor& update, int64_t steps, const std::vector<double>& coefficients, double eps) {
    on_gpu(update, "update");
    const int dt = dtype_of(update, "update");
    if (update.dim() < 2) throw py::value_error("update must have two axes at least (rows, columns)");
    if ((int64_t)coefficients.size() != 3 * steps) throw py::value_error("three coefficients to a step");
    at::AutoDispatchBelowADInplaceOrView below;
    c10::DeviceGuard guard(update.device());
    const int64_t rows = update.size(-2), cols = update.size(-1);
    int64_t batch = 1;
    for (int64_t i = 0; i + 2 < update.dim(); ++i) batch *= update.size(i);
    Tensor g = update.resolve_neg().reshape({batch, rows, cols});
    if ((cols > 1 && g.stride(2) != 1) || (rows > 1 && g.stride(1) < cols) || (batch > 1 && g.stride(0) < 0)) g = g.contiguous();
    Tensor out = at::empty(update.sizes(), update.options());
    const std::vector<float> c(coefficients.begin(), coefficients.end());
    size_t bytes = 0;
    check(da_orthogonalise_workspace(dt, batch, rows, cols, (int)steps, &bytes));
    const Tensor ws = scratch(bytes, update);
    check(da_orthogonalise(dt, batch, rows, cols, data<void>(g), rows > 1 ? g.stride(1) : cols, batch > 1 ? g.stride(0) : 0, (int)steps,
                           c.data(), (float)eps, data<void>(out), data<void>(ws), bytes, stream_of(update)));
    return out;
}

typedef std::optional<Tensor> Maybe;
Maybe maybe(const Tensor& t) { return t.defined() ? Maybe(t) : std::nullopt; }

}  // namespace

void bind_training(py::module_& mod) {
    using release = py::call_guard<py::gil_scoped_release>;
    mod.def("rms_norm", [](const Tensor& x, const Maybe& w, const Maybe& residual, double eps) {
        const auto out = rms_norm(x, w.value_or(Tensor()), residual.value_or(Tensor()), eps);
        return std::make_tuple(out.first, maybe(out.second));
    }, release());
    mod.def("rms_norm_forward", [](const Tensor& x, const Maybe& w, const Maybe& residual, double eps) {
        at::AutoDispatchBelowADInplaceOrView below;
        const RmsResult out = rms_forward(x, w.value_or(Tensor()), residual.value_or(Tensor()), eps, false);
        return std::make_tuple(out.y, maybe(out.sum));
    }, release());
    mod.def("rms_norm_backward", [](const Maybe& dy, const Maybe& dsum, const Tensor& s, const Maybe& w, double eps) {
        at::AutoDispatchBelowADInplaceOrView below;
        const auto g = rms_backward(dy.value_or(Tensor()), dsum.value_or(Tensor()), s, w.value_or(Tensor()), eps, true, w.has_value());
        return std::make_tuple(g.first, maybe(g.second));
    }, release());
    mod.def("rms_norm_e4m3", [](const Tensor& x, const Maybe& w, const Maybe& residual, double eps) {
        at::AutoDispatchBelowADInplaceOrView below;
        const RmsResult out = rms_forward(x, w.value_or(Tensor()), residual.value_or(Tensor()), eps, true);
        return std::make_tuple(out.y, out.scale, maybe(out.sum));
    }, release());
    mod.def("linear_cross_entropy", [](const Tensor& x, const Tensor& w, const Maybe& b, const Tensor& target, int reduction) {
        return linear_cross_entropy(x, w, b.value_or(Tensor()), target, reduction);
    }, release());
    mod.def("linear_cross_entropy_forward", [](const Tensor& x, const Tensor& w, const Maybe& b, const Tensor& target, int reduction) {
        at::AutoDispatchBelowADInplaceOrView below;
        return ce_forward(x, w, b.value_or(Tensor()), target, reduction);
    }, release());
    mod.def("linear_cross_entropy_backward",
            [](const Tensor& dloss, const Tensor& x, const Tensor& w, const Maybe& b, const Tensor& stats, int reduction) {
                at::AutoDispatchBelowADInplaceOrView below;
                const auto g = ce_backward(dloss, x, w, b.value_or(Tensor()), stats, reduction, true, true, b.has_value());
                return std::make_tuple(g[0], g[1], maybe(g[2]));
            }, release());
    mod.def("orthogonalise", &orthogonalise, release());
}

}  // namespace da_native
