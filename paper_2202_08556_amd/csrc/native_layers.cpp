// Layers around an aggregation (layers.py holds their Python side): group norm with an activation, the gated
// feed-forward block and the loss of a distillation, each forward and backward one C++ function with one autograd
// node.  On small inputs the device needs 5 to 20 us for one of them; the same in Python would set the pace.
//
// No device code here; all work goes through the C ABI of include/da_layers.h.
#include "native_common.h"

#include <torch/csrc/autograd/functions/basic_ops.h>

#include <array>

#include "da_layers.h"

namespace da_native {
namespace {

using torch::autograd::SavedVariable;
using torch::autograd::variable_list;

int dtype_of(const Tensor& t, const char* what) {
    if (t.scalar_type() == at::kFloat) return DA_F32;
    if (t.scalar_type() == at::kBFloat16) return DA_BF16;
    throw py::type_error(std::string(what) + " must be float32 or bfloat16");
}

void on_device_of(const Tensor& x, const Tensor& t, const char* what) {
    if (t.defined() && t.device() != x.device()) throw py::value_error(std::string(what) + " must be on the device of the input");
}

void on_gpu(const Tensor& x, const char* what) {
    if (!x.is_cuda()) throw py::value_error(std::string(what) + " must live on the GPU");
}

// The last axis as columns, all others as rows: neighbouring columns, rows at one distance
Tensor as_rows(const Tensor& t) {
    const int64_t n = t.size(-1);
    Tensor m = t.dim() == 2 ? t.resolve_neg() : t.resolve_neg().reshape({n ? t.numel() / n : t.numel(), n});
    if (n > 1 && m.stride(1) != 1) return m.contiguous();
    if (m.size(0) > 1 && m.stride(0) < n) return m.contiguous();
    return m;
}
int64_t pitch(const Tensor& m) { return m.size(0) > 1 ? m.stride(0) : m.size(1); }

Tensor scratch(size_t bytes, const Tensor& like) {
    return bytes ? at::empty({(int64_t)bytes}, like.options().dtype(at::kByte)) : Tensor();
}

// Gradients of gradients are not provided: asked for, they raise instead of coming out as zero.
variable_list once(variable_list&& grads, const char* what, const variable_list& of) {
    if (!at::GradMode::is_enabled()) return std::move(grads);
    bool any = false;
    for (const Tensor& t : of) any = any || wants_grad(t);
    if (!any) return std::move(grads);
    for (Tensor& g : grads) {
        if (!g.defined()) continue;
        torch::autograd::edge_list edges;
        for (const Tensor& t : of)
            if (wants_grad(t)) edges.push_back(torch::autograd::impl::gradient_edge(t));
        auto node = std::shared_ptr<torch::autograd::Error>(
            new torch::autograd::Error(std::string(what) + ": the gradient cannot be differentiated again", std::move(edges)),
            torch::autograd::deleteNode);
        torch::autograd::set_history(g, node);
    }
    return std::move(grads);
}

// ------------------------------------------------------------------------------------------
// group norm
// ------------------------------------------------------------------------------------------
struct NormArgs {
    int64_t groups;
    double eps;
    int act;
    Tensor offsets;              // int32, contiguous; undefined: samples by the second to last axis
};

struct NormSizes {
    int64_t rows, samples, channels;
};

NormSizes norm_sizes(const Tensor& x, const Tensor& w, const Tensor& b, const NormArgs& a) {
    on_gpu(x, "x");
    dtype_of(x, "x");
    if (x.dim() < 2) throw py::value_error("x must have at least two axes (rows, channels)");
    NormSizes n{0, 0, x.size(-1)};
    if (a.groups < 1 || n.channels % a.groups != 0) throw py::value_error("channels must be a multiple of groups");
    n.rows = 1;
    for (int64_t i = 0; i + 1 < x.dim(); ++i) n.rows *= x.size(i);
    if (a.offsets.defined()) {
        if (x.dim() != 2) throw py::value_error("with offsets x must be (rows, channels)");
        if (a.offsets.scalar_type() != at::kInt) throw py::type_error("offsets must be int32");
        if (a.offsets.dim() != 1 || a.offsets.size(0) < 1) throw py::value_error("offsets must hold samples + 1 numbers");
        on_device_of(x, a.offsets, "offsets");
        n.samples = a.offsets.size(0) - 1;
        if (n.samples == 0 && n.rows > 0) throw py::value_error("offsets must hold samples + 1 numbers");
    } else {
        n.samples = x.size(-2) ? n.rows / x.size(-2) : 0;
    }
    for (const auto& p : {std::make_pair(&w, "weight"), std::make_pair(&b, "bias")}) {
        if (!p.first->defined()) continue;
        on_device_of(x, *p.first, p.second);
        dtype_of(*p.first, p.second);
        if (p.first->dim() != 1 || p.first->size(0) != n.channels) throw py::value_error(std::string(p.second) + " must hold one number a channel");
    }
    if (w.defined() && b.defined() && w.scalar_type() != b.scalar_type()) throw py::type_error("weight and bias must have one type");
    return n;
}

int norm_param_dtype(const Tensor& w, const Tensor& b) {
    return w.defined() ? dtype_of(w, "weight") : b.defined() ? dtype_of(b, "bias") : DA_F32;
}

// y, and the statistics that the backward pass wants (undefined without `train` or where it wants none)
std::pair<Tensor, Tensor> norm_forward(const Tensor& x, const Tensor& weight, const Tensor& bias, const NormArgs& a, bool train) {
    const NormSizes n = norm_sizes(x, weight, bias, a);
    c10::DeviceGuard guard(x.device());
    const Tensor m = as_rows(x), w = weight.defined() ? weight.resolve_neg().contiguous() : weight,
                 b = bias.defined() ? bias.resolve_neg().contiguous() : bias;
    const int dt = dtype_of(x, "x");
    Tensor y = at::empty(x.sizes(), x.options()), stats;
    size_t keep = 0, fwd = 0, bwd = 0;
    check(da_group_norm_sizes(dt, n.rows, n.samples, a.offsets.defined(), n.channels, a.groups, train, &keep, &fwd, &bwd));
    if (keep) stats = at::empty({(int64_t)keep}, x.options().dtype(at::kFloat));
    const Tensor ws = scratch(fwd, x);
    check(da_group_norm(dt, n.rows, n.samples, data<int32_t>(a.offsets), n.channels, a.groups, data<void>(m), pitch(m), data<void>(w),
                        data<void>(b), norm_param_dtype(w, b), (float)a.eps, a.act, data<void>(y), data<float>(stats), data<void>(ws),
                        fwd, stream_of(x)));
    return {y, stats};
}

variable_list norm_backward(const Tensor& dy, const Tensor& x, const Tensor& weight, const Tensor& bias, const Tensor& stats,
                            const NormArgs& a, bool need_w, bool need_b) {
    const NormSizes n = norm_sizes(x, weight, bias, a);
    if (!dy.sizes().equals(x.sizes()) || dy.scalar_type() != x.scalar_type()) throw py::value_error("dy must be like x");
    on_device_of(x, dy, "dy");
    c10::DeviceGuard guard(x.device());
    const Tensor m = as_rows(x), d = as_rows(dy), w = weight.defined() ? weight.resolve_neg().contiguous() : weight,
                 b = bias.defined() ? bias.resolve_neg().contiguous() : bias;
    const int dt = dtype_of(x, "x");
    Tensor dx = at::empty(x.sizes(), x.options()), dw, db;
    if (need_w) dw = at::empty(w.sizes(), w.options());
    if (need_b) db = at::empty(b.sizes(), b.options());
    size_t keep = 0, fwd = 0, bwd = 0;
    check(da_group_norm_sizes(dt, n.rows, n.samples, a.offsets.defined(), n.channels, a.groups, 1, &keep, &fwd, &bwd));
    const Tensor ws = scratch(bwd, x);
    check(da_group_norm_backward(dt, n.rows, n.samples, data<int32_t>(a.offsets), n.channels, a.groups, data<void>(m), pitch(m),
                                 data<void>(d), pitch(d), data<void>(w), data<void>(b), norm_param_dtype(w, b), (float)a.eps, a.act,
                                 data<float>(stats), data<void>(dx), data<void>(dw), data<void>(db), data<void>(ws), bwd,
                                 stream_of(x)));
    return {dx, dw, db};
}

struct GroupNormBackward : torch::autograd::Node {
    SavedVariable x, w, b, offsets, stats;
    NormArgs args;               // without offsets

    void release_variables() override {
        std::lock_guard<std::mutex> lk(mutex_);
        x.reset_data();
        w.reset_data();
        b.reset_data();
        offsets.reset_data();
        stats.reset_data();
    }
    variable_list apply(variable_list&& grads) override {
        return in_backward([&] { return gradients(grads); });
    }
    variable_list gradients(const variable_list& grads) {
        if (!grads[0].defined()) return variable_list(3);
        Tensor X, W, B, S;
        NormArgs a = args;
        {
            std::lock_guard<std::mutex> lk(mutex_);
            X = x.unpack();
            W = w.unpack();
            B = b.unpack();
            a.offsets = offsets.unpack();
            S = stats.unpack();
        }
        variable_list result;
        {
            at::AutoDispatchBelowADInplaceOrView below;
            result = norm_backward(grads[0], X, W, B, S, a, W.defined() && task_should_compute_output(1),
                                   B.defined() && task_should_compute_output(2));
        }
        if (!task_should_compute_output(0)) result[0] = Tensor();
        return once(std::move(result), "group_norm", {grads[0], X, W, B});
    }
    std::string name() const override { return "GroupNormBackward"; }
};

NormArgs norm_args(int64_t groups, double eps, int act, const std::optional<Tensor>& offsets) {
    NormArgs a{groups, eps, act, Tensor()};
    if (offsets) a.offsets = offsets->contiguous();
    return a;
}

Tensor group_norm(const Tensor& x, int64_t groups, const std::optional<Tensor>& weight, const std::optional<Tensor>& bias, double eps,
                  int act, const std::optional<Tensor>& offsets) {
    const Tensor w = weight.value_or(Tensor()), b = bias.value_or(Tensor());
    const NormArgs a = norm_args(groups, eps, act, offsets);
    const bool train = at::GradMode::is_enabled() && (wants_grad(x) || wants_grad(w) || wants_grad(b));
    std::pair<Tensor, Tensor> out;
    {
        at::AutoDispatchBelowADInplaceOrView below;
        out = norm_forward(x, w, b, a, train);
    }
    if (train) {
        auto node = std::shared_ptr<GroupNormBackward>(new GroupNormBackward(), torch::autograd::deleteNode);
        node->args = NormArgs{a.groups, a.eps, a.act, Tensor()};
        node->offsets = SavedVariable(a.offsets, false);
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
// distillation
// ------------------------------------------------------------------------------------------
struct DistillArgs {
    Tensor index, top;           // rows x best, contiguous
    double temperature;
};

void distill_check(const Tensor& z, const DistillArgs& a) {
    on_gpu(z, "logits");
    dtype_of(z, "logits");
    if (z.dim() < 1) throw py::value_error("logits must have a last axis of classes");
    if (a.index.scalar_type() != at::kInt && a.index.scalar_type() != at::kLong) throw py::type_error("top_index must be int32 or int64");
    dtype_of(a.top, "top_logits");
    on_device_of(z, a.index, "top_index");
    on_device_of(z, a.top, "top_logits");
    if (a.index.dim() != z.dim() || !a.index.sizes().equals(a.top.sizes()) ||
        !a.index.sizes().slice(0, z.dim() - 1).equals(z.sizes().slice(0, z.dim() - 1)))
        throw py::value_error("top_index and top_logits must have the rows of logits and one last axis");
}

int64_t distill_rows(const Tensor& z) {
    int64_t rows = 1;
    for (int64_t i = 0; i + 1 < z.dim(); ++i) rows *= z.size(i);
    return rows;
}

std::pair<Tensor, Tensor> distill_forward(const Tensor& z, const DistillArgs& a, bool train) {
    distill_check(z, a);
    c10::DeviceGuard guard(z.device());
    const int64_t rows = distill_rows(z), classes = z.size(-1), best = a.index.size(-1);
    const Tensor m = as_rows(z);
    const auto f32 = z.options().dtype(at::kFloat);
    Tensor loss = at::empty(z.sizes().slice(0, z.dim() - 1), f32), stats;
    if (train) stats = at::empty({2 * rows}, f32);
    size_t bytes = 0;
    check(da_distill_workspace(rows, classes, &bytes));
    const Tensor ws = scratch(bytes, z);
    check(da_distill(dtype_of(z, "logits"), rows, classes, best, data<void>(m), z.dim() == 1 ? classes : pitch(m), data<void>(a.index),
                     a.index.scalar_type() == at::kLong, data<void>(a.top), dtype_of(a.top, "top_logits"), (float)a.temperature,
                     data<float>(loss), data<float>(stats), data<void>(ws), bytes, stream_of(z)));
    return {loss, stats};
}

Tensor distill_backward(const Tensor& dloss, const Tensor& z, const Tensor& stats, const DistillArgs& a) {
    distill_check(z, a);
    c10::DeviceGuard guard(z.device());
    const int64_t rows = distill_rows(z), classes = z.size(-1), best = a.index.size(-1);
    const Tensor m = as_rows(z);
    if (dloss.numel() != rows || dloss.scalar_type() != at::kFloat) throw py::value_error("the loss's gradient must be float32, one a row");
    on_device_of(z, dloss, "the loss's gradient");
    Tensor d = dloss.resolve_neg().reshape({rows});
    if (rows > 1 && d.stride(0) < 0) d = d.contiguous();
    Tensor dz = at::empty(z.sizes(), z.options());
    check(da_distill_backward(dtype_of(z, "logits"), rows, classes, best, data<void>(m), z.dim() == 1 ? classes : pitch(m),
                              data<void>(a.index), a.index.scalar_type() == at::kLong, data<void>(a.top),
                              dtype_of(a.top, "top_logits"), (float)a.temperature, data<float>(stats), data<float>(d),
                              rows > 1 ? d.stride(0) : 1, data<void>(dz), stream_of(z)));
    return dz;
}

struct DistillBackward : torch::autograd::Node {
    SavedVariable z;
    SavedVariable index, top, stats;
    double temperature = 1.0;

    void release_variables() override {
        std::lock_guard<std::mutex> lk(mutex_);
        z.reset_data();
        index.reset_data();
        top.reset_data();
        stats.reset_data();
    }
    variable_list apply(variable_list&& grads) override {
        return in_backward([&] { return gradients(grads); });
    }
    variable_list gradients(const variable_list& grads) {
        if (!grads[0].defined() || !task_should_compute_output(0)) return variable_list(1);
        Tensor Z, S;
        DistillArgs a;
        {
            std::lock_guard<std::mutex> lk(mutex_);
            Z = z.unpack();
            a = DistillArgs{index.unpack(), top.unpack(), temperature};
            S = stats.unpack();
        }
        variable_list result(1);
        {
            at::AutoDispatchBelowADInplaceOrView below;
            result[0] = distill_backward(grads[0], Z, S, a);
        }
        return once(std::move(result), "distill_loss", {grads[0], Z});
    }
    std::string name() const override { return "DistillBackward"; }
};

DistillArgs distill_args(const Tensor& index, const Tensor& top, double temperature) {
    return DistillArgs{index.detach().contiguous(), top.detach().resolve_neg().contiguous(), temperature};
}

Tensor distill(const Tensor& z, const Tensor& index, const Tensor& top, double temperature) {
    DistillArgs a;
    const bool train = at::GradMode::is_enabled() && wants_grad(z);
    std::pair<Tensor, Tensor> out;
    {
        at::AutoDispatchBelowADInplaceOrView below;
        a = distill_args(index, top, temperature);
        out = distill_forward(z, a, train);
    }
    if (train) {
        auto node = std::shared_ptr<DistillBackward>(new DistillBackward(), torch::autograd::deleteNode);
        node->temperature = temperature;
        node->stats = SavedVariable(out.second, false);
        node->z = SavedVariable(z, false);
        node->index = SavedVariable(a.index, false);
        node->top = SavedVariable(a.top, false);
        node->set_next_edges(torch::autograd::collect_next_edges(z));
        torch::autograd::set_history(out.first, node);
    }
    return out.first;
}

// ------------------------------------------------------------------------------------------
// gated feed-forward block
// ------------------------------------------------------------------------------------------
struct Weights {
    Tensor gate, up, down;       // contiguous
};

struct GatedSizes {
    int64_t rows, d, h, dout;
};

GatedSizes gated_sizes(const Tensor& x, const Weights& w) {
    on_gpu(x, "x");
    dtype_of(x, "x");
    if (x.dim() < 1) throw py::value_error("x must have a last axis");
    for (const auto& p : {std::make_pair(&w.gate, "w_gate"), std::make_pair(&w.up, "w_up"), std::make_pair(&w.down, "w_down")}) {
        on_device_of(x, *p.first, p.second);
        if (p.first->scalar_type() != x.scalar_type()) throw py::type_error(std::string(p.second) + " must have the type of x");
        if (p.first->dim() != 2) throw py::value_error(std::string(p.second) + " must be a matrix");
    }
    GatedSizes s{1, x.size(-1), w.gate.size(1), w.down.size(1)};
    for (int64_t i = 0; i + 1 < x.dim(); ++i) s.rows *= x.size(i);
    if (w.gate.size(0) != s.d || !w.up.sizes().equals(w.gate.sizes()) || w.down.size(0) != s.h)
        throw py::value_error("sizes do not match: x (..., d), w_gate and w_up (d, h), w_down (h, d_out)");
    return s;
}

Weights whole(const Weights& w) {
    return {w.gate.resolve_neg().contiguous(), w.up.resolve_neg().contiguous(), w.down.resolve_neg().contiguous()};
}

std::vector<int64_t> with_last(at::IntArrayRef sizes, int64_t last) {
    std::vector<int64_t> v(sizes.begin(), sizes.end());
    v.back() = last;
    return v;
}

struct GatedKept {
    Tensor u, v, a;
};

int64_t gated_pitch(const Tensor& t, const Tensor& m) { return t.dim() == 1 ? t.size(0) : pitch(m); }

Tensor gated_forward(const Tensor& x, const Weights& weights, int act, bool train, GatedKept* kept) {
    const GatedSizes s = gated_sizes(x, weights);
    const Weights w = whole(weights);
    c10::DeviceGuard guard(x.device());
    const Tensor m = as_rows(x);
    const int dt = dtype_of(x, "x");
    Tensor y = at::empty(with_last(x.sizes(), s.dout), x.options());
    kept->a = at::empty({s.rows, s.h}, x.options());
    if (train) {
        kept->u = at::empty({s.rows, s.h}, x.options().dtype(at::kFloat));
        kept->v = at::empty({s.rows, s.h}, x.options().dtype(at::kFloat));
    }
    size_t fwd = 0, bwd = 0;
    check(da_gated_workspace(dt, s.rows, s.d, s.h, s.dout, &fwd, &bwd));
    const Tensor ws = scratch(fwd, x);
    check(da_gated(dt, s.rows, s.d, s.h, s.dout, data<void>(m), gated_pitch(x, m), data<void>(w.gate), data<void>(w.up),
                   data<void>(w.down), act, data<void>(y), data<float>(kept->u), data<float>(kept->v), data<void>(kept->a),
                   data<void>(ws), fwd, stream_of(x)));
    return y;
}

variable_list gated_backward(const Tensor& dy, const Tensor& x, const Weights& weights, int act, const GatedKept& kept,
                             const std::array<bool, 4>& need) {
    const GatedSizes s = gated_sizes(x, weights);
    const Weights w = whole(weights);
    if (dy.dim() != x.dim() || dy.scalar_type() != x.scalar_type() || dy.size(-1) != s.dout || dy.numel() != s.rows * s.dout)
        throw py::value_error("dy must be like y");
    on_device_of(x, dy, "dy");
    c10::DeviceGuard guard(x.device());
    const Tensor m = as_rows(x), d = as_rows(dy);
    const int dt = dtype_of(x, "x");
    variable_list out(4);
    if (need[0]) out[0] = at::empty(x.sizes(), x.options());
    if (need[1]) out[1] = at::empty(w.gate.sizes(), w.gate.options());
    if (need[2]) out[2] = at::empty(w.up.sizes(), w.up.options());
    if (need[3]) out[3] = at::empty(w.down.sizes(), w.down.options());
    size_t fwd = 0, bwd = 0;
    check(da_gated_workspace(dt, s.rows, s.d, s.h, s.dout, &fwd, &bwd));
    const Tensor ws = scratch(bwd, x);
    check(da_gated_backward(dt, s.rows, s.d, s.h, s.dout, data<void>(m), gated_pitch(x, m), data<void>(d), gated_pitch(dy, d),
                            data<void>(w.gate), data<void>(w.up), data<void>(w.down), act, data<float>(kept.u),
                            data<float>(kept.v), data<void>(kept.a), data<void>(out[0]), data<void>(out[1]), data<void>(out[2]),
                            data<void>(out[3]), data<void>(ws), bwd, stream_of(x)));
    return out;
}

struct GatedBackward : torch::autograd::Node {
    SavedVariable x, gate, up, down;
    SavedVariable u, v, a;       // the largest: hooks for saved tensors see them, too
    int act = 0;

    void release_variables() override {
        std::lock_guard<std::mutex> lk(mutex_);
        x.reset_data();
        gate.reset_data();
        up.reset_data();
        down.reset_data();
        u.reset_data();
        v.reset_data();
        a.reset_data();
    }
    variable_list apply(variable_list&& grads) override {
        return in_backward([&] { return gradients(grads); });
    }
    variable_list gradients(const variable_list& grads) {
        if (!grads[0].defined()) return variable_list(4);
        Tensor X;
        Weights w;
        GatedKept k;
        {
            std::lock_guard<std::mutex> lk(mutex_);
            X = x.unpack();
            w = Weights{gate.unpack(), up.unpack(), down.unpack()};
            k = GatedKept{u.unpack(), v.unpack(), a.unpack()};
        }
        std::array<bool, 4> need;
        for (int i = 0; i < 4; ++i) need[i] = task_should_compute_output(i);
        variable_list result;
        {
            at::AutoDispatchBelowADInplaceOrView below;
            result = gated_backward(grads[0], X, w, act, k, need);
        }
        return once(std::move(result), "gated_feed_forward", {grads[0], X, w.gate, w.up, w.down});
    }
    std::string name() const override { return "GatedBackward"; }
};

Tensor gated(const Tensor& x, const Tensor& gate, const Tensor& up, const Tensor& down, int act) {
    const Weights w{gate, up, down};
    const bool train = at::GradMode::is_enabled() && (wants_grad(x) || wants_grad(gate) || wants_grad(up) || wants_grad(down));
    GatedKept kept;
    Tensor y;
    {
        at::AutoDispatchBelowADInplaceOrView below;
        y = gated_forward(x, w, act, train, &kept);
    }
    if (train) {
        auto node = std::shared_ptr<GatedBackward>(new GatedBackward(), torch::autograd::deleteNode);
        node->act = act;
        node->u = SavedVariable(kept.u, false);
        node->v = SavedVariable(kept.v, false);
        node->a = SavedVariable(kept.a, false);
        node->x = SavedVariable(x, false);
        node->gate = SavedVariable(gate, false);
        node->up = SavedVariable(up, false);
        node->down = SavedVariable(down, false);
        node->set_next_edges(torch::autograd::collect_next_edges(x, gate, up, down));
        torch::autograd::set_history(y, node);
    }
    return y;
}

}  // namespace

void bind_layers(py::module_& mod) {
    using release = py::call_guard<py::gil_scoped_release>;
    // Whether all operands are tensors and nothing else, and torch does nothing around an operation but differentiate
    // backwards: the functions below then make their own autograd nodes.
    mod.def("layers_take", [](const py::args& operands) {
        if (!ordinary_context()) return false;
        for (const auto& t : operands)
            if (!t.is_none() && !ordinary(t)) return false;
        return true;
    });
    mod.def("group_norm", &group_norm, release());
    mod.def("group_norm_forward",
            [](const Tensor& x, int64_t groups, const std::optional<Tensor>& w, const std::optional<Tensor>& b, double eps, int act,
               const std::optional<Tensor>& offsets) {
                at::AutoDispatchBelowADInplaceOrView below;
                const auto out = norm_forward(x, w.value_or(Tensor()), b.value_or(Tensor()), norm_args(groups, eps, act, offsets), true);
                return std::make_tuple(out.first, out.second.defined() ? std::optional<Tensor>(out.second) : std::nullopt);
            }, release());
    mod.def("group_norm_backward",
            [](const Tensor& dy, const Tensor& x, int64_t groups, const std::optional<Tensor>& w, const std::optional<Tensor>& b,
               double eps, int act, const std::optional<Tensor>& offsets, const std::optional<Tensor>& stats) {
                at::AutoDispatchBelowADInplaceOrView below;
                const auto g = norm_backward(dy, x, w.value_or(Tensor()), b.value_or(Tensor()), stats.value_or(Tensor()),
                                             norm_args(groups, eps, act, offsets), w.has_value(), b.has_value());
                auto some = [](const Tensor& t) { return t.defined() ? std::optional<Tensor>(t) : std::nullopt; };
                return std::make_tuple(g[0], some(g[1]), some(g[2]));
            }, release());
    mod.def("gated", &gated, release());
    mod.def("gated_forward", [](const Tensor& x, const Tensor& gate, const Tensor& up, const Tensor& down, int act) {
        at::AutoDispatchBelowADInplaceOrView below;
        GatedKept k;
        const Tensor y = gated_forward(x, Weights{gate, up, down}, act, true, &k);
        return std::make_tuple(y, k.u, k.v, k.a);
    }, release());
    mod.def("gated_backward",
            [](const Tensor& dy, const Tensor& x, const Tensor& gate, const Tensor& up, const Tensor& down, int act, const Tensor& u,
               const Tensor& v, const Tensor& a) {
                at::AutoDispatchBelowADInplaceOrView below;
                const auto g = gated_backward(dy, x, Weights{gate, up, down}, act, GatedKept{u, v, a}, {true, true, true, true});
                return std::make_tuple(g[0], g[1], g[2], g[3]);
            }, release());
    mod.def("distill", &distill, release());
    mod.def("distill_forward", [](const Tensor& z, const Tensor& index, const Tensor& top, double temperature) {
        at::AutoDispatchBelowADInplaceOrView below;
        return distill_forward(z, distill_args(index, top, temperature), true);
    }, release());
    mod.def("distill_backward",
            [](const Tensor& dloss, const Tensor& z, const Tensor& stats, const Tensor& index, const Tensor& top, double temperature) {
                at::AutoDispatchBelowADInplaceOrView below;
                return distill_backward(dloss, z, stats, distill_args(index, top, temperature));
            }, release());
}

}  // namespace da_native
