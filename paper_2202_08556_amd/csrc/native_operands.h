// Operands and gradients of the operators of include/da_layers.h and include/da_training.h on their way to the C ABI.
#pragma once
#include "native_common.h"

#include <torch/csrc/autograd/functions/basic_ops.h>

#include "da_layers.h"

namespace da_native {

using torch::autograd::SavedVariable;
using torch::autograd::variable_list;

inline int dtype_of(const Tensor& t, const char* what) {
    if (t.scalar_type() == at::kFloat) return DA_F32;
    if (t.scalar_type() == at::kBFloat16) return DA_BF16;
    throw py::type_error(std::string(what) + " must be float32 or bfloat16");
}

inline void on_device_of(const Tensor& x, const Tensor& t, const char* what) {
    if (t.defined() && t.device() != x.device()) throw py::value_error(std::string(what) + " must be on the device of the input");
}

inline void on_gpu(const Tensor& x, const char* what) {
    if (!x.is_cuda()) throw py::value_error(std::string(what) + " must live on the GPU");
}

// The last axis as columns, all others as rows: neighbouring columns, rows at one distance
inline Tensor as_rows(const Tensor& t) {
    const int64_t n = t.size(-1);
    Tensor m = t.dim() == 2 ? t.resolve_neg() : t.resolve_neg().reshape({n ? t.numel() / n : t.numel(), n});
    if (n > 1 && m.stride(1) != 1) return m.contiguous();
    if (m.size(0) > 1 && m.stride(0) < n) return m.contiguous();
    return m;
}
inline int64_t pitch(const Tensor& m) { return m.size(0) > 1 ? m.stride(0) : m.size(1); }

inline Tensor scratch(size_t bytes, const Tensor& like) {
    return bytes ? at::empty({(int64_t)bytes}, like.options().dtype(at::kByte)) : Tensor();
}

// Gradients of gradients are not provided: asked for, they raise instead of coming out as zero.
inline variable_list once(variable_list&& grads, const char* what, const variable_list& of) {
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

}  // namespace da_native
