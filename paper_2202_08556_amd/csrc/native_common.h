// What the translation units of the Python module `_native` share.
#pragma once
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/autocast_mode.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/function.h>
#include <torch/csrc/autograd/functions/utils.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/autograd/saved_variable.h>
#include <torch/csrc/jit/frontend/tracer.h>
#include <torch/csrc/utils/pybind.h>
#include <hip/hip_runtime.h>

#include <exception>
#include <memory>
#include <optional>
#include <stdexcept>
#include <string>
#include <utility>
#include <vector>

#include "da_spmm.h"

namespace da_native {

using at::Tensor;

extern PyObject* g_error;             // binding.DaSpmmError

// A failed call of the C ABI, to be raised as binding.DaSpmmError
struct DaError : std::exception {
    int status;
    std::string text;
    explicit DaError(int st) : status(st), text(da_spmm_last_error()) {}
    const char* what() const noexcept override { return text.c_str(); }
};

inline void check(int status) {
    if (status != DA_OK) throw DaError(status);
}

inline void set_error(const DaError& e) {                // the interpreter lock is held
    const py::object err = py::reinterpret_borrow<py::object>(g_error)(e.status, e.text);
    PyErr_SetObject(g_error, err.ptr());
}

// Runs a step of a backward pass.  The autograd engine hands Python exceptions on and makes a plain RuntimeError of
// all others, so errors become Python exceptions here.
template <class F>
auto in_backward(F&& f) {
    auto raise = [](const auto& set) {
        py::gil_scoped_acquire gil;
        set();
        python_error err;
        err.persist();
        throw err;
    };
    try {
        return f();
    } catch (const DaError& e) {
        raise([&] { set_error(e); });
    } catch (const py::builtin_exception& e) {
        raise([&] { e.set_error(); });
    }
    throw std::logic_error("not reached");
}

inline void* stream_of(const Tensor& t) { return c10::hip::getCurrentHIPStream(t.device().index()).stream(); }

template <class T> T* data(const Tensor& t) { return t.defined() ? static_cast<T*>(t.data_ptr()) : nullptr; }

// Whether torch does nothing around an operation but differentiate backwards: no tracer that records, no mode
// and no function transform that intercepts
inline bool ordinary_context() {
    return !torch::jit::tracer::isTracing() && !c10::impl::TorchDispatchModeTLS::any_modes_set() &&
           !at::impl::torch_function_mode_enabled() &&
           !c10::impl::tls_is_dispatch_key_included(c10::DispatchKey::FuncTorchDynamicLayerFrontMode);
}

// Whether a tensor is its memory and nothing else: no wrapper, no lazy negation, no tangent
inline bool ordinary(const Tensor& t) {
    constexpr c10::DispatchKeySet wrapped(
        {c10::DispatchKey::Python, c10::DispatchKey::FuncTorchBatched, c10::DispatchKey::FuncTorchGradWrapper,
         c10::DispatchKey::Functionalize, c10::DispatchKey::Negative, c10::DispatchKey::Conjugate, c10::DispatchKey::ZeroTensor});
    return t.layout() == at::kStrided && !t.key_set().has_any(wrapped) && !t._fw_grad(0).defined();
}

// ... and its Python object is a Tensor or Parameter, no subclass that overrides operations
inline bool ordinary(py::handle x) { return THPVariable_CheckExact(x.ptr()) && ordinary(THPVariable_Unpack(x.ptr())); }

inline bool wants_grad(const Tensor& t) { return t.defined() && t.requires_grad(); }

void bind_layers(py::module_& mod);
void bind_training(py::module_& mod);

}  // namespace da_native
