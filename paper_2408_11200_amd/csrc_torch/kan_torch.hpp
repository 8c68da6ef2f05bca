// What the autograd nodes share: errors of the C ABI as Python exceptions, pointers of tensors, the stream, workspaces.
#pragma once
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/jit/frontend/tracer.h>
#include <torch/csrc/utils/pybind.h>
#include <torch/library.h>
#include <ATen/ops/empty.h>
#include <c10/hip/HIPStream.h>
#include "kan.h"

namespace {

using at::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

[[noreturn]] void raise_kan_error(int status, const char *where)
{
    py::gil_scoped_acquire lock;
    const py::object type = py::module_::import("paper_2408_11200_amd.binding").attr("KanError");
    PyErr_SetObject(type.ptr(), type(status, where).ptr());
    throw py::error_already_set();
}

void check(int status, const char *where)
{
    if (status != KAN_OK) raise_kan_error(status, where);
}

[[noreturn]] void refuse(const char *what)
{
    py::gil_scoped_acquire lock;
    PyErr_SetString(PyExc_AssertionError, what);
    throw py::error_already_set();
}

// pointer of a device-resident contiguous fp32 tensor (null: no tensor); anything else is refused as binding.py refuses it
float *f32(const Tensor &t)
{
    if (!t.defined()) return nullptr;
    if (t.scalar_type() != at::kFloat || !t.is_cuda() || !t.is_contiguous()) refuse("device-resident contiguous float32 tensors only");
    return static_cast<float *>(t.data_ptr());
}

// What a forward pass left for its backward pass, as the graph hands it back: a hook on saved tensors may have replaced it.
void *kept(const Tensor &t)
{
    if (!t.is_cuda() || !t.is_contiguous()) refuse("device-resident contiguous tensors only");
    return t.data_ptr();
}

Tensor or_none(const std::optional<Tensor> &t) { return t ? *t : Tensor(); }

Tensor whole(const Tensor &t) { return t.defined() ? t.contiguous() : t; }

// the current device's current stream: during backward the one of the forward pass, which the engine has set
void *stream() { return (void *)c10::hip::getCurrentHIPStream().stream(); }

Tensor bytes_like(const Tensor &x, size_t n) { return at::empty({(int64_t)(n > 256 ? n : 256)}, x.options().dtype(at::kByte)); }

// A struct of plain values carried from forward to backward.
template <class T>
c10::IValue pack(const T &v) { return std::string(reinterpret_cast<const char *>(&v), sizeof(T)); }
template <class T>
T unpack(const c10::IValue &v)
{
    T t;
    std::memcpy(&t, v.toStringRef().data(), sizeof(T));
    return t;
}

// A layer as an operator of torch's dispatcher: what torch.jit.trace records.  It sees dispatched calls only, so a node applied
// directly would leave nothing in the graph but the allocation of its result.  Outside a trace the dispatcher is passed by.
template <class F, class... A>
auto call(const char *op, F f, const A &...a)
{
    py::gil_scoped_release unlock;
    if (!torch::jit::tracer::isTracing()) return f(a...);
    return c10::Dispatcher::singleton().findSchemaOrThrow(op, "").typed<std::remove_pointer_t<F>>().call(a...);
}

}  // namespace
