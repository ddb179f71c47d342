// What the operators on torch tensors share: reading and checking of arguments, new tensors, streams, and exceptions on their way
// to Python.
#pragma once

#include "ptq_torch.h"

#include <ATen/cuda/EmptyTensor.h>
#include <ATen/ops/zeros.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <optional>
#include <stdexcept>
#include <string>
#include <vector>

#include "../../include/ptq_block.h"

namespace {

using Shape = std::vector<int64_t>;

// A refused argument; becomes a ValueError (TypeError where the object has the wrong class).
struct Refusal : std::runtime_error {
    PyObject *cls;
    Refusal(PyObject *c, const std::string &text) : std::runtime_error(text), cls(c) {}
};
[[noreturn]] void refuse(const std::string &text) { throw Refusal(PyExc_ValueError, text); }

template <class Fn>
PyObject *guarded(Fn fn)
{
    HANDLE_TH_ERRORS
    try {
        return fn();
    } catch (const Refusal &r) {
        PyErr_SetString(r.cls, r.what());
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

std::string text(const Shape &s)
{
    std::string t = "[";
    for (size_t i = 0; i < s.size(); ++i) t += (i ? "," : "") + std::to_string(s[i]);
    return t + "]";
}

// One call's arguments, read in their order.
class Args {
public:
    Args(PyObject *const *args, Py_ssize_t n, Py_ssize_t want) : at_(args)
    {
        if (n != want) throw Refusal(PyExc_TypeError, std::to_string(want) + " arguments are wanted");
    }
    // The next argument, null for None.
    const at::Tensor *optional(const char *name)
    {
        PyObject *o = *at_++;
        if (o == Py_None) return nullptr;
        if (!THPVariable_Check(o)) throw Refusal(PyExc_TypeError, std::string(name) + " must be a tensor");
        const at::Tensor &t = THPVariable_Unpack(o);
        if (!t.is_cuda()) refuse(std::string(name) + " must be a CUDA tensor");
        if (!device_)
            device_ = t.device();
        else if (*device_ != t.device())
            refuse(std::string(name) + " is on another device");
        return &t;
    }
    const at::Tensor &tensor(const char *name)
    {
        const at::Tensor *t = optional(name);
        if (!t) throw Refusal(PyExc_TypeError, std::string(name) + " must be a tensor");
        return *t;
    }
    PyObject *object() { return *at_++; }
    long integer()
    {
        const long v = PyLong_AsLong(*at_++);
        if (v == -1 && PyErr_Occurred()) {
            PyErr_Clear();
            throw Refusal(PyExc_TypeError, "an integer is wanted");
        }
        return v;
    }
    double number()
    {
        const double v = PyFloat_AsDouble(*at_++);
        if (v == -1.0 && PyErr_Occurred()) {
            PyErr_Clear();
            throw Refusal(PyExc_TypeError, "a number is wanted");
        }
        return v;
    }
    c10::Device device() const { return *device_; }

private:
    PyObject *const *at_;
    std::optional<c10::Device> device_;
};

int dtype_code(const at::Tensor &t, const char *name)
{
    switch (t.scalar_type()) {
        case at::kHalf: return PTQ_F16;
        case at::kBFloat16: return PTQ_BF16;
        case at::kFloat: return PTQ_F32;
        default: refuse(std::string(name) + " must be float16, bfloat16 or float32");
    }
}
int small(int64_t v, const char *what)
{
    if (v > 0x7fffffff) refuse(std::string(what) + " is too large");
    return static_cast<int>(v);
}

// Rows that lie anywhere but with the elements of a row next to each other.
void check_rows(const at::Tensor &t, const char *name, at::ScalarType type, const Shape &shape)
{
    if (t.scalar_type() != type) refuse(std::string(name) + " has the wrong type");
    if (t.sizes() != at::IntArrayRef(shape)) refuse(std::string(name) + " must be " + text(shape));
    if (t.size(-1) > 1 && t.stride(-1) != 1) refuse(std::string(name) + ": the elements of a row must be next to each other");
}
void check_dense(const at::Tensor &t, const char *name, at::ScalarType type, const Shape &shape)
{
    if (t.scalar_type() != type) refuse(std::string(name) + " has the wrong type");
    if (t.sizes() != at::IntArrayRef(shape)) refuse(std::string(name) + " must be " + text(shape));
    if (!t.is_contiguous()) refuse(std::string(name) + " must be contiguous");
}
const void *ptr(const at::Tensor *t) { return t ? t->const_data_ptr() : nullptr; }
template <typename V>
V *mut(const at::Tensor &t) { return t.defined() ? static_cast<V *>(t.data_ptr()) : nullptr; }

at::Tensor empty(const Shape &shape, at::ScalarType type, c10::Device device) { return at::Tensor(at::detail::empty_cuda(shape, type, device, std::nullopt)); }
at::Tensor space(size_t bytes, c10::Device device)
{
    return bytes ? empty({static_cast<int64_t>(bytes)}, at::kByte, device) : at::Tensor();
}
void *current_stream(c10::Device device) { return c10::cuda::getCurrentCUDAStream(device.index()).stream(); }

PyObject *wrap(const at::Tensor &t)
{
    if (!t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(t);
}
PyObject *tuple_of(std::initializer_list<at::Tensor> ts)
{
    PyObject *out = PyTuple_New(static_cast<Py_ssize_t>(ts.size()));
    if (!out) return nullptr;
    Py_ssize_t i = 0;
    for (const at::Tensor &t : ts) {
        PyObject *o = wrap(t);
        if (!o) {
            Py_DECREF(out);
            return nullptr;
        }
        PyTuple_SET_ITEM(out, i++, o);
    }
    return out;
}
// The output the caller passed, or a new one.  Rows behind the end of a sequence are left as they are: zeros in a new output.
at::Tensor output(const at::Tensor *given, const char *name, const Shape &shape, at::ScalarType type, c10::Device device, bool ragged)
{
    if (given) {
        check_dense(*given, name, type, shape);
        return *given;
    }
    return ragged ? at::zeros(shape, at::TensorOptions().dtype(type).device(device)) : empty(shape, type, device);
}
// How far apart the rows of a tensor of any shape are, where that is one distance.
int64_t row_pitch(const at::Tensor &t, const char *name)
{
    int64_t pitch = 0, want = -1;
    for (int64_t i = t.dim() - 2; i >= 0; --i) {
        if (t.size(i) == 1) continue;
        if (want < 0)
            pitch = t.stride(i);
        else if (t.stride(i) != want)
            refuse(std::string(name) + ": the rows must be one distance apart");
        want = t.stride(i) * t.size(i);
    }
    return pitch;
}

}  // namespace
