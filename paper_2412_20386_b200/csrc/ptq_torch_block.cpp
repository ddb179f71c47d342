// The operators of include/ptq_block.h on torch tensors (the functions gated_scan, block_norm, short_conv and their backward
// passes of block.py): checks of types, shapes and devices, allocation of what the caller did not pass, the current stream of the
// tensors' device and the C ABI call.
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

decltype(&ptq_scan_workspace_bytes) f_scan_ws = nullptr;
decltype(&ptq_scan_forward) f_scan = nullptr;
decltype(&ptq_scan_backward) f_scan_back = nullptr;
decltype(&ptq_norm_forward) f_norm = nullptr;
decltype(&ptq_norm_workspace_bytes) f_norm_ws = nullptr;
decltype(&ptq_norm_backward) f_norm_back = nullptr;
decltype(&ptq_conv_forward) f_conv = nullptr;
decltype(&ptq_conv_workspace_bytes) f_conv_ws = nullptr;
decltype(&ptq_conv_backward) f_conv_back = nullptr;

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

// ---------------------------------------------------------------------------------------------------- scan
struct ScanCall {
    ptq_scan_t s = {};
    at::ScalarType type;
    Shape tokens, states, bc;         // [batch, length, channels] (without length for single tokens), [batch, channels, states], shape of B
    bool ragged;
    int64_t batch, length, channels, n;
};
// u, delta, A, B, C, D, z, delta_bias, state, lengths, flags
ScanCall read_scan(Args &a, bool step)
{
    ScanCall c;
    const at::Tensor &u = a.tensor("u");
    const int dims = step ? 2 : 3;
    if (u.dim() != dims) refuse(step ? "u must be [batch,channels]" : "u must be [batch,length,channels]");
    c.s.dtype = dtype_code(u, "u");
    c.type = u.scalar_type();
    c.batch = u.size(0);
    c.length = step ? 1 : u.size(1);
    c.channels = u.size(-1);
    c.tokens = u.sizes().vec();
    check_rows(u, "u", c.type, c.tokens);
    const at::Tensor &delta = a.tensor("delta"), &A = a.tensor("A"), &B = a.tensor("B"), &C = a.tensor("C");
    check_rows(delta, "delta", c.type, c.tokens);
    if (A.dim() != 2) refuse("A must be [channels,states]");
    c.n = A.size(1);
    check_dense(A, "A", at::kFloat, {c.channels, c.n});
    const bool grouped = B.dim() == dims + 1;
    const int64_t groups = grouped ? B.size(-2) : 1;
    c.bc.assign(c.tokens.begin(), c.tokens.end() - 1);
    if (grouped) c.bc.push_back(groups);
    c.bc.push_back(c.n);
    check_rows(B, "B", c.type, c.bc);
    check_rows(C, "C", c.type, c.bc);
    const Shape per_channel = {c.channels};
    c.states = {c.batch, c.channels, c.n};
    const at::Tensor *D = a.optional("D"), *z = a.optional("z"), *bias = a.optional("delta_bias"), *state = a.optional("state"),
                     *lengths = a.optional("lengths");
    if (D) check_dense(*D, "D", at::kFloat, per_channel);
    if (z) check_rows(*z, "z", c.type, c.tokens);
    if (bias) check_dense(*bias, "delta_bias", at::kFloat, per_channel);
    if (state) check_dense(*state, "state", at::kFloat, c.states);
    if (lengths) check_dense(*lengths, "lengths", at::kInt, {c.batch});
    c.ragged = lengths != nullptr;
    ptq_scan_t &s = c.s;
    s.batch = small(c.batch, "the batch");
    s.length = small(c.length, "the length");
    s.channels = small(c.channels, "the number of channels");
    s.states = small(c.n, "the number of states");
    s.groups = small(groups, "the number of groups");
    s.flags = static_cast<unsigned>(a.integer());
    s.u = ptr(&u);
    s.delta = ptr(&delta);
    s.z = ptr(z);
    s.B = ptr(&B);
    s.C = ptr(&C);
    const auto rows = [&](const at::Tensor &t, int64_t *pitch) {
        pitch[0] = t.stride(0);
        pitch[1] = step ? 0 : t.stride(1);
    };
    rows(u, s.u_pitch);
    rows(delta, s.delta_pitch);
    if (z) rows(*z, s.z_pitch);
    rows(B, s.B_pitch);
    rows(C, s.C_pitch);
    s.B_pitch[2] = grouped ? B.stride(-2) : 0;
    s.C_pitch[2] = grouped ? C.stride(-2) : 0;
    s.A = static_cast<const float *>(ptr(&A));
    s.D = static_cast<const float *>(ptr(D));
    s.delta_bias = static_cast<const float *>(ptr(bias));
    s.state = static_cast<const float *>(ptr(state));
    s.lengths = static_cast<const int32_t *>(ptr(lengths));
    return c;
}

// scan(step, <scan>, y, final_state, history) -> y or status
PyObject *py_scan(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        Args a(args, n, 15);
        const bool step = a.integer() != 0;
        const ScanCall c = read_scan(a, step);
        PyObject *y_arg = args[12];
        const at::Tensor *y_given = a.optional("y"), *final_state = a.optional("final_state"), *history = a.optional("history");
        if (final_state) check_dense(*final_state, step ? "new_state" : "final_state", at::kFloat, c.states);
        if (history)
            check_dense(*history, "history", at::kFloat, {c.batch, (c.length + PTQ_SCAN_HISTORY - 1) / PTQ_SCAN_HISTORY, c.channels, c.n});
        const c10::cuda::CUDAGuard on(a.device());
        const at::Tensor y = output(y_given, "y", c.tokens, c.type, a.device(), c.ragged);
        const size_t bytes = f_scan_ws(&c.s, 0);
        const at::Tensor ws = space(bytes, a.device());
        void *yp = y.data_ptr(), *wp = mut<void>(ws), *stream = current_stream(a.device());
        float *fp = final_state ? static_cast<float *>(final_state->data_ptr()) : nullptr;
        float *hp = history ? static_cast<float *>(history->data_ptr()) : nullptr;
        ptq_status_t st;
        Py_BEGIN_ALLOW_THREADS
        st = f_scan(&c.s, yp, fp, hp, wp, bytes, stream);
        Py_END_ALLOW_THREADS
        if (st != PTQ_OK) return PyLong_FromLong(st);
        if (!y_given) return THPVariable_Wrap(y);
        Py_INCREF(y_arg);
        return y_arg;
    });
}

// scan_backward(<scan>, dy, history, dfinal) -> (du, ddelta, dA, dB, dC, dD, dz, ddelta_bias, dstate) or status
PyObject *py_scan_backward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        Args a(args, n, 14);
        const ScanCall c = read_scan(a, false);
        const at::Tensor &dy = a.tensor("dy"), &history = a.tensor("history");
        const at::Tensor *dfinal = a.optional("dfinal");
        check_dense(dy, "dy", c.type, c.tokens);
        check_dense(history, "history", at::kFloat, {c.batch, (c.length + PTQ_SCAN_HISTORY - 1) / PTQ_SCAN_HISTORY, c.channels, c.n});
        if (dfinal) check_dense(*dfinal, "dfinal", at::kFloat, c.states);
        const c10::Device dev = a.device();
        const c10::cuda::CUDAGuard on(dev);
        const size_t bytes = f_scan_ws(&c.s, 1);
        const at::Tensor ws = space(bytes, dev);
        at::Tensor du = empty(c.tokens, c.type, dev), dd = empty(c.tokens, c.type, dev), dB = empty(c.bc, c.type, dev), dC = empty(c.bc, c.type, dev),
                   dA = empty({c.channels, c.n}, at::kFloat, dev), dz, dD, db, ds;
        if (c.s.z) dz = empty(c.tokens, c.type, dev);
        if (c.s.D) dD = empty({c.channels}, at::kFloat, dev);
        if (c.s.delta_bias) db = empty({c.channels}, at::kFloat, dev);
        if (c.s.state) ds = empty(c.states, at::kFloat, dev);
        const ptq_scan_grads_t g = {mut<void>(du), mut<void>(dd), mut<void>(dz), mut<void>(dB), mut<void>(dC), mut<float>(dA),
                                    mut<float>(dD), mut<float>(db), mut<float>(ds)};
        const float *hp = static_cast<const float *>(ptr(&history)), *fp = static_cast<const float *>(ptr(dfinal));
        const void *dyp = ptr(&dy);
        void *wp = mut<void>(ws), *stream = current_stream(dev);
        ptq_status_t st;
        Py_BEGIN_ALLOW_THREADS
        st = f_scan_back(&c.s, hp, dyp, fp, &g, wp, bytes, stream);
        Py_END_ALLOW_THREADS
        if (st != PTQ_OK) return PyLong_FromLong(st);
        return tuple_of({du, dd, dA, dB, dC, dD, dz, db, ds});
    });
}

// ---------------------------------------------------------------------------------------------------- norm
struct NormCall {
    ptq_norm_t n = {};
    at::ScalarType type, residual_type;
    Shape shape;
};
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
// x, weight, bias, residual, scale, gate, flags, eps
NormCall read_norm(Args &a)
{
    NormCall c;
    const at::Tensor &x = a.tensor("x");
    if (x.dim() < 1) refuse("x must be [...,channels]");
    c.n.dtype = dtype_code(x, "x");
    c.type = x.scalar_type();
    c.shape = x.sizes().vec();
    check_rows(x, "x", c.type, c.shape);
    const int64_t cols = x.size(-1);
    const at::Tensor *w = a.optional("weight"), *b = a.optional("bias"), *r = a.optional("residual"), *s = a.optional("scale"), *g = a.optional("gate");
    for (auto [t, name] : {std::pair{w, "weight"}, {b, "bias"}, {s, "scale"}})
        if (t) check_dense(*t, name, at::kFloat, {cols});
    if (g) check_rows(*g, "gate", c.type, c.shape);
    c.residual_type = r ? r->scalar_type() : c.type;
    c.n.residual_dtype = c.n.dtype;
    if (r) {
        c.n.residual_dtype = dtype_code(*r, "residual");
        check_rows(*r, "residual", c.residual_type, c.shape);
    }
    c.n.rows = cols ? x.numel() / cols : 0;
    c.n.cols = small(cols, "the number of channels");
    c.n.flags = static_cast<unsigned>(a.integer());
    c.n.eps = static_cast<float>(a.number());
    c.n.x = ptr(&x);
    c.n.residual = ptr(r);
    c.n.gate = ptr(g);
    c.n.x_pitch = row_pitch(x, "x");
    if (r) c.n.residual_pitch = row_pitch(*r, "residual");
    if (g) c.n.gate_pitch = row_pitch(*g, "gate");
    c.n.weight = static_cast<const float *>(ptr(w));
    c.n.bias = static_cast<const float *>(ptr(b));
    c.n.scale = static_cast<const float *>(ptr(s));
    return c;
}

// Without a residual the stream that begins here has the type of r, or of its gradient, as the caller holds it: x's or binary32.
void begin_stream(NormCall &c, const at::Tensor *r)
{
    if (c.n.residual || !r || r->scalar_type() != at::kFloat) return;
    c.residual_type = at::kFloat;
    c.n.residual_dtype = PTQ_F32;
}

// norm(<norm>, y, residual_out) -> (y, residual_out or None) or status
PyObject *py_norm(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        Args a(args, n, 10);
        NormCall c = read_norm(a);
        const at::Tensor *y_given = a.optional("y"), *r_given = a.optional("residual_out");
        begin_stream(c, r_given);
        const c10::cuda::CUDAGuard on(a.device());
        const at::Tensor y = output(y_given, "y", c.shape, c.type, a.device(), false);
        at::Tensor r;
        if (c.n.residual || r_given) r = output(r_given, "residual_out", c.shape, c.residual_type, a.device(), false);
        void *yp = y.data_ptr(), *rp = mut<void>(r), *stream = current_stream(a.device());
        ptq_status_t st;
        Py_BEGIN_ALLOW_THREADS
        st = f_norm(&c.n, yp, rp, stream);
        Py_END_ALLOW_THREADS
        if (st != PTQ_OK) return PyLong_FromLong(st);
        return tuple_of({y, r});
    });
}

// norm_backward(<norm>, dy, dresidual_out) -> (dx, dweight, dbias, dresidual, dscale, dgate) or status
PyObject *py_norm_backward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        Args a(args, n, 10);
        NormCall c = read_norm(a);
        const at::Tensor &dy = a.tensor("dy");
        const at::Tensor *dr_out = a.optional("dresidual_out");
        begin_stream(c, dr_out);
        check_dense(dy, "dy", c.type, c.shape);
        if (dr_out) check_dense(*dr_out, "dresidual_out", c.residual_type, c.shape);
        const c10::Device dev = a.device();
        const c10::cuda::CUDAGuard on(dev);
        const size_t bytes = f_norm_ws(&c.n);
        const at::Tensor ws = space(bytes, dev);
        const Shape cols = {c.n.cols};
        at::Tensor dx = empty(c.shape, c.type, dev), dw, db, dr, ds, dg;
        if (c.n.weight) dw = empty(cols, at::kFloat, dev);
        if (c.n.bias) db = empty(cols, at::kFloat, dev);
        if (c.n.scale) ds = empty(cols, at::kFloat, dev);
        if (c.n.residual) dr = empty(c.shape, c.residual_type, dev);
        if (c.n.gate) dg = empty(c.shape, c.type, dev);
        const ptq_norm_grads_t g = {mut<void>(dx), mut<void>(dg), mut<void>(dr), mut<float>(dw), mut<float>(db), mut<float>(ds)};
        const void *dyp = ptr(&dy), *drp = ptr(dr_out);
        void *wp = mut<void>(ws), *stream = current_stream(dev);
        ptq_status_t st;
        Py_BEGIN_ALLOW_THREADS
        st = f_norm_back(&c.n, dyp, drp, &g, wp, bytes, stream);
        Py_END_ALLOW_THREADS
        if (st != PTQ_OK) return PyLong_FromLong(st);
        return tuple_of({dx, dw, db, dr, ds, dg});
    });
}

// ---------------------------------------------------------------------------------------------------- conv
struct ConvCall {
    ptq_conv_t c = {};
    at::ScalarType type;
    Shape tokens, states, weight;
    bool ragged;
};
// x, weight, bias, state, lengths, flags
ConvCall read_conv(Args &a)
{
    ConvCall c;
    const at::Tensor &x = a.tensor("x"), &w = a.tensor("weight");
    if (x.dim() != 3) refuse("x must be [batch,length,channels]");
    c.c.dtype = dtype_code(x, "x");
    c.type = x.scalar_type();
    c.tokens = x.sizes().vec();
    check_rows(x, "x", c.type, c.tokens);
    const int64_t channels = x.size(2);
    if (w.dim() != 2) refuse("weight must be [channels,taps]");
    c.weight = {channels, w.size(1)};
    check_dense(w, "weight", at::kFloat, c.weight);
    c.states = {x.size(0), w.size(1) - 1, channels};
    const at::Tensor *b = a.optional("bias"), *state = a.optional("state"), *lengths = a.optional("lengths");
    if (b) check_dense(*b, "bias", at::kFloat, {channels});
    if (state) check_dense(*state, "state", c.type, c.states);
    if (lengths) check_dense(*lengths, "lengths", at::kInt, {x.size(0)});
    c.ragged = lengths != nullptr;
    c.c.batch = small(x.size(0), "the batch");
    c.c.length = small(x.size(1), "the length");
    c.c.channels = small(channels, "the number of channels");
    c.c.taps = small(w.size(1), "the number of taps");
    c.c.flags = static_cast<unsigned>(a.integer());
    c.c.x = ptr(&x);
    c.c.x_pitch[0] = x.stride(0);
    c.c.x_pitch[1] = x.stride(1);
    c.c.weight = static_cast<const float *>(ptr(&w));
    c.c.bias = static_cast<const float *>(ptr(b));
    c.c.state = ptr(state);
    c.c.lengths = static_cast<const int32_t *>(ptr(lengths));
    return c;
}

// conv(<conv>, y, final_state) -> y or status
PyObject *py_conv(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        Args a(args, n, 8);
        const ConvCall c = read_conv(a);
        PyObject *y_arg = args[6];
        const at::Tensor *y_given = a.optional("y"), *final_state = a.optional("final_state");
        if (final_state) check_dense(*final_state, "final_state", c.type, c.states);
        const c10::cuda::CUDAGuard on(a.device());
        const at::Tensor y = output(y_given, "y", c.tokens, c.type, a.device(), c.ragged);
        void *yp = y.data_ptr(), *fp = final_state ? final_state->data_ptr() : nullptr, *stream = current_stream(a.device());
        ptq_status_t st;
        Py_BEGIN_ALLOW_THREADS
        st = f_conv(&c.c, yp, fp, stream);
        Py_END_ALLOW_THREADS
        if (st != PTQ_OK) return PyLong_FromLong(st);
        if (!y_given) return THPVariable_Wrap(y);
        Py_INCREF(y_arg);
        return y_arg;
    });
}

// conv_backward(<conv>, dy, dfinal) -> (dx, dweight, dbias, dstate) or status
PyObject *py_conv_backward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        Args a(args, n, 8);
        const ConvCall c = read_conv(a);
        const at::Tensor &dy = a.tensor("dy");
        const at::Tensor *dfinal = a.optional("dfinal");
        check_dense(dy, "dy", c.type, c.tokens);
        if (dfinal) check_dense(*dfinal, "dfinal", c.type, c.states);
        const c10::Device dev = a.device();
        const c10::cuda::CUDAGuard on(dev);
        const size_t bytes = f_conv_ws(&c.c);
        const at::Tensor ws = space(bytes, dev);
        at::Tensor dx = empty(c.tokens, c.type, dev), dw = empty(c.weight, at::kFloat, dev), db, ds;
        if (c.c.bias) db = empty({c.c.channels}, at::kFloat, dev);
        if (c.c.state) ds = empty(c.states, c.type, dev);
        const ptq_conv_grads_t g = {mut<void>(dx), mut<void>(ds), mut<float>(dw), mut<float>(db)};
        const void *dyp = ptr(&dy), *fp = ptr(dfinal);
        void *wp = mut<void>(ws), *stream = current_stream(dev);
        ptq_status_t st;
        Py_BEGIN_ALLOW_THREADS
        st = f_conv_back(&c.c, dyp, fp, &g, wp, bytes, stream);
        Py_END_ALLOW_THREADS
        if (st != PTQ_OK) return PyLong_FromLong(st);
        return tuple_of({dx, dw, db, ds});
    });
}

PyObject *py_bind_block(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 9) {
        PyErr_SetString(PyExc_TypeError, "nine addresses are wanted");
        return nullptr;
    }
    void *p[9];
    for (int i = 0; i < 9; ++i) p[i] = PyLong_AsVoidPtr(args[i]);
    if (PyErr_Occurred()) return nullptr;
    f_scan_ws = reinterpret_cast<decltype(f_scan_ws)>(p[0]);
    f_scan = reinterpret_cast<decltype(f_scan)>(p[1]);
    f_scan_back = reinterpret_cast<decltype(f_scan_back)>(p[2]);
    f_norm = reinterpret_cast<decltype(f_norm)>(p[3]);
    f_norm_ws = reinterpret_cast<decltype(f_norm_ws)>(p[4]);
    f_norm_back = reinterpret_cast<decltype(f_norm_back)>(p[5]);
    f_conv = reinterpret_cast<decltype(f_conv)>(p[6]);
    f_conv_ws = reinterpret_cast<decltype(f_conv_ws)>(p[7]);
    f_conv_back = reinterpret_cast<decltype(f_conv_back)>(p[8]);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {PTQ_METHOD("bind_block", py_bind_block),  PTQ_METHOD("scan", py_scan),   PTQ_METHOD("scan_backward", py_scan_backward),
                         PTQ_METHOD("norm", py_norm),              PTQ_METHOD("norm_backward", py_norm_backward),
                         PTQ_METHOD("conv", py_conv),              PTQ_METHOD("conv_backward", py_conv_backward),
                         {nullptr, nullptr, 0, nullptr}};

}  // namespace

int ptq_add_block_methods(PyObject *module) { return PyModule_AddFunctions(module, methods); }
