// The operators of include/ptq_heads.h on torch tensors (heads.py).
#include "ptq_torch_tensors.h"

#include "../../include/ptq_heads.h"

namespace {

decltype(&ptq_heads_workspace_bytes) f_ws = nullptr;
decltype(&ptq_heads_forward) f_forward = nullptr;
decltype(&ptq_heads_backward) f_backward = nullptr;

struct HeadsCall {
    ptq_heads_t s = {};
    at::ScalarType type;
    Shape tokens, steps, states, bc, history;         // shapes of u, delta, state, B, the history
    bool ragged;
};
// u, delta, A, B, C, D, delta_bias, state, lengths, flags; step: u [batch,heads,columns], without a length
HeadsCall read_heads(Args &a, bool step)
{
    HeadsCall c;
    const at::Tensor &u = a.tensor("u");
    const int dims = step ? 3 : 4;
    if (u.dim() != dims) refuse(step ? "u must be [batch,heads,columns]" : "u must be [batch,length,heads,columns]");
    ptq_heads_t &s = c.s;
    s.dtype = dtype_code(u, "u");
    c.type = u.scalar_type();
    c.tokens = u.sizes().vec();
    check_rows(u, "u", c.type, c.tokens);
    c.steps.assign(c.tokens.begin(), c.tokens.end() - 1);
    const int64_t batch = u.size(0), length = step ? 1 : u.size(1), heads = u.size(-2), cols = u.size(-1);
    const at::Tensor *delta = a.optional("delta");
    const at::Tensor &A = a.tensor("A"), &B = a.tensor("B"), &C = a.tensor("C");
    if (delta) {
        if (delta->scalar_type() != c.type) refuse("delta has the wrong type");
        if (delta->sizes() != at::IntArrayRef(c.steps)) refuse("delta must be " + text(c.steps));
    }
    check_dense(A, "A", at::kFloat, {heads});
    const bool grouped = B.dim() == dims;
    if (!grouped && B.dim() != dims - 1) refuse("B must have a dimension of groups or none");
    const int64_t groups = grouped ? B.size(-2) : 1, states = B.size(-1);
    c.bc.assign(c.tokens.begin(), c.tokens.end() - 2);
    if (grouped) c.bc.push_back(groups);
    c.bc.push_back(states);
    check_rows(B, "B", c.type, c.bc);
    check_rows(C, "C", c.type, c.bc);
    c.states = {batch, heads, cols, states};
    c.history = {batch, (length + PTQ_HEADS_HISTORY - 1) / PTQ_HEADS_HISTORY, heads, cols, states};
    const at::Tensor *D = a.optional("D"), *bias = a.optional("delta_bias"), *state = a.optional("state"), *lengths = a.optional("lengths");
    if (D) check_dense(*D, "D", at::kFloat, {heads});
    if (bias) check_dense(*bias, "delta_bias", at::kFloat, {heads});
    if (state) check_dense(*state, "state", at::kFloat, c.states);
    if (lengths) check_dense(*lengths, "lengths", at::kInt, {batch});
    c.ragged = lengths != nullptr;
    s.batch = small(batch, "the batch");
    s.length = small(length, "the length");
    s.heads = small(heads, "the number of heads");
    s.cols = small(cols, "the number of columns");
    s.states = small(states, "the number of states");
    s.groups = small(groups, "the number of groups");
    s.flags = static_cast<unsigned>(a.integer());
    s.u = ptr(&u);
    s.delta = ptr(delta);
    s.B = ptr(&B);
    s.C = ptr(&C);
    const auto pitches = [&](const at::Tensor &t, int64_t *pitch, bool inner) {
        pitch[0] = t.stride(0);
        pitch[1] = step ? 0 : t.stride(1);
        pitch[2] = inner ? t.stride(step ? 1 : 2) : 0;
    };
    pitches(u, s.u_pitch, true);
    if (delta) pitches(*delta, s.delta_pitch, true);
    pitches(B, s.B_pitch, grouped);
    pitches(C, s.C_pitch, grouped);
    s.A = static_cast<const float *>(ptr(&A));
    s.D = static_cast<const float *>(ptr(D));
    s.delta_bias = static_cast<const float *>(ptr(bias));
    s.state = static_cast<const float *>(ptr(state));
    s.lengths = static_cast<const int32_t *>(ptr(lengths));
    return c;
}

// heads(step, <heads>, y, final_state, history) -> y or status
PyObject *py_heads(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        Args a(args, n, 14);
        const bool step = a.integer() != 0;
        const HeadsCall c = read_heads(a, step);
        PyObject *y_arg = args[11];
        const at::Tensor *y_given = a.optional("y"), *final_state = a.optional("final_state"), *history = a.optional("history");
        if (final_state) check_dense(*final_state, step ? "new_state" : "final_state", at::kFloat, c.states);
        if (history) check_dense(*history, "history", at::kFloat, c.history);
        const c10::cuda::CUDAGuard on(a.device());
        const at::Tensor y = output(y_given, "y", c.tokens, c.type, a.device(), c.ragged);
        const size_t bytes = f_ws(&c.s, 0);
        const at::Tensor ws = space(bytes, a.device());
        void *yp = y.data_ptr(), *wp = mut<void>(ws), *stream = current_stream(a.device());
        float *fp = final_state ? static_cast<float *>(final_state->data_ptr()) : nullptr;
        float *hp = history ? static_cast<float *>(history->data_ptr()) : nullptr;
        ptq_status_t st;
        Py_BEGIN_ALLOW_THREADS
        st = f_forward(&c.s, yp, fp, hp, wp, bytes, stream);
        Py_END_ALLOW_THREADS
        if (st != PTQ_OK) return PyLong_FromLong(st);
        if (!y_given) return THPVariable_Wrap(y);
        Py_INCREF(y_arg);
        return y_arg;
    });
}

// heads_backward(<heads>, dy, history, dfinal) -> (du, ddelta, dA, dB, dC, dD, ddelta_bias, dstate) or status
PyObject *py_heads_backward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        Args a(args, n, 13);
        const HeadsCall c = read_heads(a, false);
        const at::Tensor &dy = a.tensor("dy"), &history = a.tensor("history");
        const at::Tensor *dfinal = a.optional("dfinal");
        check_dense(dy, "dy", c.type, c.tokens);
        check_dense(history, "history", at::kFloat, c.history);
        if (dfinal) check_dense(*dfinal, "dfinal", at::kFloat, c.states);
        const c10::Device dev = a.device();
        const c10::cuda::CUDAGuard on(dev);
        const size_t bytes = f_ws(&c.s, 1);
        const at::Tensor ws = space(bytes, dev);
        const Shape heads = {c.s.heads};
        at::Tensor du = empty(c.tokens, c.type, dev), dB = empty(c.bc, c.type, dev), dC = empty(c.bc, c.type, dev), dA = empty(heads, at::kFloat, dev), dd, dD,
                   db, ds;
        if (c.s.delta) dd = empty(c.steps, c.type, dev);
        if (c.s.D) dD = empty(heads, at::kFloat, dev);
        if (c.s.delta_bias) db = empty(heads, at::kFloat, dev);
        if (c.s.state) ds = empty(c.states, at::kFloat, dev);
        const ptq_heads_grads_t g = {mut<void>(du), mut<void>(dd), mut<void>(dB), mut<void>(dC), mut<float>(dA), mut<float>(dD), mut<float>(db), mut<float>(ds)};
        const float *hp = static_cast<const float *>(ptr(&history)), *fp = static_cast<const float *>(ptr(dfinal));
        const void *dyp = ptr(&dy);
        void *wp = mut<void>(ws), *stream = current_stream(dev);
        ptq_status_t st;
        Py_BEGIN_ALLOW_THREADS
        st = f_backward(&c.s, hp, dyp, fp, &g, wp, bytes, stream);
        Py_END_ALLOW_THREADS
        if (st != PTQ_OK) return PyLong_FromLong(st);
        return tuple_of({du, dd, dA, dB, dC, dD, db, ds});
    });
}

PyObject *py_bind_heads(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 3) {
        PyErr_SetString(PyExc_TypeError, "three addresses are wanted");
        return nullptr;
    }
    void *p[3];
    for (int i = 0; i < 3; ++i) p[i] = PyLong_AsVoidPtr(args[i]);
    if (PyErr_Occurred()) return nullptr;
    f_ws = reinterpret_cast<decltype(f_ws)>(p[0]);
    f_forward = reinterpret_cast<decltype(f_forward)>(p[1]);
    f_backward = reinterpret_cast<decltype(f_backward)>(p[2]);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {PTQ_METHOD("bind_heads", py_bind_heads), PTQ_METHOD("heads", py_heads), PTQ_METHOD("heads_backward", py_heads_backward),
                         {nullptr, nullptr, 0, nullptr}};

}  // namespace

int ptq_add_heads_methods(PyObject *module) { return PyModule_AddFunctions(module, methods); }
