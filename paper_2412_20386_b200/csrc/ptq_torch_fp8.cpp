// The operators of include/ptq_fp8.h on torch tensors (fp8.py).
#include "ptq_torch_tensors.h"

#include "../../include/ptq_fp8.h"

namespace {

decltype(&ptq_fp8_quantize) f_quantize = nullptr;
decltype(&ptq_fp8_quantize_weight) f_quantize_weight = nullptr;
decltype(&ptq_fp8_matmul) f_matmul = nullptr;
decltype(&ptq_fp8_linear_workspace_bytes) f_linear_ws = nullptr;
decltype(&ptq_fp8_linear) f_linear = nullptr;

int64_t blocks_of(int64_t cols) { return (cols + PTQ_FP8_BLOCK - 1) / PTQ_FP8_BLOCK; }
Shape with_last(const at::Tensor &t, int64_t last)
{
    Shape s = t.sizes().vec();
    s.back() = last;
    return s;
}

// New codes: rows on 16-byte boundaries.
at::Tensor new_codes(const Shape &shape, c10::Device device)
{
    Shape wide = shape;
    wide.back() = (shape.back() + 15) / 16 * 16;
    const at::Tensor t = empty(wide, at::kFloat8_e4m3fn, device);
    return wide == shape ? t : t.narrow(-1, 0, shape.back());
}
// New scales [..., blocks] of `rows` rows, those of a block next to each other.
at::Tensor new_scales(const at::Tensor &x, int64_t blocks)
{
    const Shape shape = with_last(x, blocks);
    std::vector<int64_t> strides(shape.size());
    int64_t rows = 1;
    for (size_t i = shape.size() - 1; i-- > 0;) {
        strides[i] = rows;
        rows *= shape[i];
    }
    strides.back() = rows;
    return empty({rows * blocks}, at::kFloat, x.device()).as_strided(shape, strides);
}

ptq_fp8_input_t read_input(const at::Tensor &x)
{
    if (x.dim() < 1) refuse("x must be [...,channels]");
    ptq_fp8_input_t in = {};
    in.dtype = dtype_code(x, "x");
    check_rows(x, "x", x.scalar_type(), x.sizes().vec());
    in.cols = small(x.size(-1), "the number of channels");
    in.rows = in.cols ? x.numel() / in.cols : 0;
    in.x = ptr(&x);
    in.x_pitch = row_pitch(x, "x");
    return in;
}
// Codes [..., cols], each row somewhere: the distance between rows; a single row's is the least that the library takes.
int64_t codes_pitch(const at::Tensor &t, const char *name, const Shape &shape)
{
    check_rows(t, name, at::kFloat8_e4m3fn, shape);
    return shape.size() < 2 || t.numel() == t.size(-1) ? (t.size(-1) + 15) / 16 * 16 : row_pitch(t, name);
}
struct Scales {
    int64_t pitch[2];
};
Scales read_scales(const at::Tensor &t, const char *name, const Shape &shape)
{
    if (t.scalar_type() != at::kFloat) refuse(std::string(name) + " has the wrong type");
    if (t.sizes() != at::IntArrayRef(shape)) refuse(std::string(name) + " must be " + text(shape));
    return {{row_pitch(t, name), t.size(-1) > 1 ? t.stride(-1) : 0}};
}
ptq_fp8_weight_t read_weight(Args &a, int64_t cols)
{
    const at::Tensor &w = a.tensor("w"), &s = a.tensor("w_scales");
    const at::Tensor *bias = a.optional("bias");
    if (w.dim() != 2) refuse("w must be [outputs,channels]");
    ptq_fp8_weight_t d = {};
    d.codes_pitch = codes_pitch(w, "w", {w.size(0), cols});
    check_dense(s, "w_scales", at::kFloat, {blocks_of(w.size(0)), blocks_of(cols)});
    if (bias) check_dense(*bias, "bias", at::kFloat, {w.size(0)});
    d.cols = small(cols, "the number of channels");
    d.outputs = small(w.size(0), "the number of outputs");
    d.codes = ptr(&w);
    d.scales = static_cast<const float *>(ptr(&s));
    d.bias = static_cast<const float *>(ptr(bias));
    return d;
}
struct Output {
    at::Tensor t;
    int64_t pitch;
};
Output read_output(const at::Tensor *given, const Shape &shape, at::ScalarType type, c10::Device device)
{
    if (!given) return {empty(shape, type, device), shape.back()};
    check_rows(*given, "y", type, shape);
    return {*given, given->numel() == given->size(-1) ? given->size(-1) : row_pitch(*given, "y")};
}

// fp8_quantize(x, codes, scales) -> (codes, scales) or status
PyObject *py_quantize(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        Args a(args, n, 3);
        const at::Tensor &x = a.tensor("x");
        const at::Tensor *codes_given = a.optional("codes"), *scales_given = a.optional("scales");
        const ptq_fp8_input_t in = read_input(x);
        const c10::cuda::CUDAGuard on(a.device());
        const Shape shape = x.sizes().vec(), scales_shape = with_last(x, blocks_of(in.cols));
        const at::Tensor codes = codes_given ? *codes_given : new_codes(shape, a.device());
        const at::Tensor scales = scales_given ? *scales_given : new_scales(x, blocks_of(in.cols));
        const int64_t pitch = codes_pitch(codes, "codes", shape);
        const Scales s = read_scales(scales, "scales", scales_shape);
        void *cp = codes.data_ptr(), *stream = current_stream(a.device());
        float *sp = static_cast<float *>(scales.data_ptr());
        ptq_status_t st;
        Py_BEGIN_ALLOW_THREADS
        st = f_quantize(&in, cp, pitch, sp, s.pitch, stream);
        Py_END_ALLOW_THREADS
        if (st != PTQ_OK) return PyLong_FromLong(st);
        return tuple_of({codes, scales});
    });
}

// fp8_quantize_weight(w) -> (codes, scales) or status
PyObject *py_quantize_weight(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        Args a(args, n, 1);
        const at::Tensor &w = a.tensor("w");
        if (w.dim() != 2) refuse("w must be [outputs,channels]");
        const ptq_fp8_input_t in = read_input(w);
        const c10::cuda::CUDAGuard on(a.device());
        const at::Tensor codes = new_codes(w.sizes().vec(), a.device());
        const at::Tensor scales = empty({blocks_of(in.rows), blocks_of(in.cols)}, at::kFloat, a.device());
        const int64_t pitch = codes_pitch(codes, "codes", w.sizes().vec());
        void *cp = codes.data_ptr(), *stream = current_stream(a.device());
        float *sp = static_cast<float *>(scales.data_ptr());
        ptq_status_t st;
        Py_BEGIN_ALLOW_THREADS
        st = f_quantize_weight(&in, cp, pitch, sp, stream);
        Py_END_ALLOW_THREADS
        if (st != PTQ_OK) return PyLong_FromLong(st);
        return tuple_of({codes, scales});
    });
}

// fp8_matmul(a, a_scales, w, w_scales, bias, type (0, 1, 2), y) -> y or status
PyObject *py_matmul(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        Args a(args, n, 7);
        const at::Tensor &x = a.tensor("a"), &xs = a.tensor("a_scales");
        if (x.dim() < 1) refuse("a must be [...,channels]");
        const int64_t cols = x.size(-1), rows = cols ? x.numel() / cols : 0;
        const ptq_fp8_weight_t w = read_weight(a, cols);
        const long code = a.integer();
        PyObject *y_arg = args[6];
        const at::Tensor *y_given = a.optional("y");
        const int64_t pitch = codes_pitch(x, "a", x.sizes().vec());
        const Scales s = read_scales(xs, "a_scales", with_last(x, blocks_of(cols)));
        const c10::cuda::CUDAGuard on(a.device());
        const at::ScalarType type = code == PTQ_F16 ? at::kHalf : code == PTQ_BF16 ? at::kBFloat16 : at::kFloat;
        const Output y = read_output(y_given, with_last(x, w.outputs), type, a.device());
        const void *xp = ptr(&x);
        const float *sp = static_cast<const float *>(ptr(&xs));
        void *yp = y.t.data_ptr(), *stream = current_stream(a.device());
        ptq_status_t st;
        Py_BEGIN_ALLOW_THREADS
        st = f_matmul(&w, rows, xp, pitch, sp, s.pitch, yp, static_cast<int>(code), y.pitch, stream);
        Py_END_ALLOW_THREADS
        if (st != PTQ_OK) return PyLong_FromLong(st);
        if (!y_given) return THPVariable_Wrap(y.t);
        Py_INCREF(y_arg);
        return y_arg;
    });
}

// fp8_linear(x, w, w_scales, bias, y) -> y or status
PyObject *py_linear(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        Args a(args, n, 5);
        const at::Tensor &x = a.tensor("x");
        const ptq_fp8_input_t in = read_input(x);
        const ptq_fp8_weight_t w = read_weight(a, in.cols);
        PyObject *y_arg = args[4];
        const at::Tensor *y_given = a.optional("y");
        const c10::cuda::CUDAGuard on(a.device());
        const Output y = read_output(y_given, with_last(x, w.outputs), x.scalar_type(), a.device());
        const size_t bytes = f_linear_ws(in.rows, in.cols, w.outputs);
        const at::Tensor ws = space(bytes, a.device());
        void *yp = y.t.data_ptr(), *wp = mut<void>(ws), *stream = current_stream(a.device());
        ptq_status_t st;
        Py_BEGIN_ALLOW_THREADS
        st = f_linear(&w, &in, yp, y.pitch, wp, bytes, stream);
        Py_END_ALLOW_THREADS
        if (st != PTQ_OK) return PyLong_FromLong(st);
        if (!y_given) return THPVariable_Wrap(y.t);
        Py_INCREF(y_arg);
        return y_arg;
    });
}

PyObject *py_bind_fp8(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 5) {
        PyErr_SetString(PyExc_TypeError, "five addresses are wanted");
        return nullptr;
    }
    void *p[5];
    for (int i = 0; i < 5; ++i) p[i] = PyLong_AsVoidPtr(args[i]);
    if (PyErr_Occurred()) return nullptr;
    f_quantize = reinterpret_cast<decltype(f_quantize)>(p[0]);
    f_quantize_weight = reinterpret_cast<decltype(f_quantize_weight)>(p[1]);
    f_matmul = reinterpret_cast<decltype(f_matmul)>(p[2]);
    f_linear_ws = reinterpret_cast<decltype(f_linear_ws)>(p[3]);
    f_linear = reinterpret_cast<decltype(f_linear)>(p[4]);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {PTQ_METHOD("bind_fp8", py_bind_fp8),     PTQ_METHOD("fp8_quantize", py_quantize),
                         PTQ_METHOD("fp8_quantize_weight", py_quantize_weight), PTQ_METHOD("fp8_matmul", py_matmul),
                         PTQ_METHOD("fp8_linear", py_linear),     {nullptr, nullptr, 0, nullptr}};

}  // namespace

int ptq_add_fp8_methods(PyObject *module) { return PyModule_AddFunctions(module, methods); }
