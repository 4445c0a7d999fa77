// Argument marshalling between Python and the C ABI (include/hq.h): checks of the tensors, allocation of the
// results, PyTorch's current stream.  No arithmetic and no device code.
//
// Why native: interpreted, a call spent about 11 us on attribute look-ups, checks and the foreign-function layer
// before its kernel was launched - more than most of the kernels take; here it is about 4 us, most of it the launch.
// (Two calls back to back on small layers: 23 .. 24 us a layer before, 9.8 .. 10.4 us with this; linear
// 8192 x 384 -> 1152: 23.4 -> 15.1 us, bound by its kernels.)
//
// The entry points of the library are handed over as addresses (bind), so that the library is loaded in one place.
#include <Python.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ATen.h>
#include <ATen/EmptyTensor.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/core/GradMode.h>
#include <c10/hip/HIPStream.h>

#include <initializer_list>
#include <string>

#include "hq.h"
#include "hq_overlap.h"

// (build.py looks for this text in the file)
extern "C" __attribute__((used, visibility("default"))) const char hq_marshal_built_for[] = HQ_BUILT_FOR;

namespace {

// ---- the library ------------------------------------------------------------------------------------------
#define HQ_ENTRY_POINTS(X)                                                                                          \
    X(hq_status_string) X(hq_quantize_weights) X(hq_act_hadamard_quant) X(hq_int_linear) X(hq_int_conv2d)            \
    X(hq_act_hadamard_quant_static) X(hq_int_linear_static) X(hq_int_conv2d_static) X(hq_quantize_weights_single)    \
    X(hq_int_linear_single) X(hq_act_hadamard_quant_width) X(hq_int_conv2d_width) X(hq_int_linear_i8)                \
    X(hq_int_conv2d_i8) X(hq_act_hadamard_quant_i8) X(hq_act_quant_int_conv2d) X(hq_act_quant_int_linear) \
    X(hq_fp8_quantize_rows) X(hq_fp8_quantize_blocks) X(hq_fp8_linear) X(hq_act_quant_fp8_linear)                    \
    X(hq_act_quant_fp8_linear_workspace) X(hq_fp8_linear_backward) X(hq_fp8_linear_backward_workspace)               \
    X(hq_qk_norm_rope) X(hq_qk_norm_rope_backward) X(hq_qk_norm_rope_backward_workspace)

struct Library {
#define X(name) decltype(&::name) name;
    HQ_ENTRY_POINTS(X)
#undef X
} lib;
PyObject *error_class = nullptr;   // HqError(fn, code, text)

// ---- errors -----------------------------------------------------------------------------------------------
struct PythonError {};   // the interpreter's error indicator is set

[[noreturn]] void refuse(const std::string &text) {
    PyErr_SetString(PyExc_ValueError, text.c_str());
    throw PythonError();
}

void check(const char *fn, hq_status st) {
    if (st == HQ_OK) return;
    PyObject *e = PyObject_CallFunction(error_class, "sis", fn, static_cast<int>(st), lib.hq_status_string(st));
    if (e) {
        PyErr_SetObject(error_class, e);
        Py_DECREF(e);
    }
    throw PythonError();
}

// The library only enqueues work; other threads may run meanwhile.  Its arguments are values: all that can fail (sizes that do
// not fit, storage without memory, the stream) is evaluated by the caller, with the interpreter's lock held.
struct Unlocked {
    PyThreadState *const state = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(state); }
};
template <class... Parameters, class... Values>
hq_status call(hq_status (*f)(Parameters...), Values... values) {
    const Unlocked unlocked;
    return f(values...);
}

// ---- arguments --------------------------------------------------------------------------------------------
struct Args {
    PyObject *const *v;
    Py_ssize_t n, at = 0;
    PyObject *next() {
        if (at >= n) {
            PyErr_SetString(PyExc_TypeError, "too few arguments");
            throw PythonError();
        }
        return v[at++];
    }
    int integer() {
        const long x = PyLong_AsLong(next());
        if (x == -1 && PyErr_Occurred()) throw PythonError();
        if (x > 0x7FFFFFFFL || x < -0x7FFFFFFFL) refuse("an integer argument does not fit 32 bits");
        return static_cast<int>(x);
    }
    at::ScalarType dtype() {
        PyObject *o = next();
        if (!THPDtype_Check(o)) {
            PyErr_SetObject(PyExc_KeyError, o);
            throw PythonError();
        }
        return reinterpret_cast<THPDtype *>(o)->scalar_type;
    }
    bool none() const { return at < n && v[at] == Py_None; }
    // a tensor; must be one
    const at::Tensor &tensor(const char *name) {
        PyObject *o = next();
        if (!THPVariable_Check(o)) {
            PyErr_Format(PyExc_TypeError, "%s must be a tensor", name);
            throw PythonError();
        }
        return THPVariable_Unpack(o);
    }
    // contiguous, on the device
    const at::Tensor &device(const char *name) {
        const at::Tensor &t = tensor(name);
        if (!t.is_cuda() || !t.is_contiguous()) refuse(std::string(name) + " must be a contiguous device tensor");
        return t;
    }
    const at::Tensor &codes(at::ScalarType dt, const char *name) {
        const at::Tensor &t = device(name);
        if (t.scalar_type() != dt)
            refuse(std::string(name) + " must hold " + (dt == at::kByte ? "torch.uint8" : "torch.int8") + " codes");
        return t;
    }
    // an optional vector: exactly n elements of dt; the pointer, or null for None
    const void *vec(int64_t count, at::ScalarType dt, const char *name) {
        if (none()) {
            next();
            return nullptr;
        }
        const at::Tensor &t = tensor(name);
        if (!t.is_cuda() || !t.is_contiguous() || t.scalar_type() != dt || t.numel() != count)
            refuse(std::string(name) + " must be a contiguous device tensor of " + c10::toString(dt) + " with " +
                   std::to_string(count) + " elements");
        return t.const_data_ptr();
    }
    // one float32 on the device
    const float *scalar() {
        if (none()) refuse("x_scale must be a device tensor holding one float32");
        const at::Tensor &t = tensor("x_scale");
        if (!t.is_cuda() || t.scalar_type() != at::kFloat || t.numel() != 1)
            refuse("x_scale must be a device tensor holding one float32");
        return static_cast<const float *>(t.const_data_ptr());
    }
};

const float *f32(const void *p) { return static_cast<const float *>(p); }
const uint8_t *u8(const at::Tensor &t) { return static_cast<const uint8_t *>(t.const_data_ptr()); }

hq_dtype hq_type(at::ScalarType dt) {
    switch (dt) {
        case at::kHalf: return HQ_F16;
        case at::kFloat: return HQ_F32;
        case at::kInt: return HQ_I32;
        default:
            PyErr_SetString(PyExc_KeyError, c10::toString(dt));
            throw PythonError();
    }
}

void *stream() { return c10::hip::getCurrentHIPStream().stream(); }

at::Tensor empty(at::IntArrayRef shape, at::ScalarType dt, const at::Tensor &like) {
    return at::detail::empty_cuda(shape, dt, like.device(), std::nullopt);
}

// A caller's result buffer (the argument `o`; must hold exactly the result) or a new one.
at::Tensor result(PyObject *o, at::IntArrayRef shape, at::ScalarType dt, const at::Tensor &like) {
    if (o == Py_None) return empty(shape, dt, like);
    if (!THPVariable_Check(o)) {
        PyErr_SetString(PyExc_TypeError, "out must be a tensor");
        throw PythonError();
    }
    const at::Tensor &t = THPVariable_Unpack(o);
    int64_t count = 1;
    for (const int64_t d : shape) count *= d;
    if (!t.is_cuda() || t.scalar_type() != dt || t.numel() != count || !t.is_contiguous())
        refuse(std::string("out must be a contiguous device tensor of ") + c10::toString(dt) + " with " +
               std::to_string(count) + " elements");
    return t;
}

// out = None or a pair of buffers (any sequence of them)
struct Pair {
    PyObject *a = Py_None, *b = Py_None;
    explicit Pair(PyObject *o) {
        if (o == Py_None) return;
        owned = true;
        a = PySequence_GetItem(o, 0);
        b = a ? PySequence_GetItem(o, 1) : nullptr;
        if (!b) {
            Py_XDECREF(a);
            throw PythonError();
        }
    }
    ~Pair() {
        if (!owned) return;
        Py_DECREF(a);
        Py_DECREF(b);
    }
    Pair(const Pair &) = delete;

private:
    bool owned = false;
};

using Shape = c10::SmallVector<int64_t, 6>;

Shape with_last(const at::Tensor &t, int64_t last) {
    Shape s(t.sizes().begin(), t.sizes().end());
    s.back() = last;
    return s;
}
Shape without_last(const at::Tensor &t) { return Shape(t.sizes().begin(), t.sizes().end() - 1); }

PyObject *wrap(const at::Tensor &t) { return THPVariable_Wrap(t); }
PyObject *wrap(const at::Tensor &a, const at::Tensor &b) {
    PyObject *pa = THPVariable_Wrap(a), *pb = THPVariable_Wrap(b);
    PyObject *p = pa && pb ? PyTuple_Pack(2, pa, pb) : nullptr;
    Py_XDECREF(pa);
    Py_XDECREF(pb);
    return p;
}

PyObject *wrap(std::initializer_list<at::Tensor> ts) {   // None for one that is not defined
    PyObject *p = PyTuple_New(static_cast<Py_ssize_t>(ts.size()));
    Py_ssize_t i = 0;
    for (const at::Tensor &t : ts) {
        PyObject *o = p ? t.defined() ? THPVariable_Wrap(t) : Py_NewRef(Py_None) : nullptr;
        if (!o) {
            Py_XDECREF(p);
            return nullptr;
        }
        PyTuple_SET_ITEM(p, i++, o);
    }
    return p;
}

// The library takes sizes of 32 bits (but for the rows of a matrix).
void expect_32bit(std::initializer_list<int64_t> sizes) {
    for (const int64_t v : sizes)
        if (v > 0x7FFFFFFFLL) refuse("a size does not fit 32 bits");
}
int narrow(int64_t v) { return static_cast<int>(v); }

void expect_dims(const at::Tensor &t, int64_t dims, const char *text) {
    if (t.dim() != dims) refuse(text);
}

struct ConvOut {
    int64_t h, w;
};
ConvOut conv_out(int64_t h, int64_t w, int ksize, int stride, int pad) {
    if (stride < 1 || pad < 0 || ksize < 1) refuse("bad convolution geometry");
    // (rounded down, as for positive sizes; a window larger than the padded image is refused by the library)
    auto out = [&](int64_t n) {
        const int64_t d = n + int64_t{2} * pad - ksize;
        return (d >= 0 ? d / stride : -((-d + stride - 1) / stride)) + 1;
    };
    return {out(h), out(w)};
}
void expect_result(const ConvOut &o) {
    if (o.h < 0 || o.w < 0) refuse("bad convolution geometry");
}
int padding(Args &a, int ksize) {
    if (a.none()) {
        a.next();
        return (ksize - 1) / 2;
    }
    return a.integer();
}

// ---- calls: arguments in the order of the functions of binding.py -----------------------------------------------
PyObject *quantize_weights(Args a) {
    const at::Tensor &w = a.device("w");
    const int block = a.integer(), bits = a.integer();
    expect_dims(w, 3, "w must be [n_out, taps, k_in]");
    const int64_t n = w.size(0), taps = w.size(1), k = w.size(2);
    expect_32bit({n, taps, k});
    const at::Tensor wq = empty({n, taps, bits == 8 ? k : k / 2}, bits == 8 ? at::kChar : at::kByte, w);
    const at::Tensor ws = empty({n}, at::kFloat, w);
    const hq_dtype dt = hq_type(w.scalar_type());
    check("hq_quantize_weights", call(lib.hq_quantize_weights, w.const_data_ptr(), dt, narrow(n), narrow(taps),
                                      narrow(k), block, bits, static_cast<uint8_t *>(wq.data_ptr()),
                                      static_cast<float *>(ws.data_ptr()), stream()));
    return wrap(wq, ws);
}

PyObject *act_hadamard_quant(Args a) {
    const at::Tensor &x = a.device("x");
    const int block = a.integer(), bits = a.integer();
    const Pair out(a.next());
    if (x.dim() < 1) refuse("x must have a channel axis");
    const int64_t k = x.size(-1), m = k ? x.numel() / k : 0;
    expect_32bit({k});
    const at::Tensor xq = result(out.a, with_last(x, bits == 8 ? k : k / 2), bits == 8 ? at::kChar : at::kByte, x);
    const at::Tensor xs = result(out.b, without_last(x), at::kFloat, x);
    const hq_dtype dt = hq_type(x.scalar_type());
    check("hq_act_hadamard_quant", call(lib.hq_act_hadamard_quant, x.const_data_ptr(), dt, m, narrow(k), block, bits,
                                        static_cast<uint8_t *>(xq.data_ptr()), static_cast<float *>(xs.data_ptr()),
                                        stream()));
    return wrap(xq, xs);
}

PyObject *act_hadamard_quant_i8(Args a) {
    const at::Tensor &x = a.device("x");
    const int block = a.integer(), bits = a.integer();
    if (x.dim() < 1) refuse("x must have a channel axis");
    const int64_t k = x.size(-1), m = k ? x.numel() / k : 0;
    expect_32bit({k});
    const at::Tensor xq = empty(x.sizes(), at::kChar, x);
    const at::Tensor xs = empty(without_last(x), at::kFloat, x);
    const hq_dtype dt = hq_type(x.scalar_type());
    check("hq_act_hadamard_quant_i8", call(lib.hq_act_hadamard_quant_i8, x.const_data_ptr(), dt, m, narrow(k), block,
                                           bits, static_cast<int8_t *>(xq.data_ptr()),
                                           static_cast<float *>(xs.data_ptr()), stream()));
    return wrap(xq, xs);
}

PyObject *act_hadamard_quant_static(Args a) {
    const at::Tensor &x = a.device("x");
    PyObject *scale = a.next();
    const int block = a.integer(), bits = a.integer();
    if (x.dim() < 1) refuse("x must have a channel axis");
    const int64_t k = x.size(-1), m = k ? x.numel() / k : 0;
    expect_32bit({k});
    const at::Tensor xq = result(a.next(), with_last(x, k / 2), at::kByte, x);
    Args one{&scale, 1};
    const float *s = one.scalar();
    const hq_dtype dt = hq_type(x.scalar_type());
    check("hq_act_hadamard_quant_static", call(lib.hq_act_hadamard_quant_static, x.const_data_ptr(), dt, m, narrow(k),
                                               block, bits, s, static_cast<uint8_t *>(xq.data_ptr()), stream()));
    return wrap(xq);
}

// hq_int_linear, hq_int_linear_static, hq_int_linear_i8
enum class Scales { dynamic, fixed };

template <class Code>
PyObject *int_linear(Args &a, const char *fn, hq_status (*f)(const Code *, const float *, const Code *, const float *, const void *,
                                                              int64_t, int, int, void *, hq_dtype, void *), Scales scales) {
    constexpr bool bytes = std::is_same<Code, int8_t>::value;   // one code per byte
    constexpr at::ScalarType code = bytes ? at::kChar : at::kByte;
    const at::Tensor &xq = a.codes(code, "xq");
    PyObject *x_scale = a.next();
    const at::Tensor &wq = a.codes(code, "wq");
    PyObject *w_scale = a.next(), *bias = a.next();
    const at::ScalarType ydt = a.dtype();
    expect_dims(xq, 2, "xq must be [m, k]");
    const int64_t m = xq.size(0), kb = xq.size(1), n = wq.dim() ? wq.size(0) : 0;
    expect_32bit({n, bytes ? kb : kb * 2});
    if (wq.numel() != n * kb) refuse("wq does not match xq in k");
    const void *sx = Args{&x_scale, 1}.vec(scales == Scales::fixed ? 1 : m, at::kFloat, "x_scale");
    const void *sw = Args{&w_scale, 1}.vec(n, at::kFloat, "w_scale");
    const void *b = Args{&bias, 1}.vec(n, ydt, "bias");
    const at::Tensor y = result(a.next(), {m, n}, ydt, xq);
    const hq_dtype dt = hq_type(ydt);
    check(fn, call(f, static_cast<const Code *>(xq.const_data_ptr()), f32(sx),
                   static_cast<const Code *>(wq.const_data_ptr()), f32(sw), b, m, narrow(n),
                   narrow(bytes ? kb : kb * 2), y.data_ptr(), dt, stream()));
    return wrap(y);
}
PyObject *linear(Args a) { return int_linear<uint8_t>(a, "hq_int_linear", lib.hq_int_linear, Scales::dynamic); }
PyObject *linear_static(Args a) { return int_linear<uint8_t>(a, "hq_int_linear_static", lib.hq_int_linear_static, Scales::fixed); }
PyObject *linear_i8(Args a) { return int_linear<int8_t>(a, "hq_int_linear_i8", lib.hq_int_linear_i8, Scales::dynamic); }

// hq_int_conv2d, hq_int_conv2d_static, hq_int_conv2d_i8
template <class Code>
PyObject *int_conv2d(Args &a, const char *fn,
                     hq_status (*f)(const Code *, const float *, const Code *, const float *, const void *, int, int, int, int,
                                    int, int, int, int, int, void *, hq_dtype, void *),
                     Scales scales) {
    constexpr bool bytes = std::is_same<Code, int8_t>::value;
    constexpr at::ScalarType code = bytes ? at::kChar : at::kByte;
    const at::Tensor &xq = a.codes(code, "xq");
    PyObject *x_scale = a.next();
    const at::Tensor &wq = a.codes(code, "wq");
    PyObject *w_scale = a.next(), *bias = a.next();
    const int ksize = a.integer(), stride = a.integer(), pad = padding(a, ksize);
    const at::ScalarType ydt = a.dtype();
    expect_dims(xq, 4, "xq must be [nb, h, w, c]");
    const int64_t nb = xq.size(0), h = xq.size(1), w = xq.size(2), cb = xq.size(3), n = wq.dim() ? wq.size(0) : 0;
    const int64_t taps = static_cast<int64_t>(ksize) * ksize;
    expect_32bit({nb, h, w, bytes ? cb : cb * 2, n});
    if (wq.numel() != n * taps * cb) refuse("wq does not match xq / ksize");
    const void *sx = Args{&x_scale, 1}.vec(scales == Scales::fixed ? 1 : nb * h * w, at::kFloat, "x_scale");
    const void *sw = Args{&w_scale, 1}.vec(n, at::kFloat, "w_scale");
    const void *b = Args{&bias, 1}.vec(n, ydt, "bias");
    const ConvOut o = conv_out(h, w, ksize, stride, pad);
    expect_result(o);
    Shape shape{nb, o.h, o.w};
    if (ydt == at::kInt && scales == Scales::dynamic && (!bytes || taps > 1)) shape.push_back(taps);   // per-tap sums
    shape.push_back(n);
    const at::Tensor y = result(a.next(), shape, ydt, xq);
    const hq_dtype dt = hq_type(ydt);
    check(fn, call(f, static_cast<const Code *>(xq.const_data_ptr()), f32(sx),
                   static_cast<const Code *>(wq.const_data_ptr()), f32(sw), b, narrow(nb), narrow(h), narrow(w),
                   narrow(bytes ? cb : cb * 2), narrow(n), ksize, ksize, stride, pad, y.data_ptr(), dt, stream()));
    return wrap(y);
}
PyObject *conv2d(Args a) { return int_conv2d<uint8_t>(a, "hq_int_conv2d", lib.hq_int_conv2d, Scales::dynamic); }
PyObject *conv2d_static(Args a) { return int_conv2d<uint8_t>(a, "hq_int_conv2d_static", lib.hq_int_conv2d_static, Scales::fixed); }
PyObject *conv2d_i8(Args a) { return int_conv2d<int8_t>(a, "hq_int_conv2d_i8", lib.hq_int_conv2d_i8, Scales::dynamic); }

PyObject *act_quant_conv2d(Args a) {
    const at::Tensor &x = a.device("x"), &wq = a.codes(at::kByte, "wq");
    PyObject *w_scale = a.next(), *bias = a.next();
    const int block = a.integer(), bits = a.integer(), ksize = a.integer(), stride = a.integer(), pad = padding(a, ksize);
    const at::ScalarType ydt = a.dtype();
    PyObject *out = a.next(), *codes = a.next();
    const Pair codes_out(codes);
    expect_dims(x, 4, "x must be [nb, h, w, c]");
    const int64_t nb = x.size(0), h = x.size(1), w = x.size(2), cin = x.size(3), n = wq.dim() ? wq.size(0) : 0;
    const int64_t taps = static_cast<int64_t>(ksize) * ksize;
    expect_32bit({nb, h, w, cin, n});
    if (wq.numel() != n * taps * (cin / 2)) refuse("wq does not match x / ksize");
    const void *sw = Args{&w_scale, 1}.vec(n, at::kFloat, "w_scale");
    const void *b = Args{&bias, 1}.vec(n, ydt, "bias");
    const ConvOut o = conv_out(h, w, ksize, stride, pad);
    expect_result(o);
    Shape shape{nb, o.h, o.w};
    if (ydt == at::kInt) shape.push_back(taps);
    shape.push_back(n);
    const at::Tensor y = result(out, shape, ydt, x);
    at::Tensor xq, sx;
    if (codes != Py_None) {
        xq = result(codes_out.a, {nb, h, w, cin / 2}, at::kByte, x);
        sx = result(codes_out.b, {nb, h, w}, at::kFloat, x);
    }
    const hq_dtype xdt = hq_type(x.scalar_type()), dt = hq_type(ydt);
    check("hq_act_quant_int_conv2d", call(lib.hq_act_quant_int_conv2d, x.const_data_ptr(), xdt, u8(wq), f32(sw), b,
                                          narrow(nb), narrow(h), narrow(w), narrow(cin), narrow(n), ksize, ksize,
                                          stride, pad, block, bits, y.data_ptr(), dt,
                                          xq.defined() ? static_cast<uint8_t *>(xq.data_ptr()) : nullptr,
                                          sx.defined() ? static_cast<float *>(sx.data_ptr()) : nullptr, stream()));
    return wrap(y);
}

PyObject *act_quant_linear(Args a) {
    const at::Tensor &x = a.device("x"), &wq = a.codes(at::kByte, "wq");
    PyObject *w_scale = a.next(), *bias = a.next();
    const int block = a.integer(), bits = a.integer();
    const at::ScalarType ydt = a.dtype();
    PyObject *out = a.next(), *codes = a.next();
    const Pair codes_out(codes);
    if (x.dim() < 1) refuse("x must have a channel axis");
    const int64_t k = x.size(-1), m = k ? x.numel() / k : 0, n = wq.dim() ? wq.size(0) : 0;
    expect_32bit({n, k});
    if (wq.numel() != n * (k / 2)) refuse("wq does not match x");
    const void *sw = Args{&w_scale, 1}.vec(n, at::kFloat, "w_scale");
    const void *b = Args{&bias, 1}.vec(n, ydt, "bias");
    const at::Tensor y = result(out, with_last(x, n), ydt, x);
    at::Tensor xq, sx;
    if (codes != Py_None) {
        xq = result(codes_out.a, with_last(x, k / 2), at::kByte, x);
        sx = result(codes_out.b, without_last(x), at::kFloat, x);
    }
    const hq_dtype xdt = hq_type(x.scalar_type()), dt = hq_type(ydt);
    check("hq_act_quant_int_linear", call(lib.hq_act_quant_int_linear, x.const_data_ptr(), xdt, u8(wq), f32(sw), b, m,
                                          narrow(n), narrow(k), block, bits, y.data_ptr(), dt,
                                          xq.defined() ? static_cast<uint8_t *>(xq.data_ptr()) : nullptr,
                                          sx.defined() ? static_cast<float *>(sx.data_ptr()) : nullptr, stream()));
    return wrap(y);
}

PyObject *quantize_weights_single(Args a) {
    const at::Tensor &w = a.device("w");
    const int block = a.integer(), bits = a.integer();
    expect_dims(w, 2, "w must be [n_out, k_in]");
    const int64_t n = w.size(0), k = w.size(1);
    expect_32bit({n, k});
    const at::Tensor wq3 = empty({n, 3, k / 2}, at::kByte, w);
    const at::Tensor ws = empty({n}, at::kFloat, w);
    const hq_dtype dt = hq_type(w.scalar_type());
    check("hq_quantize_weights_single", call(lib.hq_quantize_weights_single, w.const_data_ptr(), dt, narrow(n),
                                             narrow(k), block, bits, static_cast<uint8_t *>(wq3.data_ptr()),
                                             static_cast<float *>(ws.data_ptr()), stream()));
    return wrap(wq3, ws);
}

PyObject *linear_single(Args a) {
    const at::Tensor &xq = a.codes(at::kByte, "xq");
    PyObject *x_scale = a.next();
    const at::Tensor &wq3 = a.codes(at::kByte, "wq3");
    PyObject *w_scale = a.next(), *bias = a.next();
    const int block = a.integer();
    const at::ScalarType ydt = a.dtype();
    expect_dims(xq, 2, "xq must be [m, k]");
    const int64_t m = xq.size(0), kb = xq.size(1), n = wq3.dim() ? wq3.size(0) : 0;
    expect_32bit({n, kb * 2});
    if (wq3.numel() != n * 3 * kb) refuse("wq3 does not match xq in k");
    const void *sx = Args{&x_scale, 1}.vec(m, at::kFloat, "x_scale");
    const void *sw = Args{&w_scale, 1}.vec(n, at::kFloat, "w_scale");
    const void *b = Args{&bias, 1}.vec(n, ydt, "bias");
    Shape shape{m, n};
    if (ydt == at::kInt) shape = {m, 3, n};
    const at::Tensor y = result(a.next(), shape, ydt, xq);
    const hq_dtype dt = hq_type(ydt);
    check("hq_int_linear_single", call(lib.hq_int_linear_single, u8(xq), f32(sx), u8(wq3), f32(sw), b, m, narrow(n),
                                       narrow(kb * 2), block, y.data_ptr(), dt, stream()));
    return wrap(y);
}

PyObject *act_hadamard_quant_width(Args a) {
    const at::Tensor &x = a.device("x");
    const float *scale = a.scalar();
    const int block = a.integer(), bits = a.integer();
    expect_dims(x, 4, "x must be [N, H, W, C]");
    const int64_t nb = x.size(0), h = x.size(1), w = x.size(2), c = x.size(3);
    expect_32bit({nb, h, w, c});
    const at::Tensor xu3 = result(a.next(), {3, nb, h, w, c / 2}, at::kByte, x);
    const hq_dtype dt = hq_type(x.scalar_type());
    check("hq_act_hadamard_quant_width", call(lib.hq_act_hadamard_quant_width, x.const_data_ptr(), dt, narrow(nb),
                                              narrow(h), narrow(w), narrow(c), block, bits, scale,
                                              static_cast<uint8_t *>(xu3.data_ptr()), stream()));
    return wrap(xu3);
}

PyObject *conv2d_width(Args a) {
    const at::Tensor &xu3 = a.codes(at::kByte, "xu3");
    PyObject *x_scale = a.next();
    const at::Tensor &wq = a.codes(at::kByte, "wq");
    PyObject *w_scale = a.next(), *bias = a.next();
    const int block = a.integer();
    const at::ScalarType ydt = a.dtype();
    PyObject *out = a.next();
    const int stride = a.integer();
    if (xu3.dim() != 5 || xu3.size(0) != 3) refuse("xu3 must be [3, N, H, W, Cin/2]");
    const int64_t nb = xu3.size(1), h = xu3.size(2), w = xu3.size(3), kb = xu3.size(4), n = wq.dim() ? wq.size(0) : 0;
    expect_32bit({nb, h, w, kb * 2, n});
    if (wq.numel() != n * 9 * kb) refuse("wq does not match xu3 in Cin or is not a 3x3 kernel");
    const void *sx = Args{&x_scale, 1}.vec(1, at::kFloat, "x_scale");
    const void *sw = Args{&w_scale, 1}.vec(n, at::kFloat, "w_scale");
    const void *b = Args{&bias, 1}.vec(n, ydt, "bias");
    const ConvOut o = conv_out(h, w, 3, stride, 1);
    expect_result(o);
    const at::Tensor y = result(out, {nb, o.h, o.w, n}, ydt, xu3);
    const hq_dtype dt = hq_type(ydt);
    check("hq_int_conv2d_width", call(lib.hq_int_conv2d_width, u8(xu3), f32(sx), u8(wq), f32(sw), b, narrow(nb),
                                      narrow(h), narrow(w), narrow(kb * 2), narrow(n), 3, 3, stride, 1, block,
                                      y.data_ptr(), dt, stream()));
    return wrap(y);
}

// ---- 8-bit floats with block scales ----------------------------------------------------------------------------
constexpr at::ScalarType kE4m3 = at::kFloat8_e4m3fn;
int64_t pitch_of(int64_t values) { return (values + 15) / 16 * 16; }
int64_t groups_of(int64_t values) { return (values + 127) / 128; }

hq_dtype float_type(at::ScalarType dt, const char *name) {
    switch (dt) {
        case at::kHalf: return HQ_F16;
        case at::kFloat: return HQ_F32;
        case at::kBFloat16: return HQ_BF16;
        default: refuse(std::string(name) + " must be torch.float16, torch.bfloat16 or torch.float32");
    }
}

bool truth(PyObject *o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw PythonError();
    return v != 0;
}

// Calls that take activations record nothing for autograd: a tensor that needs a gradient would lose it without a word.
void expect_no_gradient(const at::Tensor &t, const char *name) {
    if (t.requires_grad() && c10::GradMode::is_enabled())
        refuse(std::string(name) + " requires a gradient, which this call does not record: make it under torch.no_grad() (or in an "
                                   "autograd function), with the _backward call for gradients");
}
void expect_no_gradient(PyObject *o, const char *name) {
    if (THPVariable_Check(o)) expect_no_gradient(THPVariable_Unpack(o), name);
}

// A matrix of contiguous rows: a contiguous tensor, its leading axes taken together, or a matrix whose rows are apart.
struct Rows {
    const at::Tensor &t;
    hq_dtype type;
    int64_t m, k, stride;
};
Rows rows_of(Args &a, const char *name) {
    const at::Tensor &t = a.tensor(name);
    if (!t.is_cuda()) refuse(std::string(name) + " must be a device tensor");
    if (t.dim() < 1) refuse(std::string(name) + " must have a channel axis");
    const int64_t k = t.size(-1);
    if (k < 1) refuse(std::string(name) + " has no channels");
    const hq_dtype type = float_type(t.scalar_type(), name);
    expect_32bit({k});
    if (t.is_contiguous()) return {t, type, t.numel() / k, k, k};
    if (t.dim() != 2 || (t.stride(1) != 1 && k > 1) || t.stride(0) < 0)
        refuse(std::string(name) + " must be contiguous, or a matrix of contiguous rows");
    return {t, type, t.size(0), k, t.stride(0)};
}

const at::Tensor &fp8_codes(Args &a, const char *name) {
    const at::Tensor &t = a.device(name);
    if (t.scalar_type() != kE4m3) refuse(std::string(name) + " must hold torch.float8_e4m3fn codes");
    if (t.dim() < 1 || t.size(-1) < 1 || t.size(-1) % 16) refuse(std::string(name) + " must have rows of a multiple of 16 codes");
    return t;
}

// scales [rows, columns], or the transposed view of such a matrix that is contiguous: then *turned
const float *block_scales(Args &a, const char *name, int64_t rows, int64_t columns, int *turned) {
    const at::Tensor &t = a.tensor(name);
    const bool plain = t.is_contiguous();
    if (!t.is_cuda() || t.scalar_type() != at::kFloat || t.dim() != 2 || t.size(0) != rows || t.size(1) != columns ||
        (!plain && !(t.stride(0) == 1 && t.stride(1) == rows)))
        refuse(std::string(name) + " must be a device tensor of Float, [" + std::to_string(rows) + ", " + std::to_string(columns) +
               "], contiguous or the transposed view of a contiguous one");
    *turned = plain ? 0 : 1;
    return static_cast<const float *>(t.const_data_ptr());
}

// memory as the checks of results see it: a matrix of rows, a tensor [t, heads, d], and what lies in one piece
hq::Rows2 memory_of(const Rows &r) {
    const int64_t size = static_cast<int64_t>(r.t.element_size());
    return {reinterpret_cast<int64_t>(r.t.const_data_ptr()), {r.m, 1}, {r.stride * size, 0}, r.k * size};
}
hq::Rows2 memory_of(const at::Tensor &t) {
    const int64_t size = static_cast<int64_t>(t.element_size());
    const int64_t at = reinterpret_cast<int64_t>(t.const_data_ptr());
    return {at, {t.size(0), t.size(1)}, {t.stride(0) * size, t.stride(1) * size}, t.size(2) * size};
}
hq::Rows2 memory_of(const void *p, int64_t bytes) { return {reinterpret_cast<int64_t>(p), {1, 1}, {0, 0}, p ? bytes : 0}; }
void expect_apart(const hq::Rows2 &a, const hq::Rows2 &b, const char *name, const char *other) {
    if (hq::rows_overlap(a, b)) refuse(std::string(name) + " must not overlap " + other);
}
hq::Rows2 piece_of(const at::Tensor &t) { return memory_of(t.const_data_ptr(), static_cast<int64_t>(t.nbytes())); }
// A caller's buffer for y: the workgroups of one launch write it while others still read.
void expect_result_apart(PyObject *out, const at::Tensor &y, const hq::Rows2 &x, const char *x_name, const at::Tensor &wq,
                         const float *w_scale, int64_t scales, const void *bias, int64_t n) {
    if (out == Py_None) return;
    const hq::Rows2 to = piece_of(y);
    expect_apart(to, x, "out", x_name);
    expect_apart(to, piece_of(wq), "out", "wq");
    expect_apart(to, memory_of(w_scale, scales * 4), "out", "w_scale");
    expect_apart(to, memory_of(bias, n * static_cast<int64_t>(y.element_size())), "out", "bias");
}

PyObject *fp8_quantize_rows(Args a) {
    const Rows x = rows_of(a, "x");
    expect_no_gradient(x.t, "x");
    const at::Tensor xq = empty(with_last(x.t, pitch_of(x.k)), kE4m3, x.t);
    const at::Tensor xs = empty({groups_of(x.k), x.m}, at::kFloat, x.t);
    check("hq_fp8_quantize_rows", call(lib.hq_fp8_quantize_rows, x.t.const_data_ptr(), x.type, x.m, narrow(x.k), x.stride,
                                       static_cast<uint8_t *>(xq.data_ptr()), static_cast<float *>(xs.data_ptr()), stream()));
    return wrap(xq, xs);
}

PyObject *fp8_quantize_blocks(Args a) {
    const Rows w = rows_of(a, "w");
    const bool transposed = truth(a.next());
    expect_dims(w.t, 2, "w must be [n, k]");
    if (w.m < 1) refuse("w has no rows");
    const at::Tensor wq = empty({w.m, pitch_of(w.k)}, kE4m3, w.t);
    const at::Tensor ws = empty({groups_of(w.m), groups_of(w.k)}, at::kFloat, w.t);
    at::Tensor wt;
    if (transposed) wt = empty({w.k, pitch_of(w.m)}, kE4m3, w.t);
    check("hq_fp8_quantize_blocks", call(lib.hq_fp8_quantize_blocks, w.t.const_data_ptr(), w.type, w.m, narrow(w.k), w.stride,
                                         static_cast<uint8_t *>(wq.data_ptr()),
                                         transposed ? static_cast<uint8_t *>(wt.data_ptr()) : nullptr,
                                         static_cast<float *>(ws.data_ptr()), stream()));
    return transposed ? wrap({wq, wt, ws}) : wrap(wq, ws);
}

PyObject *fp8_linear(Args a) {
    const at::Tensor &xq = fp8_codes(a, "xq");
    const int64_t kp = xq.size(-1), m = xq.numel() / kp;
    expect_32bit({kp});
    const at::Tensor &sx = a.device("x_scale");
    if (sx.scalar_type() != at::kFloat || sx.numel() != groups_of(kp) * m || sx.dim() < 1 || sx.size(0) != groups_of(kp))
        refuse("x_scale must be a contiguous device tensor of Float, [" + std::to_string(groups_of(kp)) + ", " + std::to_string(m) + "]");
    const at::Tensor &wq = fp8_codes(a, "wq");
    if (wq.dim() != 2 || wq.size(1) != kp) refuse("wq does not match xq in k");
    const int64_t n = wq.size(0);
    expect_32bit({n});
    int turned = 0;
    const float *sw = block_scales(a, "w_scale", groups_of(n), groups_of(kp), &turned);
    PyObject *bias = a.next();
    expect_no_gradient(bias, "bias");
    const at::ScalarType ydt = a.dtype();
    const hq_dtype dt = float_type(ydt, "y_dtype");
    const void *b = Args{&bias, 1}.vec(n, ydt, "bias");
    PyObject *out = a.next();
    const at::Tensor y = result(out, with_last(xq, n), ydt, xq);
    expect_result_apart(out, y, piece_of(xq), "xq", wq, sw, groups_of(n) * groups_of(kp), b, n);
    if (out != Py_None) expect_apart(piece_of(y), piece_of(sx), "out", "x_scale");
    check("hq_fp8_linear", call(lib.hq_fp8_linear, u8(xq), f32(sx.const_data_ptr()), u8(wq), sw, turned, b, m, narrow(n), narrow(kp),
                                y.data_ptr(), dt, stream()));
    return wrap(y);
}

PyObject *act_quant_fp8_linear(Args a) {
    const Rows x = rows_of(a, "x");
    expect_no_gradient(x.t, "x");
    const at::Tensor &wq = fp8_codes(a, "wq");
    if (wq.dim() != 2 || wq.size(1) != pitch_of(x.k)) refuse("wq does not match x in k");
    const int64_t n = wq.size(0);
    expect_32bit({n});
    int turned = 0;
    const float *sw = block_scales(a, "w_scale", groups_of(n), groups_of(x.k), &turned);
    if (turned) refuse("w_scale must be contiguous");
    PyObject *bias = a.next();
    expect_no_gradient(bias, "bias");
    const at::ScalarType ydt = a.dtype();
    const hq_dtype dt = float_type(ydt, "y_dtype");
    const void *b = Args{&bias, 1}.vec(n, ydt, "bias");
    PyObject *out = a.next();
    const at::Tensor y = result(out, with_last(x.t, n), ydt, x.t);
    expect_result_apart(out, y, memory_of(x), "x", wq, sw, groups_of(n) * groups_of(x.k), b, n);
    at::Tensor space;
    const int64_t bytes = lib.hq_act_quant_fp8_linear_workspace(x.type, x.m, narrow(n), narrow(x.k), dt);
    if (bytes) space = empty({bytes}, at::kByte, x.t);
    check("hq_act_quant_fp8_linear", call(lib.hq_act_quant_fp8_linear, x.t.const_data_ptr(), x.type, x.stride, u8(wq), sw, b, x.m,
                                          narrow(n), narrow(x.k), bytes ? space.data_ptr() : nullptr, y.data_ptr(), dt, stream()));
    return wrap(y);
}

PyObject *fp8_linear_backward(Args a) {
    const Rows dy = rows_of(a, "dy"), x = rows_of(a, "x");
    if (x.type != dy.type) refuse("dy and x must have one type");
    if (x.m != dy.m) refuse("dy does not match x in rows");
    const at::Tensor &wt = fp8_codes(a, "wq_t");
    if (wt.dim() != 2 || wt.size(0) != x.k || wt.size(1) != pitch_of(dy.k)) refuse("wq_t does not match x and dy");
    int turned = 0;
    const float *sw = block_scales(a, "w_scale", groups_of(dy.k), groups_of(x.k), &turned);
    if (turned) refuse("w_scale must be contiguous");
    const bool bias = truth(a.next());
    const at::Tensor dx = empty(with_last(x.t, x.k), x.t.scalar_type(), x.t);
    const at::Tensor dw = empty({dy.k, x.k}, at::kFloat, x.t);
    at::Tensor db;
    if (bias) db = empty({dy.k}, at::kFloat, x.t);
    const at::Tensor space = empty({lib.hq_fp8_linear_backward_workspace(x.m, narrow(dy.k), narrow(x.k))}, at::kByte, x.t);
    check("hq_fp8_linear_backward",
          call(lib.hq_fp8_linear_backward, dy.t.const_data_ptr(), dy.stride, x.t.const_data_ptr(), x.stride, x.type, u8(wt), sw, x.m,
               narrow(dy.k), narrow(x.k), space.data_ptr(), dx.data_ptr(), static_cast<float *>(dw.data_ptr()),
               bias ? static_cast<float *>(db.data_ptr()) : nullptr, stream()));
    return wrap({dx, dw, db});
}

// ---- query and key heads ---------------------------------------------------------------------------------------------
// [t, heads, d] with contiguous channels
const at::Tensor &heads_of(PyObject *o, const char *name, const at::Tensor *like) {
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s must be a tensor", name);
        throw PythonError();
    }
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.dim() != 3 || (t.stride(2) != 1 && t.size(2) > 1))
        refuse(std::string(name) + " must be a device tensor [tokens, heads, channels] with contiguous channels");
    if (like && (t.scalar_type() != like->scalar_type() || t.sizes() != like->sizes()))
        refuse(std::string(name) + " has another type or shape than what it belongs to");
    return t;
}
// memory that is written through strides: no element twice
void expect_distinct(const at::Tensor &t, const char *name) {
    const int64_t n0 = t.size(0), n1 = t.size(1), d = t.size(2), s0 = t.stride(0), s1 = t.stride(1);
    const bool heads_inside = (n1 < 2 || s1 >= d) && (n0 < 2 || s0 >= (n1 - 1) * s1 + d);
    const bool tokens_inside = (n0 < 2 || s0 >= d) && (n1 < 2 || s1 >= (n0 - 1) * s0 + d);
    if (!heads_inside && !tokens_inside) refuse(std::string(name) + " must not overlap itself");
}

struct Qk {
    const at::Tensor &q, &k;
    hq_dtype type, weight_type;
    const void *q_weight, *k_weight;
    const float *cos, *sin;
    int64_t positions;
    int rotary;
    const void *pos;
    int pos_size;
    float eps;
    int interleaved;
    PyObject *weights[2];
    int64_t t() const { return q.size(0); }
    int d() const { return narrow(q.size(2)); }
    int heads() const { return narrow(q.size(1)); }
    int kv_heads() const { return narrow(k.size(1)); }
};
Qk qk_of(Args &a) {
    const at::Tensor &q = heads_of(a.next(), "q", nullptr), &k = heads_of(a.next(), "k", nullptr);
    const hq_dtype type = float_type(q.scalar_type(), "q");
    if (k.scalar_type() != q.scalar_type() || k.size(0) != q.size(0) || k.size(2) != q.size(2)) refuse("k does not match q");
    expect_32bit({q.size(1), k.size(1), q.size(2)});
    PyObject *w[2] = {a.next(), a.next()};
    at::ScalarType wdt = q.scalar_type();
    for (PyObject *o : w)
        if (THPVariable_Check(o) && THPVariable_Unpack(o).scalar_type() == at::kFloat) wdt = at::kFloat;
    const void *qw = Args{&w[0], 1}.vec(q.size(2), wdt, "q_weight"), *kw = Args{&w[1], 1}.vec(q.size(2), wdt, "k_weight");
    const at::Tensor &cos = a.device("cos"), &sin = a.device("sin");
    if (cos.scalar_type() != at::kFloat || sin.scalar_type() != at::kFloat || cos.dim() != 2 || cos.sizes() != sin.sizes())
        refuse("cos and sin must be Float, [positions, rotary / 2]");
    expect_32bit({cos.size(1) * 2});
    const void *pos = nullptr;
    int pos_size = 0;
    if (a.none()) {
        a.next();
    } else {
        const at::Tensor &p = a.device("positions");
        if ((p.scalar_type() != at::kInt && p.scalar_type() != at::kLong) || p.numel() != q.size(0))
            refuse("positions must hold one torch.int32 or torch.int64 for each token");
        pos = p.const_data_ptr();
        pos_size = p.scalar_type() == at::kLong ? 8 : 4;
    }
    const double eps = PyFloat_AsDouble(a.next());
    if (eps == -1.0 && PyErr_Occurred()) throw PythonError();
    const bool interleaved = truth(a.next());
    return {q, k, type, float_type(wdt, "q_weight"), qw, kw, f32(cos.const_data_ptr()), f32(sin.const_data_ptr()), cos.size(0),
            narrow(cos.size(1) * 2), pos, pos_size, static_cast<float>(eps), interleaved ? 1 : 0, {w[0], w[1]}};
}

// The results: new, or the caller's.  Workgroups read their inputs while others write: a result may lie on the input that the same
// workgroup reads (q, or dq where there is one, for that of q), and shares memory with nothing else.
struct QkOut {
    at::Tensor q, k;
    QkOut(PyObject *out, const Qk &in, const at::Tensor *dq = nullptr, const at::Tensor *dk = nullptr) {
        if (out == Py_None) {
            q = empty(in.q.sizes(), in.q.scalar_type(), in.q);
            k = empty(in.k.sizes(), in.k.scalar_type(), in.k);
            return;
        }
        const Pair pair(out);
        q = heads_of(pair.a, "out[0]", &in.q);
        k = heads_of(pair.b, "out[1]", &in.k);
        expect_distinct(q, "out[0]");
        expect_distinct(k, "out[1]");
        const hq::Rows2 to_q = memory_of(q), to_k = memory_of(k);
        expect_apart(to_q, to_k, "out[0]", "out[1]");
        expect_inputs(to_q, "out[0]", in, in.q, dq, "q, unless it is q", "dq, unless it is dq", in.k, dk, "k", "dk");
        expect_inputs(to_k, "out[1]", in, in.k, dk, "k, unless it is k", "dk, unless it is dk", in.q, dq, "q", "dq");
    }

private:
    static void expect_inputs(const hq::Rows2 &to, const char *name, const Qk &in, const at::Tensor &own, const at::Tensor *own_grad,
                              const char *own_name, const char *own_grad_name, const at::Tensor &other, const at::Tensor *other_grad,
                              const char *other_name, const char *other_grad_name) {
        const auto own_or_apart = [&](const at::Tensor &t, const char *text) {
            const hq::Rows2 m = memory_of(t);
            if (!hq::same_rows(to, m)) expect_apart(to, m, name, text);
        };
        own_or_apart(own, own_name);
        if (own_grad) own_or_apart(*own_grad, own_grad_name);
        expect_apart(to, memory_of(other), name, other_name);
        if (other_grad) expect_apart(to, memory_of(*other_grad), name, other_grad_name);
        const int64_t weight = in.q.size(2) * (in.weight_type == HQ_F32 ? 4 : 2), table = in.positions * in.rotary * 2;
        expect_apart(to, memory_of(in.q_weight, weight), name, "q_weight");
        expect_apart(to, memory_of(in.k_weight, weight), name, "k_weight");
        expect_apart(to, memory_of(in.cos, table), name, "cos");
        expect_apart(to, memory_of(in.sin, table), name, "sin");
        expect_apart(to, memory_of(in.pos, in.q.size(0) * in.pos_size), name, "positions");
    }
};

PyObject *qk_norm_rope(Args a) {
    const Qk in = qk_of(a);
    expect_no_gradient(in.q, "q");
    expect_no_gradient(in.k, "k");
    expect_no_gradient(in.weights[0], "q_weight");
    expect_no_gradient(in.weights[1], "k_weight");
    const QkOut out(a.next(), in);
    const int64_t strides[8] = {in.q.stride(0), in.q.stride(1), in.k.stride(0), in.k.stride(1),
                                out.q.stride(0), out.q.stride(1), out.k.stride(0), out.k.stride(1)};
    check("hq_qk_norm_rope", call(lib.hq_qk_norm_rope, in.q.const_data_ptr(), in.k.const_data_ptr(), in.type, in.t(), in.heads(),
                                  in.kv_heads(), in.d(), static_cast<const int64_t *>(strides), in.q_weight, in.k_weight, in.weight_type,
                                  in.cos, in.sin, in.positions, in.rotary, in.interleaved, in.pos, in.pos_size, in.eps,
                                  out.q.data_ptr(), out.k.data_ptr(), stream()));
    return wrap(out.q, out.k);
}

PyObject *qk_norm_rope_backward(Args a) {
    PyObject *dq_o = a.next(), *dk_o = a.next();
    const Qk in = qk_of(a);
    const at::Tensor &dq = heads_of(dq_o, "dq", &in.q), &dk = heads_of(dk_o, "dk", &in.k);
    const QkOut out(a.next(), in, &dq, &dk);
    at::Tensor qw, kw;
    if (in.q_weight) qw = empty({in.d()}, at::kFloat, in.q);
    if (in.k_weight) kw = empty({in.d()}, at::kFloat, in.q);
    const at::Tensor space = empty({lib.hq_qk_norm_rope_backward_workspace(in.type, in.t(), in.heads(), in.kv_heads(), in.d(), in.rotary)},
                                   at::kByte, in.q);
    const int64_t strides[12] = {in.q.stride(0), in.q.stride(1), in.k.stride(0), in.k.stride(1), dq.stride(0), dq.stride(1),
                                 dk.stride(0), dk.stride(1), out.q.stride(0), out.q.stride(1), out.k.stride(0), out.k.stride(1)};
    check("hq_qk_norm_rope_backward",
          call(lib.hq_qk_norm_rope_backward, dq.const_data_ptr(), dk.const_data_ptr(), in.q.const_data_ptr(), in.k.const_data_ptr(),
               in.type, in.t(), in.heads(), in.kv_heads(), in.d(), static_cast<const int64_t *>(strides), in.q_weight, in.k_weight,
               in.weight_type, in.cos, in.sin, in.positions, in.rotary, in.interleaved, in.pos, in.pos_size, in.eps, space.data_ptr(),
               out.q.data_ptr(), out.k.data_ptr(), qw.defined() ? static_cast<float *>(qw.data_ptr()) : nullptr,
               kw.defined() ? static_cast<float *>(kw.data_ptr()) : nullptr, stream()));
    return wrap({out.q, out.k, qw, kw});
}

// ---- module -----------------------------------------------------------------------------------------------------
template <PyObject *(*F)(Args)>
PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n) {
    try {
        return F(Args{args, n});
    } catch (const PythonError &) {
        return nullptr;
    } catch (const std::exception &e) {   // (an allocation that failed)
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// bind({name: address}, HqError)
PyObject *bind(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 2 || !PyDict_Check(args[0])) {
        PyErr_SetString(PyExc_TypeError, "bind(addresses, error class)");
        return nullptr;
    }
    Library l{};
#define X(name)                                                                   \
    {                                                                             \
        PyObject *v = PyDict_GetItemString(args[0], #name);                       \
        void *p = v ? PyLong_AsVoidPtr(v) : nullptr;                              \
        if (!p) {                                                                 \
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_KeyError, #name);        \
            return nullptr;                                                       \
        }                                                                         \
        l.name = reinterpret_cast<decltype(l.name)>(p);                           \
    }
    HQ_ENTRY_POINTS(X)
#undef X
    lib = l;
    Py_INCREF(args[1]);
    Py_XDECREF(error_class);
    error_class = args[1];
    Py_RETURN_NONE;
}

#define HQ_METHOD(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(entry<f>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    HQ_METHOD(quantize_weights), HQ_METHOD(act_hadamard_quant), HQ_METHOD(act_hadamard_quant_i8),
    HQ_METHOD(act_hadamard_quant_static), HQ_METHOD(linear), HQ_METHOD(linear_static), HQ_METHOD(linear_i8),
    HQ_METHOD(conv2d), HQ_METHOD(conv2d_static), HQ_METHOD(conv2d_i8),
    HQ_METHOD(act_quant_conv2d), HQ_METHOD(act_quant_linear), HQ_METHOD(quantize_weights_single), HQ_METHOD(linear_single),
    HQ_METHOD(act_hadamard_quant_width), HQ_METHOD(conv2d_width),
    HQ_METHOD(fp8_quantize_rows), HQ_METHOD(fp8_quantize_blocks), HQ_METHOD(fp8_linear), HQ_METHOD(act_quant_fp8_linear),
    HQ_METHOD(fp8_linear_backward), HQ_METHOD(qk_norm_rope), HQ_METHOD(qk_norm_rope_backward),
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(bind)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "Argument marshalling of the HIP library.", -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
