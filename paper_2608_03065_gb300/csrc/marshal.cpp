// A Python module (_marshal) that does for the small calls what psc.py does for all: takes torch
// tensors apart into addresses and strides, checks them, and calls the library's entry.  Each attribute of
// a tensor costs about as much from here as from Python, but what lies between them does not: a norm's call takes
// the host 4.4 us this way and 7.6 from Python.  A call that is not plainly in order gets None back and goes
// through psc.py's own checks, which say what is wrong with it.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <cstdint>

namespace {

PyObject *s_shape, *s_dtype, *s_stride, *s_data_ptr, *s_numel, *s_is_contiguous, *s_get_device;
PyObject *t_bf16, *t_f32, *t_i8, *t_u8, *t_i32;

using NormRows = int32_t (*)(const void*, int32_t, int64_t, const void*, int64_t, void*, int64_t, const float*, float,
                             int32_t, int32_t, void*, int64_t, float*, void*);
using NormMx4 = int32_t (*)(const void*, int32_t, int64_t, const void*, int64_t, void*, int64_t, const float*, float,
                            int32_t, int32_t, void*, int64_t, void*, float*, void*);
using Quantize = int32_t (*)(const void*, int32_t, int64_t, int32_t, int32_t, void*, int64_t, void*, void*);
using Dequantize = int32_t (*)(const void*, int64_t, const void*, const float*, int32_t, int32_t, void*, int32_t, int64_t,
                               void*);
using HeadMx4 = int32_t (*)(const void*, int64_t, const void*, const float*, int32_t, const void*, int64_t, const void*,
                            const float*, int32_t, int32_t, const void*, void*, int32_t, int64_t, void*);
NormRows norm_rows_entry;
NormMx4 norm_mx4_entry;
Quantize quantize_entry;
Dequantize dequantize_entry;
HeadMx4 head_entry;

// An owned reference.
struct Ref {
    PyObject* p;
    explicit Ref(PyObject* o) : p(o) {}
    Ref(const Ref&) = delete;
    ~Ref() { Py_XDECREF(p); }
};

bool attribute_is(PyObject* t, PyObject* name, PyObject* value) {
    const Ref a(PyObject_GetAttr(t, name));
    return a.p == value;
}
bool number(PyObject* t, PyObject* method, int64_t* out) {
    const Ref r(PyObject_CallMethodNoArgs(t, method));
    if (!r.p || !PyLong_Check(r.p)) return false;
    *out = (int64_t)PyLong_AsUnsignedLongLong(r.p);       // addresses may have the top bit; -1 is an error
    return !PyErr_Occurred();
}
// The two numbers of a tuple.
bool two(PyObject* tuple, int64_t* a, int64_t* b) {
    if (!tuple || !PyTuple_Check(tuple) || PyTuple_GET_SIZE(tuple) != 2) return false;
    *a = PyLong_AsLongLong(PyTuple_GET_ITEM(tuple, 0));
    *b = PyLong_AsLongLong(PyTuple_GET_ITEM(tuple, 1));
    return !PyErr_Occurred();
}
bool size_of(PyObject* t, int64_t* rows, int64_t* cols) {
    const Ref shape(PyObject_GetAttr(t, s_shape));
    return two(shape.p, rows, cols) && *rows >= 0 && *rows <= INT32_MAX && *cols > 0 && *cols <= INT32_MAX;
}
// The current device, by psc.py's _device: every tensor of a call has to be on it (those of the host give -1).
PyObject* device_function;
struct Device {
    int64_t id = -1;
    bool take() {
        const Ref here(PyObject_CallNoArgs(device_function));
        if (!here.p || !PyLong_Check(here.p)) return false;
        id = PyLong_AsLongLong(here.p);
        return id >= 0;
    }
    bool has(PyObject* t, PyObject* dtype) const {
        int64_t device;
        return attribute_is(t, s_dtype, dtype) && number(t, s_get_device, &device) && device == id;
    }
};

// A 2-D tensor of `rows` rows and at least `cols` columns, neighbouring in memory.
struct Matrix {
    int64_t at = 0, stride = 0;
    bool take(const Device& on, PyObject* t, PyObject* dtype, int64_t rows, int64_t cols) {
        int64_t r, c, unit;
        if (!on.has(t, dtype) || !size_of(t, &r, &c) || r != rows || c < cols) return false;
        const Ref strides(PyObject_CallMethodNoArgs(t, s_stride));
        if (!two(strides.p, &stride, &unit) || unit != 1) return false;
        if (rows == 1 && stride < c) stride = c;                // a row of its own may carry any stride
        return number(t, s_data_ptr, &at);
    }
    bool take_or_none(const Device& on, PyObject* t, PyObject* dtype, int64_t rows, int64_t cols) {
        return t == Py_None || take(on, t, dtype, rows, cols);
    }
};
// A contiguous tensor of at least n elements.
struct Vector {
    int64_t at = 0;
    bool take(const Device& on, PyObject* t, PyObject* dtype, int64_t n) {
        int64_t has;
        if (!on.has(t, dtype) || !number(t, s_numel, &has) || has < n) return false;
        const Ref contiguous(PyObject_CallMethodNoArgs(t, s_is_contiguous));
        return contiguous.p == Py_True && number(t, s_data_ptr, &at);
    }
    bool take_or_none(const Device& on, PyObject* t, PyObject* dtype, int64_t n) { return t == Py_None || take(on, t, dtype, n); }
};
// A matrix in 4 bits.
struct Mx4 {
    Matrix codes;
    Vector blocks;
    bool take(const Device& on, PyObject* q, PyObject* b, int64_t rows, int64_t K) {
        return codes.take(on, q, t_u8, rows, (K + 31) / 32 * 16) &&
               blocks.take(on, b, t_u8, (rows + 127) / 128 * ((K + 127) / 128) * 512);
    }
};
// bf16 or f32, as the library counts them; -1: neither.
int32_t code_of(PyObject* t, PyObject** dtype) {
    const Ref d(PyObject_GetAttr(t, s_dtype));
    *dtype = d.p;                               // torch keeps its types
    return d.p == t_bf16 ? 1 : d.p == t_f32 ? 0 : -1;
}
template <typename P = void>
P* at(int64_t a) {
    return reinterpret_cast<P*>(static_cast<uintptr_t>(a));
}
// The handle of a stream argument, by psc.py's _stream.
PyObject* stream_function;
bool stream_of(PyObject* argument, void** out) {
    const Ref s(PyObject_CallOneArg(stream_function, argument));
    if (!s.p) return false;
    *out = s.p == Py_None ? nullptr : at((int64_t)PyLong_AsUnsignedLongLong(s.p));
    return !PyErr_Occurred();
}

PyObject* not_plain() {
    PyErr_Clear();
    Py_RETURN_NONE;
}
// Calls the library without the interpreter's lock.
template <typename F>
PyObject* called(F f) {
    int32_t code;
    Py_BEGIN_ALLOW_THREADS;
    code = f();
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong(code);
}

struct NormInputs {
    int64_t T = 0, K = 0;
    int32_t code = 0;
    Matrix x, residual, sum;
    Vector gain;
    float eps = 0;
    bool take(const Device& on, PyObject* px, PyObject* pgain, PyObject* peps, PyObject* presidual, PyObject* psum) {
        PyObject* dtype;
        code = code_of(px, &dtype);
        if (code < 0 || !size_of(px, &T, &K)) return false;
        eps = (float)PyFloat_AsDouble(peps);
        return !PyErr_Occurred() && x.take(on, px, dtype, T, K) && residual.take_or_none(on, presidual, dtype, T, K) &&
               sum.take_or_none(on, psum, dtype, T, K) && gain.take_or_none(on, pgain, t_f32, K);
    }
};

// norm_rows(x, q, scale, gain, eps, residual, sum_out, stream)
PyObject* norm_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
    Device on;
    NormInputs i;
    Matrix q;
    Vector scale;
    if (n != 8 || !on.take() || !i.take(on, a[0], a[3], a[4], a[5], a[6]) || !q.take(on, a[1], t_i8, i.T, i.K) ||
        !scale.take(on, a[2], t_f32, i.T))
        return not_plain();
    void* stream;
    if (!stream_of(a[7], &stream)) return nullptr;
    return called([&] {
        return norm_rows_entry(at(i.x.at), i.code, i.x.stride, at(i.residual.at), i.residual.stride, at(i.sum.at),
                               i.sum.stride, at<float>(i.gain.at), i.eps, (int32_t)i.T, (int32_t)i.K, at(q.at), q.stride,
                               at<float>(scale.at), stream);
    });
}

// norm_mx4(x, q, blocks, scale, gain, eps, residual, sum_out, stream)
PyObject* norm_mx4(PyObject*, PyObject* const* a, Py_ssize_t n) {
    Device on;
    NormInputs i;
    Mx4 q;
    Vector scale;
    if (n != 9 || !on.take() || !i.take(on, a[0], a[4], a[5], a[6], a[7]) || !q.take(on, a[1], a[2], i.T, i.K) ||
        !scale.take(on, a[3], t_f32, i.T))
        return not_plain();
    void* stream;
    if (!stream_of(a[8], &stream)) return nullptr;
    return called([&] {
        return norm_mx4_entry(at(i.x.at), i.code, i.x.stride, at(i.residual.at), i.residual.stride, at(i.sum.at),
                              i.sum.stride, at<float>(i.gain.at), i.eps, (int32_t)i.T, (int32_t)i.K, at(q.codes.at),
                              q.codes.stride, at(q.blocks.at), at<float>(scale.at), stream);
    });
}

// quantize_mx4(x, q, blocks, stream)
PyObject* quantize_mx4(PyObject*, PyObject* const* a, Py_ssize_t n) {
    Device on;
    int64_t T, K;
    PyObject* dtype;
    Matrix x;
    Mx4 q;
    if (n != 4 || !on.take()) return not_plain();
    const int32_t code = code_of(a[0], &dtype);
    if (code < 0 || !size_of(a[0], &T, &K) || !x.take(on, a[0], dtype, T, K) || !q.take(on, a[1], a[2], T, K))
        return not_plain();
    void* stream;
    if (!stream_of(a[3], &stream)) return nullptr;
    return called([&] {
        return quantize_entry(at(x.at), code, x.stride, (int32_t)T, (int32_t)K, at(q.codes.at), q.codes.stride,
                              at(q.blocks.at), stream);
    });
}

// dequantize_mx4(q, blocks, y, scale, stream)
PyObject* dequantize_mx4(PyObject*, PyObject* const* a, Py_ssize_t n) {
    Device on;
    int64_t T, K;
    PyObject* dtype;
    Matrix y;
    Mx4 q;
    Vector scale;
    if (n != 5 || !on.take()) return not_plain();
    const int32_t code = code_of(a[2], &dtype);
    if (code < 0 || !size_of(a[2], &T, &K) || !y.take(on, a[2], dtype, T, K) || !q.take(on, a[0], a[1], T, K) ||
        !scale.take_or_none(on, a[3], t_f32, T))
        return not_plain();
    void* stream;
    if (!stream_of(a[4], &stream)) return nullptr;
    return called([&] {
        return dequantize_entry(at(q.codes.at), q.codes.stride, at(q.blocks.at), at<float>(scale.at), (int32_t)T,
                                (int32_t)K, at(y.at), code, y.stride, stream);
    });
}

// head_logits_mx4(q, q_blocks, w, w_blocks, logits, K, scale, w_scale, bitmask, stream)
PyObject* head_logits_mx4(PyObject*, PyObject* const* a, Py_ssize_t n) {
    Device on;
    int64_t T, V, c;
    PyObject* dtype;
    Mx4 q, w;
    Matrix logits;
    Vector scale, w_scale, mask;
    if (n != 10 || !PyLong_Check(a[5]) || !on.take()) return not_plain();
    const int64_t K = PyLong_AsLongLong(a[5]);
    if (PyErr_Occurred() || K <= 0 || K > INT32_MAX) return not_plain();
    const int32_t code = code_of(a[4], &dtype);
    if (code < 0 || !size_of(a[0], &T, &c) || !size_of(a[2], &V, &c) || !q.take(on, a[0], a[1], T, K) ||
        !w.take(on, a[2], a[3], V, K) || !logits.take(on, a[4], dtype, T, V) || !scale.take_or_none(on, a[6], t_f32, T) ||
        !w_scale.take_or_none(on, a[7], t_f32, V))
        return not_plain();
    if (a[8] != Py_None) {
        int64_t rows, words;
        if (!size_of(a[8], &rows, &words) || rows != T || words != (V + 31) / 32 || !mask.take(on, a[8], t_i32, T * words))
            return not_plain();
    }
    void* stream;
    if (!stream_of(a[9], &stream)) return nullptr;
    return called([&] {
        return head_entry(at(q.codes.at), q.codes.stride, at(q.blocks.at), at<float>(scale.at), (int32_t)T, at(w.codes.at),
                          w.codes.stride, at(w.blocks.at), at<float>(w_scale.at), (int32_t)V, (int32_t)K, at(mask.at),
                          at(logits.at), code, logits.stride, stream);
    });
}

// setup((bfloat16, float32, int8, uint8, int32), (addresses of the entries), psc._stream, psc._device)
PyObject* setup(PyObject*, PyObject* args) {
    PyObject* types[5];
    unsigned long long e[5];
    if (!PyArg_ParseTuple(args, "(OOOOO)(KKKKK)OO", &types[0], &types[1], &types[2], &types[3], &types[4], &e[0], &e[1], &e[2],
                          &e[3], &e[4], &stream_function,
                          &device_function))
        return nullptr;
    for (PyObject* t : types) Py_INCREF(t);
    Py_INCREF(stream_function);
    Py_INCREF(device_function);
    t_bf16 = types[0], t_f32 = types[1], t_i8 = types[2], t_u8 = types[3], t_i32 = types[4];
    norm_rows_entry = reinterpret_cast<NormRows>((uintptr_t)e[0]);
    norm_mx4_entry = reinterpret_cast<NormMx4>((uintptr_t)e[1]);
    quantize_entry = reinterpret_cast<Quantize>((uintptr_t)e[2]);
    dequantize_entry = reinterpret_cast<Dequantize>((uintptr_t)e[3]);
    head_entry = reinterpret_cast<HeadMx4>((uintptr_t)e[4]);
    Py_RETURN_NONE;
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyCFunction fast() {
    return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(F));
}
PyMethodDef methods[] = {{"setup", setup, METH_VARARGS, nullptr},
                         {"norm_rows", fast<norm_rows>(), METH_FASTCALL, nullptr},
                         {"norm_mx4", fast<norm_mx4>(), METH_FASTCALL, nullptr},
                         {"quantize_mx4", fast<quantize_mx4>(), METH_FASTCALL, nullptr},
                         {"dequantize_mx4", fast<dequantize_mx4>(), METH_FASTCALL, nullptr},
                         {"head_logits_mx4", fast<head_logits_mx4>(), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) {
    s_shape = PyUnicode_InternFromString("shape");
    s_dtype = PyUnicode_InternFromString("dtype");
    s_stride = PyUnicode_InternFromString("stride");
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_numel = PyUnicode_InternFromString("numel");
    s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    s_get_device = PyUnicode_InternFromString("get_device");
    return PyModule_Create(&module);
}
