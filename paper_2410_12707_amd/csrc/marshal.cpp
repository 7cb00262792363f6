// The calls of the library from Python: arguments read off Python objects, the C function called, its status returned.
//
// A call is a few microseconds of launches, and through ctypes as much again: the checks and addresses attribute by attribute in Python, a
// conversion per argument; for a segmented call half a microsecond per tensor on top (128 tensors of 1024 to 8192 values, compress and
// decompress: 140 us, of which 23 were the kernels').  Here it is some ten nanoseconds per argument and tensor.  us of the host per call, arrays read here and the rest in
// Python / all here: 128 small tensors compressed 9.7 / 5.9, decompressed 8.0 / 5.6, one tensor compressed 13.5 / 10.1, one message decompressed 5.3 / 4.2.  Compress and
// decompress of the 128, 15 to 18 / 11.8; of twelve bf16 tensors and a message each 75 / 63.
//
// Each function returns None for anything but the plain case (a tensor subclass, an exotic number, a buffer that is too small, a tensor that
// the library would refuse); the caller then goes through it in Python, which accepts what can be
// accepted and raises the error that fits.
#include <torch/csrc/autograd/python_variable.h>

#include <Python.h>

#include <stdint.h>

#include <vector>

#include "act8_layout.h"
#include "adatopk.h"

namespace {

struct Fast {  // borrowed items of a list or tuple
    PyObject *seq;
    Py_ssize_t n;
    bool ok;
    explicit Fast(PyObject *s) : seq(s), n(0), ok(PyList_CheckExact(s) || PyTuple_CheckExact(s)) {
        if (ok) n = PySequence_Fast_GET_SIZE(s);
    }
    PyObject *at(Py_ssize_t i) const { return PySequence_Fast_GET_ITEM(seq, i); }
};

// tensors(seq) -> (addresses, lengths, first tensor's dtype) for contiguous device tensors of one dtype: bytes objects
// that hold one pointer / one int64 per tensor.
PyObject *tensors(PyObject *, PyObject *arg) {
    const Fast f(arg);
    if (!f.ok || f.n == 0) Py_RETURN_NONE;
    PyObject *addr = PyBytes_FromStringAndSize(nullptr, f.n * static_cast<Py_ssize_t>(sizeof(void *)));
    PyObject *len = PyBytes_FromStringAndSize(nullptr, f.n * static_cast<Py_ssize_t>(sizeof(int64_t)));
    PyObject *result = nullptr;
    bool plain = addr != nullptr && len != nullptr;
    if (!plain) PyErr_Clear();
    try {
        void **a = plain ? reinterpret_cast<void **>(PyBytes_AS_STRING(addr)) : nullptr;
        int64_t *l = plain ? reinterpret_cast<int64_t *>(PyBytes_AS_STRING(len)) : nullptr;
        at::ScalarType dtype = at::ScalarType::Undefined;
        for (Py_ssize_t i = 0; plain && i < f.n; ++i) {
            if (!THPVariable_CheckExact(f.at(i))) {
                plain = false;
                break;
            }
            const at::Tensor &t = THPVariable_Unpack(f.at(i));
            if (i == 0) dtype = t.scalar_type();
            plain = t.scalar_type() == dtype && t.is_cuda() && t.is_contiguous();
            if (plain) {
                a[i] = t.mutable_data_ptr();
                l[i] = t.numel();
            }
        }
        if (plain) {
            PyObject *dt = PyObject_GetAttrString(f.at(0), "dtype");
            if (dt != nullptr) result = PyTuple_Pack(3, addr, len, dt);
            Py_XDECREF(dt);
        }
    } catch (...) {  // no address to be had (a wrapper of functorch, a tensor without storage): Python says why
        result = nullptr;
    }
    Py_XDECREF(addr);
    Py_XDECREF(len);
    if (result == nullptr) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    return result;
}

// int64s(seq, count) -> (bytes of `count` int64, their sum), or None unless seq holds exactly so many plain ints.
PyObject *int64s(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
    if (nargs != 2) {
        PyErr_SetString(PyExc_TypeError, "int64s(seq, count)");
        return nullptr;
    }
    const Fast f(args[0]);
    const Py_ssize_t count = PyLong_AsSsize_t(args[1]);
    if (count < 0 && PyErr_Occurred()) return nullptr;
    if (!f.ok || f.n != count) Py_RETURN_NONE;
    PyObject *out = PyBytes_FromStringAndSize(nullptr, f.n * static_cast<Py_ssize_t>(sizeof(int64_t)));
    if (out == nullptr) return nullptr;
    int64_t *p = reinterpret_cast<int64_t *>(PyBytes_AS_STRING(out));
    int64_t sum = 0;
    bool plain = true;
    for (Py_ssize_t i = 0; plain && i < f.n; ++i) {
        int overflow = 0;
        plain = PyLong_CheckExact(f.at(i));
        if (!plain) break;
        p[i] = PyLong_AsLongLongAndOverflow(f.at(i), &overflow);
        plain = overflow == 0 && !__builtin_add_overflow(sum, p[i], &sum);
    }
    PyObject *result = plain ? Py_BuildValue("(OL)", out, static_cast<long long>(sum)) : nullptr;
    Py_DECREF(out);
    if (plain) return result;
    Py_RETURN_NONE;
}

// ---- the calls
PyObject *g_current_device = nullptr, *g_raw_stream = nullptr;  // torch's functions, set once by streams()

// streams(current_device, raw_stream): how the stream of a call is found.
PyObject *streams(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
    if (nargs != 2) {
        PyErr_SetString(PyExc_TypeError, "streams(current_device, raw_stream)");
        return nullptr;
    }
    Py_XSETREF(g_current_device, Py_NewRef(args[0]));
    Py_XSETREF(g_raw_stream, Py_NewRef(args[1]));
    Py_RETURN_NONE;
}

struct Call {
    bool plain = true;    // so far
    bool raised = false;  // Python code that was called has raised an exception

    // Whether an object is true.
    int truth(PyObject *o) {
        const int is = plain ? PyObject_IsTrue(o) : 0;
        raised = raised || is < 0;
        plain = plain && is >= 0;
        return is;
    }
    // A plain tensor in contiguous device memory, or nullptr.
    const at::Tensor *tensor(PyObject *o) {
        if (!plain || !THPVariable_CheckExact(o)) {
            plain = false;
            return nullptr;
        }
        const at::Tensor &t = THPVariable_Unpack(o);
        plain = t.is_cuda() && t.is_contiguous();
        return plain ? &t : nullptr;
    }
    void *address(const at::Tensor *t) { return plain && t != nullptr ? t->mutable_data_ptr() : nullptr; }
    // ... with at least `count` entries of a type
    void *buffer(PyObject *o, at::ScalarType type, int64_t count) {
        const at::Tensor *t = tensor(o);
        if (t != nullptr) plain = t->scalar_type() == type && t->numel() >= count;
        return address(t);
    }
    void *error_norms(PyObject *o, int64_t count) { return o == Py_None ? nullptr : buffer(o, at::ScalarType::Float, count); }
    int64_t number(PyObject *o) {
        int overflow = 0;
        plain = plain && PyLong_CheckExact(o);
        const int64_t v = plain ? PyLong_AsLongLongAndOverflow(o, &overflow) : 0;
        plain = plain && overflow == 0;
        return v;
    }
    adatopk_dtype dtype(at::ScalarType t) {
        plain = plain && (t == at::ScalarType::Float || t == at::ScalarType::BFloat16 || t == at::ScalarType::Half);
        return t == at::ScalarType::Float ? ADATOPK_F32 : (t == at::ScalarType::BFloat16 ? ADATOPK_BF16 : ADATOPK_F16);
    }
    // `count` numbers of a list or tuple, or as many as there are (count < 0)
    bool numbers(PyObject *o, Py_ssize_t count, std::vector<int64_t> &out) {
        const Fast f(o);
        plain = plain && f.ok && (count < 0 || f.n == count);
        if (!plain) return false;
        out.resize(static_cast<size_t>(f.n));
        for (Py_ssize_t i = 0; plain && i < f.n; ++i) out[static_cast<size_t>(i)] = number(f.at(i));
        return plain;
    }
    // contiguous device tensors of one type
    bool tensors(PyObject *o, std::vector<void *> &at, std::vector<int64_t> &n, at::ScalarType &type) {
        const Fast f(o);
        plain = plain && f.ok && f.n != 0;
        if (!plain) return false;
        at.resize(static_cast<size_t>(f.n));
        n.resize(static_cast<size_t>(f.n));
        for (Py_ssize_t i = 0; plain && i < f.n; ++i) {
            const at::Tensor *t = tensor(f.at(i));
            if (t == nullptr) break;
            if (i == 0) type = t->scalar_type();
            plain = t->scalar_type() == type;
            at[static_cast<size_t>(i)] = address(t);
            n[static_cast<size_t>(i)] = t->numel();
        }
        return plain;
    }
    void *stream() {
        if (!plain) return nullptr;
        if (g_raw_stream == nullptr) {
            plain = false;
            return nullptr;
        }
        PyObject *device = PyObject_CallNoArgs(g_current_device);
        PyObject *raw = device != nullptr ? PyObject_CallOneArg(g_raw_stream, device) : nullptr;
        void *handle = raw != nullptr ? PyLong_AsVoidPtr(raw) : nullptr;
        raised = raw == nullptr;
        plain = raw != nullptr && !PyErr_Occurred();
        Py_XDECREF(device);
        Py_XDECREF(raw);
        return handle;
    }
};

// A tensor seen as rows of its last dimension, which is contiguous: its other dimensions are rows at one distance from the next.
// Without elements there is nothing to step over, whatever the strides.
struct Matrix {
    void *data = nullptr;
    int64_t stride = 0, rows = 0, cols = 0;
    at::ScalarType type = at::ScalarType::Undefined;

    Matrix(Call &c, PyObject *o) {
        if (!c.plain || !THPVariable_CheckExact(o)) {
            c.plain = false;
            return;
        }
        const at::Tensor &t = THPVariable_Unpack(o);
        const int64_t dims = t.dim();
        c.plain = t.is_cuda() && t.layout() == at::kStrided && dims >= 1;
        if (!c.plain) return;
        type = t.scalar_type();
        cols = t.size(dims - 1);
        const bool empty = t.numel() == 0;
        c.plain = empty || cols <= 1 || t.stride(dims - 1) == 1;
        rows = 1;
        stride = cols;
        for (int64_t d = dims - 2; d >= 0 && c.plain; --d) {
            const int64_t size = t.size(d), step = t.stride(d);
            if (size != 1 && !empty) {
                if (rows == 1)
                    stride = step;
                else
                    c.plain = step == rows * stride;
            }
            rows *= size;
        }
        data = c.address(&t);
    }
    // Another matrix of the call, of the same type and shape, or nothing.
    Matrix(Call &c, PyObject *o, const Matrix &like) {
        if (o == Py_None) return;
        *this = Matrix(c, o);
        c.plain = c.plain && type == like.type && rows == like.rows && cols == like.cols;
    }
};
float *floats(Call &c, PyObject *o, int64_t count) {  // exactly so many, or nothing
    if (o == Py_None) return nullptr;
    const at::Tensor *t = c.tensor(o);
    if (t != nullptr) c.plain = t->scalar_type() == at::ScalarType::Float && t->numel() == count;
    return static_cast<float *>(c.address(t));
}
void *act8(Call &c, PyObject *o, int64_t rows, int64_t cols) {
    if (o == Py_None) return nullptr;
    if (!adatopk_internal::act8_shape_ok(rows, cols)) c.plain = false;
    return c.buffer(o, at::ScalarType::Byte,
                    c.plain ? static_cast<int64_t>(adatopk_internal::act8_exponents_at(rows, cols)) + rows * (adatopk_internal::act8_pitch(cols) / adatopk_internal::ACT8_GROUP)
                            : 0);
}
struct Weights {
    const void *weight = nullptr, *bias = nullptr;
    adatopk_dtype type = ADATOPK_F32;
    Weights(Call &c, PyObject *w, PyObject *b, at::ScalarType kind, int64_t cols) {
        const at::Tensor *tw = w != Py_None ? c.tensor(w) : nullptr, *tb = b != Py_None ? c.tensor(b) : nullptr;
        const at::ScalarType own = tw != nullptr ? tw->scalar_type() : (tb != nullptr ? tb->scalar_type() : kind);
        c.plain = c.plain && (own == kind || own == at::ScalarType::Float) && (tw == nullptr || tw->numel() == cols) &&
                  (tb == nullptr || (tb->numel() == cols && tb->scalar_type() == own));
        if (!c.plain) return;
        weight = c.address(tw);
        bias = c.address(tb);
        type = c.dtype(own);
    }
};
struct Workspace {
    void *data = nullptr;
    size_t bytes = 0;
    Workspace(Call &c, PyObject *o) {
        if (o == Py_None) return;
        const at::Tensor *t = c.tensor(o);
        data = c.address(t);
        if (c.plain) bytes = t->nbytes();
    }
};

// The body of a call: `f` reads the arguments and returns the status; what it throws (a wrapper of functorch, a tensor without storage)
// and what is not plain is left to Python.  An exception out of Python code, that of a signal among them (an interrupt while the stream is asked for),
// is the call's: nothing has been enqueued.
template <typename F> PyObject *call(Py_ssize_t nargs, Py_ssize_t expected, F &&f) {
    if (nargs != expected) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    try {
        Call c;
        const long status = f(c);
        if (c.raised) return nullptr;
        if (c.plain && !PyErr_Occurred()) return PyLong_FromLong(status);
    } catch (...) {
    }
    PyErr_Clear();
    Py_RETURN_NONE;
}
// Calls the library at address `fn` without holding the interpreter, as ctypes does.
template <typename Fn, typename... Args> long without_gil(Call &c, PyObject *fn, Args... args) {
    const Fn f = c.plain ? reinterpret_cast<Fn>(PyLong_AsVoidPtr(fn)) : nullptr;
    if (f == nullptr) {
        c.plain = false;
        return 0;
    }
    long status;
    Py_BEGIN_ALLOW_THREADS
    status = static_cast<long>(f(args...));
    Py_END_ALLOW_THREADS
    return status;
}

// (fn, dense, k, idx, val, err or None, workspace)
PyObject *compress(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    return call(nargs, 7, [&](Call &c) -> long {
        const at::Tensor *x = c.tensor(a[1]);
        if (x == nullptr) return 0;
        const int64_t k = c.number(a[2]);
        const adatopk_dtype dt = c.dtype(x->scalar_type());
        void *idx = c.buffer(a[3], at::ScalarType::Int, k), *val = c.buffer(a[4], x->scalar_type(), k), *err = c.error_norms(a[5], 1);
        const at::Tensor *ws = c.tensor(a[6]);
        void *stream = c.stream();
        if (!c.plain) return 0;
        return without_gil<decltype(&adatopk_compress)>(c, a[0], c.address(x), x->numel(), dt, k, static_cast<int32_t *>(idx), val,
                                                        static_cast<float *>(err), c.address(ws), static_cast<size_t>(ws->numel()), stream);
    });
}

// (fn, idx, val, k, dense): the three ways to decompress pairs
PyObject *decompress(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    return call(nargs, 5, [&](Call &c) -> long {
        const at::Tensor *y = c.tensor(a[4]);
        if (y == nullptr) return 0;
        const int64_t k = c.number(a[3]);
        const adatopk_dtype dt = c.dtype(y->scalar_type());
        void *idx = c.buffer(a[1], at::ScalarType::Int, k), *val = c.buffer(a[2], y->scalar_type(), k), *stream = c.stream();
        if (!c.plain) return 0;
        return without_gil<decltype(&adatopk_decompress)>(c, a[0], static_cast<const int32_t *>(idx), static_cast<const void *>(val), k, dt, c.address(y),
                                                          y->numel(), stream);
    });
}

// (fn, wire, wire_bytes, index_bytes, dense, accumulate)
PyObject *decompress_wire(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    return call(nargs, 6, [&](Call &c) -> long {
        const at::Tensor *wire = c.tensor(a[1]), *y = c.tensor(a[4]);
        if (wire == nullptr || y == nullptr) return 0;
        const int64_t bytes = c.number(a[2]), ib = c.number(a[3]);
        const adatopk_dtype dt = c.dtype(y->scalar_type());
        c.plain = c.plain && bytes >= 0 && (ib == 4 || ib == 8);
        const int accumulate = c.truth(a[5]);
        void *stream = c.stream();
        if (!c.plain) return 0;
        return without_gil<decltype(&adatopk_decompress_wire)>(c, a[0], static_cast<const void *>(c.address(wire)), static_cast<size_t>(bytes), dt,
                                                               static_cast<int32_t>(ib), y->numel(), accumulate, c.address(y), stream);
    });
}

// (fn, dense, k, index_bytes, ratio, wire_out, workspace)
PyObject *compress_wire(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    return call(nargs, 7, [&](Call &c) -> long {
        const at::Tensor *x = c.tensor(a[1]), *wire = c.tensor(a[5]), *ws = c.tensor(a[6]);
        if (x == nullptr || wire == nullptr || ws == nullptr) return 0;
        const int64_t k = c.number(a[2]), ib = c.number(a[3]);
        const adatopk_dtype dt = c.dtype(x->scalar_type());
        c.plain = c.plain && PyFloat_CheckExact(a[4]) && (ib == 4 || ib == 8);
        void *stream = c.stream();
        if (!c.plain) return 0;
        return without_gil<decltype(&adatopk_compress_wire)>(c, a[0], static_cast<const void *>(c.address(x)), x->numel(), dt, k, static_cast<int32_t>(ib),
                                                             PyFloat_AS_DOUBLE(a[4]), c.address(wire), static_cast<size_t>(wire->nbytes()),
                                                             c.address(ws), static_cast<size_t>(ws->numel()), stream);
    });
}

// (fn, tensors, ks, idx, val, offsets, err or None, workspace)
PyObject *compress_segmented(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    return call(nargs, 8, [&](Call &c) -> long {
        std::vector<void *> xs;
        std::vector<int64_t> ns, ks, off;
        at::ScalarType type = at::ScalarType::Undefined;
        if (!c.tensors(a[1], xs, ns, type)) return 0;
        const Py_ssize_t S = static_cast<Py_ssize_t>(xs.size());
        const adatopk_dtype dt = c.dtype(type);
        if (!c.numbers(a[2], S, ks) || !c.numbers(a[5], S + 1, off)) return 0;
        int64_t total = 0;
        for (const int64_t k : ks) c.plain = c.plain && !__builtin_add_overflow(total, k, &total);
        void *idx = c.buffer(a[3], at::ScalarType::Int, total), *val = c.buffer(a[4], type, total), *err = c.error_norms(a[6], S);
        const at::Tensor *ws = c.tensor(a[7]);
        void *stream = c.stream();
        if (!c.plain) return 0;
        return without_gil<decltype(&adatopk_compress_segmented)>(c, a[0], static_cast<const void *const *>(xs.data()), static_cast<const int64_t *>(ns.data()),
                                                                  static_cast<const int64_t *>(ks.data()), static_cast<int32_t>(S), dt,
                                                                  static_cast<int32_t *>(idx), val, static_cast<const int64_t *>(off.data()),
                                                                  static_cast<float *>(err), c.address(ws), static_cast<size_t>(ws->numel()), stream);
    });
}

// (fn, idx, val, offsets, tensors)
PyObject *decompress_segmented(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    return call(nargs, 5, [&](Call &c) -> long {
        std::vector<void *> ys;
        std::vector<int64_t> ns, off;
        at::ScalarType type = at::ScalarType::Undefined;
        if (!c.tensors(a[4], ys, ns, type)) return 0;
        const Py_ssize_t S = static_cast<Py_ssize_t>(ys.size());
        const adatopk_dtype dt = c.dtype(type);
        if (!c.numbers(a[3], S + 1, off)) return 0;
        void *idx = c.buffer(a[1], at::ScalarType::Int, off.back()), *val = c.buffer(a[2], type, off.back()), *stream = c.stream();
        if (!c.plain) return 0;
        return without_gil<decltype(&adatopk_decompress_segmented)>(c, a[0], static_cast<const int32_t *>(idx), static_cast<const void *>(val),
                                                                    static_cast<const int64_t *>(off.data()), static_cast<int32_t>(S), dt,
                                                                    static_cast<void *const *>(ys.data()), static_cast<const int64_t *>(ns.data()), stream);
    });
}

// (fn, tensors, ks, index_bytes, ratios or None, wire_out, offsets, workspace)
PyObject *compress_wire_segmented(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    return call(nargs, 8, [&](Call &c) -> long {
        std::vector<void *> xs;
        std::vector<int64_t> ns, ks, off;
        std::vector<double> ratios;
        at::ScalarType type = at::ScalarType::Undefined;
        if (!c.tensors(a[1], xs, ns, type)) return 0;
        const Py_ssize_t S = static_cast<Py_ssize_t>(xs.size());
        const adatopk_dtype dt = c.dtype(type);
        const int64_t ib = c.number(a[3]);
        if (!c.numbers(a[2], S, ks) || !c.numbers(a[6], S, off) || (ib != 4 && ib != 8)) return c.plain = false;
        if (a[4] != Py_None) {
            const Fast f(a[4]);
            c.plain = f.ok && f.n == S;
            for (Py_ssize_t i = 0; c.plain && i < S; ++i) {
                c.plain = PyFloat_CheckExact(f.at(i));
                if (c.plain) ratios.push_back(PyFloat_AS_DOUBLE(f.at(i)));
            }
        }
        const at::Tensor *wire = c.tensor(a[5]), *ws = c.tensor(a[7]);
        void *stream = c.stream();
        if (!c.plain) return 0;
        return without_gil<decltype(&adatopk_compress_wire_segmented)>(
            c, a[0], static_cast<const void *const *>(xs.data()), static_cast<const int64_t *>(ns.data()), static_cast<const int64_t *>(ks.data()),
            static_cast<int32_t>(S), dt, static_cast<int32_t>(ib), a[4] != Py_None ? static_cast<const double *>(ratios.data()) : nullptr, c.address(wire),
            static_cast<const int64_t *>(off.data()), static_cast<size_t>(wire->nbytes()), c.address(ws), static_cast<size_t>(ws->numel()), stream);
    });
}

// (fn, x, act8)
PyObject *act8_store(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    return call(nargs, 3, [&](Call &c) -> long {
        const Matrix x(c, a[1]);
        const adatopk_dtype dt = c.dtype(x.type);
        void *q = a[2] != Py_None ? act8(c, a[2], x.rows, x.cols) : nullptr, *stream = c.stream();
        return without_gil<decltype(&adatopk_act8_store)>(c, a[0], static_cast<const void *>(x.data), x.stride, x.rows, x.cols, dt, q, stream);
    });
}

// (fn, act8, y)
PyObject *act8_load(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    return call(nargs, 3, [&](Call &c) -> long {
        const Matrix y(c, a[2]);
        const adatopk_dtype dt = c.dtype(y.type);
        void *q = act8(c, a[1], y.rows, y.cols), *stream = c.stream();
        return without_gil<decltype(&adatopk_act8_load)>(c, a[0], static_cast<const void *>(q), y.rows, y.cols, dt, y.data, y.stride, stream);
    });
}

// (fn, x, y, act8_x or None, act8_y or None, tanh)
PyObject *gelu_forward(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    return call(nargs, 6, [&](Call &c) -> long {
        const Matrix x(c, a[1]), y(c, a[2], x);
        const adatopk_dtype dt = c.dtype(x.type);
        void *qx = act8(c, a[3], x.rows, x.cols), *qy = act8(c, a[4], x.rows, x.cols);
        const int tanh = c.truth(a[5]);
        void *stream = c.stream();
        return without_gil<decltype(&adatopk_gelu_forward)>(c, a[0], static_cast<const void *>(x.data), x.stride, x.rows, x.cols, dt, tanh, y.data, y.stride, qx, qy,
                                                            stream);
    });
}

// (fn, dy, act8, dx, tanh)
PyObject *gelu_backward(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    return call(nargs, 5, [&](Call &c) -> long {
        const Matrix dy(c, a[1]), dx(c, a[3], dy);
        const adatopk_dtype dt = c.dtype(dy.type);
        void *q = act8(c, a[2], dy.rows, dy.cols);
        const int tanh = c.truth(a[4]);
        void *stream = c.stream();
        return without_gil<decltype(&adatopk_gelu_backward)>(c, a[0], static_cast<const void *>(dy.data), dy.stride, static_cast<const void *>(q), dy.rows, dy.cols,
                                                             dt, tanh, dx.data, dx.stride, stream);
    });
}

// (fn, x, weight or None, bias or None, eps, y, mean or None, rstd or None, residual or None, sum or None, act8 or None)
PyObject *layernorm_forward(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    return call(nargs, 11, [&](Call &c) -> long {
        const Matrix x(c, a[1]), y(c, a[5], x), residual(c, a[8], x), sum(c, a[9], x);
        const adatopk_dtype dt = c.dtype(x.type);
        const Weights w(c, a[2], a[3], x.type, x.cols);
        c.plain = c.plain && PyFloat_CheckExact(a[4]);
        float *mean = floats(c, a[6], x.rows), *rstd = floats(c, a[7], x.rows);
        void *q = act8(c, a[10], x.rows, x.cols), *stream = c.stream();
        if (!c.plain) return 0;
        return without_gil<decltype(&adatopk_layernorm_forward)>(
            c, a[0], static_cast<const void *>(x.data), x.stride, static_cast<const void *>(residual.data), residual.stride, w.weight, w.bias, w.type, x.rows, x.cols,
            dt, static_cast<float>(PyFloat_AS_DOUBLE(a[4])), sum.data, sum.stride, y.data, y.stride, mean, rstd, q, stream);
    });
}

// (fn, dy, x or None, act8 or None, mean or None, rstd, weight or None, dx, dweight or None, dbias or None, workspace or None, dsum or None, accumulate)
PyObject *layernorm_backward(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    return call(nargs, 13, [&](Call &c) -> long {
        const Matrix dy(c, a[1]), x(c, a[2], dy), dx(c, a[7], dy), dsum(c, a[11], dy);
        const adatopk_dtype dt = c.dtype(dy.type);
        const Weights w(c, a[6], Py_None, dy.type, dy.cols);
        void *q = act8(c, a[3], dy.rows, dy.cols);
        float *mean = floats(c, a[4], dy.rows), *rstd = floats(c, a[5], dy.rows), *dw = floats(c, a[8], dy.cols), *db = floats(c, a[9], dy.cols);
        const Workspace ws(c, a[10]);
        const int accumulate = c.truth(a[12]);
        void *stream = c.stream();
        return without_gil<decltype(&adatopk_layernorm_backward)>(
            c, a[0], static_cast<const void *>(dy.data), dy.stride, static_cast<const void *>(x.data), x.stride, static_cast<const void *>(q),
            static_cast<const float *>(mean), static_cast<const float *>(rstd), w.weight, w.type, static_cast<const void *>(dsum.data), dsum.stride, dy.rows, dy.cols,
            dt, dx.data, dx.stride, dw, db, accumulate, ws.data, ws.bytes, stream);
    });
}

// (fn, dy, act8, dw, db or None, workspace, weight or None, bias or None, accumulate)
PyObject *weight_grad(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    return call(nargs, 9, [&](Call &c) -> long {
        const Matrix dy(c, a[1]);
        const adatopk_dtype dt = c.dtype(dy.type);
        const at::Tensor *dw = c.tensor(a[3]);
        c.plain = c.plain && dw->dim() == 2 && dw->scalar_type() == at::ScalarType::Float && dw->size(0) == dy.cols;
        if (!c.plain) return 0;
        const int64_t n_in = dw->size(1);
        void *q = a[2] != Py_None ? act8(c, a[2], dy.rows, n_in) : nullptr;
        const Weights w(c, a[6], a[7], dy.type, n_in);
        float *db = floats(c, a[4], dy.cols);
        const Workspace ws(c, a[5]);
        const int accumulate = c.truth(a[8]);
        void *stream = c.stream();
        return without_gil<decltype(&adatopk_weight_grad)>(c, a[0], static_cast<const void *>(dy.data), dy.stride, static_cast<const void *>(q), dy.rows, dy.cols, n_in,
                                                           dt, w.weight, w.bias, w.type, static_cast<float *>(c.address(dw)), db, accumulate, ws.data, ws.bytes,
                                                           stream);
    });
}

template <PyObject *(*F)(PyObject *, PyObject *const *, Py_ssize_t)> constexpr PyMethodDef fast(const char *name, const char *doc) {
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(F)), METH_FASTCALL, doc};
}
PyMethodDef methods[] = {
    {"tensors", tensors, METH_O, "(addresses, lengths, dtype) of contiguous device tensors of one dtype, or None"},
    fast<int64s>("int64s", "(int64 array, sum) of a sequence of `count` ints, or None"),
    fast<streams>("streams", "how the stream of a call is found: torch's current_device and raw stream functions"),
    fast<compress>("compress", "status of the call at an address, or None"),
    fast<decompress>("decompress", "status of the call at an address, or None"),
    fast<compress_wire>("compress_wire", "status of the call at an address, or None"),
    fast<decompress_wire>("decompress_wire", "status of the call at an address, or None"),
    fast<compress_segmented>("compress_segmented", "status of the call at an address, or None"),
    fast<decompress_segmented>("decompress_segmented", "status of the call at an address, or None"),
    fast<compress_wire_segmented>("compress_wire_segmented", "status of the call at an address, or None"),
    fast<act8_store>("act8_store", "status of the call at an address, or None"),
    fast<act8_load>("act8_load", "status of the call at an address, or None"),
    fast<gelu_forward>("gelu_forward", "status of the call at an address, or None"),
    fast<gelu_backward>("gelu_backward", "status of the call at an address, or None"),
    fast<layernorm_forward>("layernorm_forward", "status of the call at an address, or None"),
    fast<layernorm_backward>("layernorm_backward", "status of the call at an address, or None"),
    fast<weight_grad>("weight_grad", "status of the call at an address, or None"),
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "The calls of the library, their arguments read in C.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&module); }
