// binding.cpp -- the Python bindings' checks of tensors, and the library's calls, for the
// operators of int8.py, rope.py and norm.py.  A call of few tokens is bound by the host:
// the same checks made in Python with ctypes behind them took 3 to 6 us of the 5.4 to
// 8.5 that such calls took, here they take 0.3.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <string>

#include "echo_int8.h"
#include "echo_norm.h"
#include "echo_rope.h"

namespace {

PyObject *g_refuse, *g_check, *g_device, *g_stream;   // of fp8.py, echo.py and torch
decltype(&echo_int8_quantize) f_quantize;
decltype(&echo_int8_gemm) f_gemm;
decltype(&echo_rope_rotate) f_rotate;
decltype(&echo_norm_join) f_join;

// Thrown with a Python exception set
struct Raised {};

[[noreturn]] void refuse(const char *where, const std::string &what) {
    Py_XDECREF(PyObject_CallFunction(g_refuse, "ss", where, what.c_str()));
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, what.c_str());
    throw Raised();
}

void check(int rc, const char *where) {
    if (rc == 0) return;
    Py_XDECREF(PyObject_CallFunction(g_check, "is", rc, where));
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, where);
    throw Raised();
}

const at::Tensor &tensor(const char *where, const char *name, PyObject *o) {
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s: %s is no tensor", where, name);
        throw Raised();
    }
    return THPVariable_Unpack(o);
}

std::string text(at::IntArrayRef v) {
    std::string s = "(";
    for (size_t i = 0; i < v.size(); ++i) s += (i ? ", " : "") + std::to_string(v[i]);
    return s + (v.size() == 1 ? ",)" : ")");
}

// counts that the library's 32-bit arguments would cut off
void sizes(const char *where, std::initializer_list<int64_t> n) {
    for (int64_t v : n)
        if (v >> 31) refuse(where, std::to_string(v) + " is not below 2^31");
}

void axes(const char *where, const char *name, const at::Tensor &t, int64_t n) {
    if (t.dim() != n) refuse(where, std::string(name) + " has " + std::to_string(t.dim()) + " axes");
}

enum Types { kF32 = 1, kBf16 = 2, kI8 = 4, kI32 = 8, kF64 = 16, kReal = kF32 | kBf16 };

int type_of(const at::Tensor &t) {
    switch (t.scalar_type()) {
        case at::kFloat: return kF32;
        case at::kBFloat16: return kBf16;
        case at::kChar: return kI8;
        case at::kInt: return kI32;
        case at::kDouble: return kF64;
        default: return 0;
    }
}

void placed(const char *where, const char *name, const at::Tensor &t, int dev) {
    if (t.get_device() != dev)
        refuse(where, std::string(name) + " is on " + t.device().str() +
                          (t.is_cuda() ? ", the current device is cuda:" + std::to_string(dev) : ", not on a GPU"));
}

void typed(const char *where, const char *name, const at::Tensor &t, int types) {
    if (!(type_of(t) & types)) refuse(where, std::string(name) + " has dtype " + c10::toString(t.scalar_type()));
}

// the type and the place that every tensor is checked for
void like(const char *where, const char *name, const at::Tensor &t, int types, int dev) {
    typed(where, name, t, types);
    placed(where, name, t, dev);
}

void shaped(const char *where, const char *name, const at::Tensor &t, at::IntArrayRef shape) {
    if (t.sizes() != shape) refuse(where, std::string(name) + " has shape " + text(t.sizes()) + ", not " + text(shape));
}

// The address of a contiguous tensor of this shape
void *address(const char *where, const char *name, const at::Tensor &t, at::IntArrayRef shape, int types, int dev) {
    shaped(where, name, t, shape);
    like(where, name, t, types, dev);
    if (!t.is_contiguous()) refuse(where, std::string(name) + " is not contiguous");
    return t.data_ptr();
}

// The address of a matrix whose rows are contiguous and any distance apart
void *rows(const char *where, const char *name, const at::Tensor &t, at::IntArrayRef shape, int types, int dev,
           int64_t *stride) {
    shaped(where, name, t, shape);
    like(where, name, t, types, dev);
    const int64_t n = shape[0], m = shape[1];
    *stride = m > 1 ? m : 1;
    if (!t.is_contiguous()) {
        if ((m > 1 && t.stride(1) != 1) || (n > 1 && t.stride(0) < m))
            refuse(where, std::string("the rows of ") + name + " are not contiguous");
        if (n > 1) *stride = t.stride(0);
    }
    return t.data_ptr();
}

int dtype_of(const at::Tensor &t) {
    const int k = type_of(t);
    return k == kF32 ? (int)ECHO_F32 : k == kBf16 ? (int)ECHO_BF16 : (int)ECHO_I8;
}

int current_device() {
    if (g_device == Py_None) return -2;   // no GPU: a device that no tensor is on
    PyObject *d = PyObject_CallNoArgs(g_device);
    if (!d) throw Raised();
    const long v = PyLong_AsLong(d);
    Py_DECREF(d);
    return (int)v;
}

void *stream_of(PyObject *stream, int dev) {
    PyObject *s;
    if (stream == Py_None) {
        PyObject *d = PyLong_FromLong(dev);
        s = PyObject_CallOneArg(g_stream, d);
        Py_DECREF(d);
    } else {
        s = PyObject_GetAttrString(stream, "cuda_stream");
    }
    if (!s) throw Raised();
    void *p = PyLong_AsVoidPtr(s);
    Py_DECREF(s);
    if (!p && PyErr_Occurred()) throw Raised();
    return p;
}

template <typename F>
PyObject *guarded(const char *where, Py_ssize_t n, Py_ssize_t want, F call) {
    if (n != want) {
        PyErr_Format(PyExc_TypeError, "%s takes %zd arguments", where, want);
        return nullptr;
    }
    try {
        call();
    } catch (const Raised &) {
        return nullptr;
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, where);
        return nullptr;
    }
    Py_RETURN_NONE;
}

template <typename F>
int unlocked(F call) {
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call();
    Py_END_ALLOW_THREADS
    return rc;
}

// x, codes, scales, stream
PyObject *quantize(PyObject *, PyObject *const *a, Py_ssize_t n) {
    static const char *where = "echo_int8_quantize";
    return guarded(where, n, 4, [&] {
        const at::Tensor &x = tensor(where, "x", a[0]), &codes = tensor(where, "codes", a[1]);
        const at::Tensor &scales = tensor(where, "scales", a[2]);
        const int dev = current_device();
        axes(where, "x", x, 2);
        const int64_t R = x.size(0), C = x.size(1);
        sizes(where, {R, C});
        int64_t stride;
        const void *xp = rows(where, "x", x, x.sizes(), kReal, dev, &stride);
        void *cp = address(where, "codes", codes, {R, C}, kI8, dev);
        void *sp = address(where, "scales", scales, {R}, kF32, dev);
        void *st = stream_of(a[3], dev);
        check(unlocked([&] { return f_quantize(xp, dtype_of(x), stride, R, C, (int8_t *)cp, (float *)sp, st); }), where);
    });
}

// x, x_scale, w, w_scale, out, bias, residual, workspace, stream
PyObject *gemm(PyObject *, PyObject *const *a, Py_ssize_t n) {
    static const char *where = "echo_int8_gemm";
    return guarded(where, n, 9, [&] {
        const at::Tensor &x = tensor(where, "x", a[0]), &xs = tensor(where, "x_scale", a[1]);
        const at::Tensor &w = tensor(where, "w", a[2]), &ws = tensor(where, "w_scale", a[3]);
        const at::Tensor &y = tensor(where, "out", a[4]);
        const int dev = current_device();
        axes(where, "x", x, 2);
        axes(where, "w", w, 2);
        const int64_t T = x.size(0), K = x.size(1), N = w.size(0);
        sizes(where, {T, K, N});
        const void *xp = address(where, "x", x, {T, K}, kI8, dev), *xsp = address(where, "x_scale", xs, {T}, kF32, dev);
        const void *wp = address(where, "w", w, {N, K}, kI8, dev), *wsp = address(where, "w_scale", ws, {N}, kF32, dev);
        int64_t stride, rs;
        void *yp = rows(where, "out", y, {T, N}, kReal, dev, &stride), *sp = nullptr;
        const void *bp = nullptr, *rp = nullptr;
        if (a[5] != Py_None) bp = address(where, "bias", tensor(where, "bias", a[5]), {N}, kF32, dev);
        if (a[6] != Py_None) {
            const at::Tensor &r = tensor(where, "residual", a[6]);
            rp = rows(where, "residual", r, {T, N}, kReal, dev, &rs);
            if (r.scalar_type() != y.scalar_type() || rs != stride)
                refuse(where, "residual has not the type and strides of out");
        }
        size_t bytes = 0;
        if (a[7] != Py_None) {
            const at::Tensor &t = tensor(where, "workspace", a[7]);
            placed(where, "workspace", t, dev);
            if (!t.is_contiguous()) refuse(where, "workspace is not contiguous");
            sp = t.data_ptr();
            bytes = t.nbytes();
        }
        void *st = stream_of(a[8], dev);
        check(unlocked([&] {
                  return f_gemm((const int8_t *)xp, (const float *)xsp, (const int8_t *)wp, (const float *)wsp, T, N, K,
                                (const float *)bp, rp, yp, dtype_of(y), stride, sp, bytes, st);
              }),
              where);
    });
}

// heads [T][heads][D]
void heads(const char *where, const char *name, const at::Tensor &t, int64_t T, int64_t D, int types, int dev, void **p,
           int32_t *n, int64_t *token, int64_t *head) {
    if (t.dim() != 3 || t.size(0) != T || t.size(2) != D)
        refuse(where, std::string(name) + " has shape " + text(t.sizes()) + ", not (" + std::to_string(T) + ", heads, " +
                          std::to_string(D) + ")");
    like(where, name, t, types, dev);
    if (t.stride(2) != 1 && D > 1) refuse(where, std::string("the columns of ") + name + " are not adjacent");
    const int64_t H = t.size(1);
    sizes(where, {H});
    *p = t.data_ptr();
    *n = (int32_t)H;
    // an axis of one has any stride
    *token = T > 1 ? t.stride(0) : H * D;
    *head = H > 1 ? t.stride(1) : D;
}

// address of the rope, its frequencies, its magnitude, positions, q, k, q_out, k_out,
// inverse, stream
PyObject *rotate(PyObject *, PyObject *const *a, Py_ssize_t n) {
    static const char *where = "echo_rope_rotate";
    return guarded(where, n, 10, [&] {
        const auto *rope = (const echo_rope_t *)PyLong_AsVoidPtr(a[0]);
        const at::Tensor &f = tensor(where, "rope.frequencies", a[1]), &pos = tensor(where, "positions", a[3]);
        const at::Tensor &q = tensor(where, "q", a[4]);
        const double magnitude = PyFloat_AsDouble(a[2]);
        const int inverse = PyObject_IsTrue(a[8]);
        if (PyErr_Occurred()) throw Raised();
        const int dev = current_device();
        axes(where, "q", q, 3);
        const int64_t T = q.size(0), D = rope->head_dim;
        sizes(where, {T});
        // what the library reads R / 2 numbers of 64 bits of (its place: below)
        shaped(where, "rope.frequencies", f, {rope->rotary_dim / 2});
        typed(where, "rope.frequencies", f, kF64);
        if (!f.is_contiguous()) refuse(where, "rope.frequencies is not contiguous");
        const int types = type_of(q) & kReal;
        if (a[5] == Py_None && a[7] != Py_None) refuse(where, "k_out without k");
        echo_rope_heads_t t[2];
        int count = 0;
        static const char *names[2][2] = {{"q", "q_out"}, {"k", "k_out"}};
        for (int i = 0; i < 2; ++i) {
            if (a[4 + i] == Py_None) continue;
            echo_rope_heads_t &h = t[count++];
            void *p;
            heads(where, names[i][0], tensor(where, names[i][0], a[4 + i]), T, D, types, dev, &p, &h.heads, &h.in_token,
                  &h.in_head);
            h.in = h.out = p;
            h.out_token = h.in_token;
            h.out_head = h.in_head;
            if (a[6 + i] == Py_None) continue;
            int32_t others;
            heads(where, names[i][1], tensor(where, names[i][1], a[6 + i]), T, D, types, dev, &h.out, &others, &h.out_token,
                  &h.out_head);
            if (others != h.heads)
                refuse(where, std::string(names[i][1]) + " has " + std::to_string(others) + " heads, " + names[i][0] + " " +
                                  std::to_string(h.heads));
        }
        const void *pp = address(where, "positions", pos, {T}, kI32, dev);
        placed(where, "rope.frequencies", f, dev);
        const void *fp = f.data_ptr();
        void *st = stream_of(a[9], dev);
        check(unlocked([&] {
                  return f_rotate(rope, (const double *)fp, magnitude, (const int32_t *)pp, T, dtype_of(q), t, count, inverse, st);
              }),
              where);
    });
}

// address of the norm, its weights' device or None, block, residual, gate, sum, y, y_scale,
// stream
PyObject *join(PyObject *, PyObject *const *a, Py_ssize_t n) {
    static const char *where = "echo_norm_join";
    return guarded(where, n, 9, [&] {
        const auto *norm = (const echo_norm_t *)PyLong_AsVoidPtr(a[0]);
        const int dev = current_device();
        if (a[1] != Py_None && PyLong_AsLong(a[1]) != dev)
            refuse(where, "the weights are on cuda:" + std::to_string(PyLong_AsLong(a[1])) + ", the current device is cuda:" +
                              std::to_string(dev));
        if (a[2] == Py_None && a[3] == Py_None) refuse(where, "neither block nor residual");
        const at::Tensor &lead = tensor(where, "block or residual", a[2] != Py_None ? a[2] : a[3]);
        axes(where, "block or residual", lead, 2);
        const int64_t T = lead.size(0), H = norm->hidden;
        sizes(where, {T});
        static const char *names[5] = {"block", "residual", "gate", "sum", "y"};
        echo_rows_t r[5] = {};
        for (int i = 0; i < 5; ++i) {
            if (a[2 + i] == Py_None) continue;
            const at::Tensor &t = tensor(where, names[i], a[2 + i]);
            if (i == 2 && t.dim() == 1) r[i].data = address(where, names[i], t, {H}, kReal, dev);   // stride 0
            else r[i].data = rows(where, names[i], t, {T, H}, i == 4 ? kReal | kI8 : kReal, dev, &r[i].stride);
            r[i].dtype = dtype_of(t);
        }
        void *sp = nullptr;
        if (a[7] != Py_None) sp = address(where, "y_scale", tensor(where, "y_scale", a[7]), {T}, kF32, dev);
        void *st = stream_of(a[8], dev);
        check(unlocked([&] { return f_join(norm, T, &r[0], &r[2], &r[1], &r[3], &r[4], (float *)sp, st); }), where);
    });
}

// refuse, check, the current device's and its stream's callables (None: no GPU), and the
// addresses of the library's entry points
PyObject *setup(PyObject *, PyObject *args) {
    PyObject *p[4], *f[4];
    if (!PyArg_ParseTuple(args, "OOOOOOOO", &p[0], &p[1], &p[2], &p[3], &f[0], &f[1], &f[2], &f[3])) return nullptr;
    for (PyObject *o : p) Py_INCREF(o);
    g_refuse = p[0], g_check = p[1], g_device = p[2], g_stream = p[3];
    f_quantize = (decltype(f_quantize))PyLong_AsVoidPtr(f[0]);
    f_gemm = (decltype(f_gemm))PyLong_AsVoidPtr(f[1]);
    f_rotate = (decltype(f_rotate))PyLong_AsVoidPtr(f[2]);
    f_join = (decltype(f_join))PyLong_AsVoidPtr(f[3]);
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"setup", setup, METH_VARARGS, nullptr},
                         {"quantize", (PyCFunction)(void (*)())quantize, METH_FASTCALL, nullptr},
                         {"gemm", (PyCFunction)(void (*)())gemm, METH_FASTCALL, nullptr},
                         {"rotate", (PyCFunction)(void (*)())rotate, METH_FASTCALL, nullptr},
                         {"join", (PyCFunction)(void (*)())join, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
