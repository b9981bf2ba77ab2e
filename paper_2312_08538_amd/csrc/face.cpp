// Python's way into the operators of a training step (conef_dropout_*, conef_norm_*, conef_mx_*): reads shapes, types, pitches and
// addresses off torch tensors, refuses those that do not fit or are on another device than the stream, and calls the library by the
// addresses that it was given.  A small operator's time is that of its call: a dropout of one row takes 3.1 us, of which 2.9 are the launch
// (marshalled in Python and by ctypes 5.0), a layer norm of one row 4.0 with what its caller does around it (7.6).
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/core/Tensor.h>

#include <exception>
#include <string>

#include "../../include/conef.h"

namespace {

struct Library {
    decltype(&conef_dropout_forward) dropout_forward;
    decltype(&conef_dropout_backward) dropout_backward;
    decltype(&conef_norm_forward) norm_forward;
    decltype(&conef_norm_workspace) norm_workspace;
    decltype(&conef_norm_backward) norm_backward;
    decltype(&conef_mx_quantise) mx_quantise;
    decltype(&conef_mx_dequantise) mx_dequantise;
    decltype(&conef_mx_product_workspace) mx_product_workspace;
    decltype(&conef_mx_product) mx_product;
    int (*stream_device)(void *stream, int *device);            // the runtime's hipStreamGetDevice
} L;

PyObject *drop_type, *error_type;       // conef_drop and ConefError of the binding

// thrown with Python's error set
struct PythonError {};

[[noreturn]] void refuse(const std::string &why)
{
    if (PyObject *e = PyObject_CallFunction(error_type, "is", CONEF_EINVAL, why.c_str())) {
        PyErr_SetObject(error_type, e);
        Py_DECREF(e);
    }
    throw PythonError();
}

PyObject *done(int code, const char *where)
{
    if (code == CONEF_OK) Py_RETURN_NONE;
    if (PyObject *e = PyObject_CallFunction(error_type, "is", code, where)) {
        PyErr_SetObject(error_type, e);
        Py_DECREF(e);
    }
    return nullptr;
}

int64_t integer(PyObject *o)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw PythonError();
    return v;
}

// seeds, steps: modulo 2^64
uint64_t bits(PyObject *o)
{
    const unsigned long long v = PyLong_AsUnsignedLongLongMask(o);
    if (v == (unsigned long long)-1 && PyErr_Occurred()) throw PythonError();
    return v;
}

float real(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw PythonError();
    return (float)v;
}

// a stream (none: the current device's default one) and the device that it belongs to, which all of a call's tensors have to be on
struct Stream {
    void *handle;
    int device = -1;

    explicit Stream(PyObject *o) : handle(o == Py_None ? nullptr : reinterpret_cast<void *>(bits(o)))
    {
        if (L.stream_device(handle, &device) != 0) device = -1;
    }
};

// a description's copy, or none
struct Drop {
    conef_drop value;
    const conef_drop *there = nullptr;

    explicit Drop(PyObject *o)
    {
        if (o == Py_None) return;
        if (!PyObject_TypeCheck(o, reinterpret_cast<PyTypeObject *>(drop_type))) refuse("a conef_drop is wanted");
        Py_buffer view;
        if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE)) throw PythonError();
        const bool fits = view.len == (Py_ssize_t)sizeof value;
        if (fits) value = *static_cast<const conef_drop *>(view.buf);
        PyBuffer_Release(&view);
        if (!fits) refuse("a conef_drop is wanted");
        there = &value;
    }
};

const at::Tensor &tensor(PyObject *o)
{
    if (!THPVariable_Check(o)) refuse(std::string("a tensor is wanted, not ") + Py_TYPE(o)->tp_name);
    return THPVariable_Unpack(o);
}

std::string about(const at::Tensor &t)
{
    std::string s = "(";
    for (int64_t i = 0; i < t.dim(); ++i) s += std::to_string(t.size(i)) + ", ";
    s += std::string(") ") + t.toString() + " strides (";
    for (int64_t i = 0; i < t.dim(); ++i) s += std::to_string(t.stride(i)) + ", ";
    return s + ")";
}

int kind_of(const at::Tensor &t)
{
    return t.scalar_type() == at::kFloat ? CONEF_F32 : t.scalar_type() == at::kBFloat16 ? CONEF_BF16 : -1;
}

bool on_device(const at::Tensor &t) { return t.is_cuda() && t.layout() == at::kStrided; }

void check_place(const Stream &st, const at::Tensor &t)
{
    if (t.device().index() == st.device) return;
    if (st.device < 0) refuse("the stream is none of this process's");
    refuse("tensors on cuda:" + std::to_string(st.device) + ", the stream's device, are wanted, not on " + t.device().str());
}

struct Matrix {
    void *data = nullptr;
    int64_t pitch = 0, rows = 0, cols = 0;
    int kind = 0;

    void take(const Stream &st, const at::Tensor &t)
    {
        check_place(st, t);
        rows = t.size(0);
        cols = t.size(1);
        pitch = rows > 1 ? t.stride(0) : cols ? cols : 1;
        data = t.data_ptr();
    }
    // two dimensions, rows contiguous
    static bool fits(const at::Tensor &t)
    {
        return on_device(t) && t.dim() == 2 && kind_of(t) >= 0 && (t.stride(1) == 1 || t.size(1) <= 1);
    }

    Matrix(const Stream &st, PyObject *o)
    {
        const at::Tensor &t = tensor(o);
        if (!fits(t)) refuse("a matrix of fp32 or bf16 on the device with contiguous rows is wanted, not " + about(t));
        kind = kind_of(t);
        take(st, t);
    }
    // another of the same shape and type, or none
    Matrix(const Stream &st, PyObject *o, const Matrix &of) : kind(of.kind)
    {
        if (o == Py_None) return;
        const at::Tensor &t = tensor(o);
        if (!fits(t) || t.size(0) != of.rows || t.size(1) != of.cols || kind_of(t) != of.kind)
            refuse("a matrix (" + std::to_string(of.rows) + ", " + std::to_string(of.cols) + (of.kind == CONEF_F32 ? ") of fp32" : ") of bf16") +
                   " on the device with contiguous rows is wanted, not " + about(t));
        take(st, t);
    }
};

// n contiguous floats, or none
float *vector(const Stream &st, PyObject *o, int64_t n)
{
    if (o == Py_None) return nullptr;
    const at::Tensor &t = tensor(o);
    if (!on_device(t) || t.dim() != 1 || t.size(0) != n || t.scalar_type() != at::kFloat || !t.is_contiguous())
        refuse(std::to_string(n) + " contiguous floats on the device are wanted, not " + about(t));
    check_place(st, t);
    return static_cast<float *>(t.data_ptr());
}

// a buffer of at least so many bytes, or none
void *room(const Stream &st, PyObject *o, size_t bytes)
{
    if (o == Py_None) return nullptr;
    const at::Tensor &t = tensor(o);
    if (!on_device(t) || !t.is_contiguous() || t.nbytes() < bytes)
        refuse("a contiguous buffer of " + std::to_string(bytes) + " bytes on the device is wanted, not " + about(t));
    check_place(st, t);
    return t.data_ptr();
}

// codes and scales of a packed operand, or none
struct Packed {
    uint8_t *codes = nullptr, *scales = nullptr;

    Packed(const Stream &st, PyObject *o, int64_t rows, int64_t cols)
    {
        if (o == Py_None) return;
        PyObject *both[2] = {};
        if (PyTuple_Check(o) && PyTuple_GET_SIZE(o) == 2) {
            both[0] = PyTuple_GET_ITEM(o, 0);
            both[1] = PyTuple_GET_ITEM(o, 1);
        } else if (PyList_Check(o) && PyList_GET_SIZE(o) == 2) {
            both[0] = PyList_GET_ITEM(o, 0);
            both[1] = PyList_GET_ITEM(o, 1);
        } else {
            refuse("a packed operand is a pair of codes and scales");
        }
        // (in 128 bits: the library refuses sides that 64 bits could not count)
        const unsigned __int128 elements = (unsigned __int128)(((uint64_t)rows + 63) / 64) * (((uint64_t)cols + 127) / 128) * 8192;
        if (rows < 0 || cols < 0 || elements >> 62) refuse("sides out of range");
        codes = static_cast<uint8_t *>(room(st, both[0], (size_t)(elements / 2)));
        scales = static_cast<uint8_t *>(room(st, both[1], (size_t)(elements / 32)));
    }
};

// `f` of n arguments, what it throws as Python's error
template <typename F>
PyObject *call(const char *name, Py_ssize_t given, Py_ssize_t n, F &&f)
{
    if (given != n) {
        PyErr_Format(PyExc_TypeError, "%s takes %zd arguments, not %zd", name, n, given);
        return nullptr;
    }
    try {
        return done(f(), name);
    } catch (const PythonError &) {
    } catch (const std::exception &e) {
        PyErr_Format(PyExc_RuntimeError, "%s: %s", name, e.what());
    }
    return nullptr;
}

// Python runs on while the library launches
template <typename F>
int unlocked(F &&f)
{
    PyThreadState *s = PyEval_SaveThread();
    const int code = f();
    PyEval_RestoreThread(s);
    return code;
}

PyObject *dropout_forward(PyObject *, PyObject *const *p, Py_ssize_t n)
{
    return call("conef_dropout_forward", n, 5, [&] {
        const Stream st(p[4]);
        const Drop d(p[0]);
        const Matrix x(st, p[1]), r(st, p[2], x), y(st, p[3], x);
        return unlocked([&] {
            return L.dropout_forward(d.there, x.rows, x.cols, x.kind, x.data, x.pitch, r.data, r.pitch, y.data, y.pitch, st.handle);
        });
    });
}

PyObject *dropout_backward(PyObject *, PyObject *const *p, Py_ssize_t n)
{
    return call("conef_dropout_backward", n, 4, [&] {
        const Stream st(p[3]);
        const Drop d(p[0]);
        const Matrix dy(st, p[1]), dx(st, p[2], dy);
        return unlocked([&] { return L.dropout_backward(d.there, dy.rows, dy.cols, dy.kind, dy.data, dy.pitch, dx.data, dx.pitch, st.handle); });
    });
}

PyObject *norm_forward(PyObject *, PyObject *const *p, Py_ssize_t n)
{
    return call("conef_norm_forward", n, 11, [&] {
        const Stream st(p[10]);
        const Drop d(p[0]);
        const float eps = real(p[1]);
        const Matrix x(st, p[2]), r(st, p[3], x), z(st, p[6], x), y(st, p[7], x);
        const float *gamma = vector(st, p[4], x.cols), *beta = vector(st, p[5], x.cols);
        float *mean = vector(st, p[8], x.rows), *rstd = vector(st, p[9], x.rows);
        return unlocked([&] {
            return L.norm_forward(d.there, eps, x.rows, x.cols, x.kind, x.data, x.pitch, r.data, r.pitch, gamma, beta, z.data, z.pitch, y.data,
                                  y.pitch, mean, rstd, st.handle);
        });
    });
}

PyObject *norm_backward(PyObject *, PyObject *const *p, Py_ssize_t n)
{
    return call("conef_norm_backward", n, 13, [&] {
        const Stream st(p[12]);
        const Drop d(p[0]);
        const Matrix dy(st, p[1]), z(st, p[2], dy), in(st, p[6], dy), dz(st, p[7], dy), dx(st, p[8], dy);
        const float *gamma = vector(st, p[3], dy.cols), *mean = vector(st, p[4], dy.rows), *rstd = vector(st, p[5], dy.rows);
        float *dgamma = vector(st, p[9], dy.cols), *dbeta = vector(st, p[10], dy.cols);
        size_t bytes = 0;
        if (p[11] != Py_None && L.norm_workspace(dy.rows, dy.cols, &bytes) != CONEF_OK) return (int)CONEF_EINVAL;
        void *ws = room(st, p[11], bytes);
        return unlocked([&] {
            return L.norm_backward(d.there, dy.rows, dy.cols, dy.kind, dy.data, dy.pitch, z.data, z.pitch, gamma, mean, rstd, in.data, in.pitch,
                                   dz.data, dz.pitch, dx.data, dx.pitch, dgamma, dbeta, ws, st.handle);
        });
    });
}

PyObject *mx_quantise(PyObject *, PyObject *const *p, Py_ssize_t n)
{
    return call("conef_mx_quantise", n, 8, [&] {
        const Stream st(p[7]);
        const Matrix x(st, p[0]);
        const int64_t rounding = integer(p[1]);
        if (rounding != CONEF_MX_NEAREST && rounding != CONEF_MX_STOCHASTIC) refuse("CONEF_MX_NEAREST or CONEF_MX_STOCHASTIC is wanted");
        const uint64_t seed = bits(p[2]), site = bits(p[3]), step = bits(p[4]);
        if (site >> 32) refuse("a site below 2^27 is wanted");
        const Packed q(st, p[5], x.rows, x.cols), t(st, p[6], x.cols, x.rows);
        return unlocked([&] {
            return L.mx_quantise(x.data, x.pitch, x.rows, x.cols, x.kind, (int)rounding, seed, (uint32_t)site, step, q.codes, q.scales, t.codes,
                                 t.scales, st.handle);
        });
    });
}

PyObject *mx_dequantise(PyObject *, PyObject *const *p, Py_ssize_t n)
{
    return call("conef_mx_dequantise", n, 3, [&] {
        const Stream st(p[2]);
        const Matrix out(st, p[1]);
        const Packed q(st, p[0], out.rows, out.cols);
        return unlocked([&] { return L.mx_dequantise(q.codes, q.scales, out.rows, out.cols, out.data, out.pitch, out.kind, st.handle); });
    });
}

PyObject *mx_product(PyObject *, PyObject *const *p, Py_ssize_t n)
{
    return call("conef_mx_product", n, 8, [&] {
        const Stream st(p[7]);
        const Matrix c(st, p[5]);
        const int64_t k = integer(p[2]);
        const Packed a(st, p[0], c.rows, k), b(st, p[1], c.cols, k);
        const float alpha = real(p[3]), beta = real(p[4]);
        size_t bytes = 0;
        if (p[6] != Py_None && L.mx_product_workspace(c.rows, c.cols, k, &bytes) != CONEF_OK) return (int)CONEF_EINVAL;
        void *ws = room(st, p[6], bytes);
        return unlocked([&] {
            return L.mx_product(a.codes, a.scales, b.codes, b.scales, c.rows, c.cols, k, alpha, beta, c.data, c.pitch, c.kind, ws, st.handle);
        });
    });
}

// connect(conef_drop, ConefError, addresses of the library's calls in Library's order)
PyObject *connect(PyObject *, PyObject *args)
{
    PyObject *drop, *error;
    unsigned long long at[10];
    if (!PyArg_ParseTuple(args, "OO(KKKKKKKKKK)", &drop, &error, at, at + 1, at + 2, at + 3, at + 4, at + 5, at + 6, at + 7, at + 8,
                          at + 9)) return nullptr;
    if (!PyType_Check(drop) || !PyType_Check(error)) {
        PyErr_SetString(PyExc_TypeError, "two types and ten addresses");
        return nullptr;
    }
    L.dropout_forward = reinterpret_cast<decltype(L.dropout_forward)>(at[0]);
    L.dropout_backward = reinterpret_cast<decltype(L.dropout_backward)>(at[1]);
    L.norm_forward = reinterpret_cast<decltype(L.norm_forward)>(at[2]);
    L.norm_workspace = reinterpret_cast<decltype(L.norm_workspace)>(at[3]);
    L.norm_backward = reinterpret_cast<decltype(L.norm_backward)>(at[4]);
    L.mx_quantise = reinterpret_cast<decltype(L.mx_quantise)>(at[5]);
    L.mx_dequantise = reinterpret_cast<decltype(L.mx_dequantise)>(at[6]);
    L.mx_product_workspace = reinterpret_cast<decltype(L.mx_product_workspace)>(at[7]);
    L.mx_product = reinterpret_cast<decltype(L.mx_product)>(at[8]);
    L.stream_device = reinterpret_cast<decltype(L.stream_device)>(at[9]);
    Py_INCREF(drop);
    Py_INCREF(error);
    Py_XSETREF(drop_type, drop);
    Py_XSETREF(error_type, error);
    Py_RETURN_NONE;
}

#define FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"connect", connect, METH_VARARGS, nullptr}, FAST(dropout_forward), FAST(dropout_backward), FAST(norm_forward),
                         FAST(norm_backward), FAST(mx_quantise), FAST(mx_dequantise), FAST(mx_product), {nullptr, nullptr, 0, nullptr}};
#undef FAST

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_face", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__face() { return PyModule_Create(&module); }
