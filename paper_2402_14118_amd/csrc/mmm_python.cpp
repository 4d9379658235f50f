// CPython entry points for the calls a program makes per step (mmm_build_maps, mmm_matmul,
// mmm_matmul_fused, mmm_matmul_epilogue, mmm_matmul_backward, mmm_block_norm, mmm_epilogue_backward,
// mmm_block_norm_backward).  They do what the ctypes functions of binding.py do -- marshal integers and call
// the C ABI -- at 0.3 instead of about 3 us per call: a small problem is bound by the host, where a
// kernel launch alone takes 3.5 us.  Pointers are passed as integers (None = NULL).  The GIL is
// released around the call, as ctypes does.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "mmm.h"

namespace {

// integer arguments; reading stops at the first bad one
struct Args {
    PyObject *const *v;
    bool ok = true;
    void *ptr(int i)
    {
        if (!ok || v[i] == Py_None) return nullptr;
        void *p = PyLong_AsVoidPtr(v[i]);
        if (p == nullptr && PyErr_Occurred()) ok = false;
        return p;
    }
    int64_t num(int i)
    {
        if (!ok) return 0;
        const long long n = PyLong_AsLongLong(v[i]);
        if (n == -1 && PyErr_Occurred()) ok = false;
        return (int64_t)n;
    }
    float real(int i)
    {
        if (!ok) return 0.f;
        const double d = PyFloat_AsDouble(v[i]);
        if (d == -1.0 && PyErr_Occurred()) ok = false;
        return (float)d;
    }
};

bool arity(const char *name, Py_ssize_t n, Py_ssize_t want)
{
    if (n == want) return true;
    PyErr_Format(PyExc_TypeError, "%s takes %zd arguments, got %zd", name, want, n);
    return false;
}

// build_maps(maps, dtype, X, ldx, has_ma, pred, threshold, keep_a, Y, ldy, has_mb, block_width, keep_rows, keep_blocks, stream)
PyObject *build_maps(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    if (!arity("build_maps", n, 15)) return nullptr;
    Args a{v};
    mmm_maps *maps = static_cast<mmm_maps *>(a.ptr(0));
    const mmm_dtype dt = (mmm_dtype)a.num(1);
    const void *X = a.ptr(2);
    const int64_t ldx = a.num(3);
    const bool has_ma = a.num(4) != 0;
    const mmm_mask_a ma{(int32_t)a.num(5), a.real(6), static_cast<const uint64_t *>(a.ptr(7))};
    const void *Y = a.ptr(8);
    const int64_t ldy = a.num(9);
    const bool has_mb = a.num(10) != 0;
    const mmm_mask_b mb{(int32_t)a.num(11), static_cast<const uint64_t *>(a.ptr(12)), static_cast<const uint64_t *>(a.ptr(13))};
    void *stream = a.ptr(14);
    if (!a.ok) return nullptr;
    mmm_status st;
    Py_BEGIN_ALLOW_THREADS
    st = mmm_build_maps(maps, dt, X, ldx, has_ma ? &ma : nullptr, Y, ldy, has_mb ? &mb : nullptr, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

// matmul(maps, dtype, X, ldx, Y, ldy, C, ldc, accumulate, stream)
PyObject *matmul(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    if (!arity("matmul", n, 10)) return nullptr;
    Args a{v};
    const mmm_maps *maps = static_cast<const mmm_maps *>(a.ptr(0));
    const mmm_dtype dt = (mmm_dtype)a.num(1);
    const void *X = a.ptr(2);
    const int64_t ldx = a.num(3);
    const void *Y = a.ptr(4);
    const int64_t ldy = a.num(5);
    void *C = a.ptr(6);
    const int64_t ldc = a.num(7);
    const int32_t acc = (int32_t)a.num(8);
    void *stream = a.ptr(9);
    if (!a.ok) return nullptr;
    mmm_status st;
    Py_BEGIN_ALLOW_THREADS
    st = mmm_matmul(maps, dt, X, ldx, Y, ldy, C, ldc, acc, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

// matmul_fused(maps, dtype, X, ldx, pred, threshold, keep_a, Y, ldy, C, ldc, accumulate, stream)
PyObject *matmul_fused(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    if (!arity("matmul_fused", n, 13)) return nullptr;
    Args a{v};
    const mmm_maps *maps = static_cast<const mmm_maps *>(a.ptr(0));
    const mmm_dtype dt = (mmm_dtype)a.num(1);
    const void *X = a.ptr(2);
    const int64_t ldx = a.num(3);
    const mmm_mask_a ma{(int32_t)a.num(4), a.real(5), static_cast<const uint64_t *>(a.ptr(6))};
    const void *Y = a.ptr(7);
    const int64_t ldy = a.num(8);
    void *C = a.ptr(9);
    const int64_t ldc = a.num(10);
    const int32_t acc = (int32_t)a.num(11);
    void *stream = a.ptr(12);
    if (!a.ok) return nullptr;
    mmm_status st;
    Py_BEGIN_ALLOW_THREADS
    st = mmm_matmul_fused(maps, dt, X, ldx, &ma, Y, ldy, C, ldc, acc, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

// matmul_epilogue(maps, dtype, X, ldx, has_ma, pred, threshold, keep_a, Y, ldy, C, ldc, activation, out_dtype, bias, residual, ldr, preact, ldp,
// stream)
PyObject *matmul_epilogue(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    if (!arity("matmul_epilogue", n, 20)) return nullptr;
    Args a{v};
    const mmm_maps *maps = static_cast<const mmm_maps *>(a.ptr(0));
    const mmm_dtype dt = (mmm_dtype)a.num(1);
    const void *X = a.ptr(2);
    const int64_t ldx = a.num(3);
    const bool has_ma = a.num(4) != 0;
    const mmm_mask_a ma{(int32_t)a.num(5), a.real(6), static_cast<const uint64_t *>(a.ptr(7))};
    const void *Y = a.ptr(8);
    const int64_t ldy = a.num(9);
    void *C = a.ptr(10);
    const int64_t ldc = a.num(11);
    const int32_t activation = (int32_t)a.num(12), out_dtype = (int32_t)a.num(13);
    const void *bias = a.ptr(14), *residual = a.ptr(15);
    const int64_t ldr = a.num(16);
    void *preact = a.ptr(17);
    const int64_t ldp = a.num(18);
    const mmm_epilogue e{activation, out_dtype, bias, residual, ldr, preact, ldp};
    void *stream = a.ptr(19);
    if (!a.ok) return nullptr;
    mmm_status st;
    Py_BEGIN_ALLOW_THREADS
    st = mmm_matmul_epilogue(maps, dt, X, ldx, has_ma ? &ma : nullptr, Y, ldy, C, ldc, &e, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

// A mmm_block_norm_desc from (M, N, dt, dt_h, dt_y, post, pre, gate, eps, alpha).
bool description(PyObject *t, mmm_block_norm_desc &d)
{
    if (!PyTuple_Check(t) || PyTuple_GET_SIZE(t) != 10) {
        PyErr_SetString(PyExc_TypeError, "the description of a norm has ten fields");
        return false;
    }
    Args a{&PyTuple_GET_ITEM(t, 0)};
    d.M = a.num(0);
    d.N = a.num(1);
    d.dt = (int32_t)a.num(2);
    d.dt_h = (int32_t)a.num(3);
    d.dt_y = (int32_t)a.num(4);
    d.post = (int32_t)a.num(5);
    d.pre = (int32_t)a.num(6);
    d.gate = (int32_t)a.num(7);
    d.eps = a.real(8);
    d.alpha = a.real(9);
    return a.ok;
}

// block_norm(description, h, ldh, y, ldy, gate, ldgate, post_weight, post_bias, pre_weight, pre_bias, h_out, ldh_out, n, ldn, stream)
PyObject *block_norm(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    if (!arity("block_norm", n, 16)) return nullptr;
    mmm_block_norm_desc d;
    if (!description(v[0], d)) return nullptr;
    Args a{v};
    const void *h = a.ptr(1);
    const int64_t ldh = a.num(2);
    const void *y = a.ptr(3);
    const int64_t ldy = a.num(4);
    const void *gate = a.ptr(5);
    const int64_t ldgate = a.num(6);
    const void *post_weight = a.ptr(7), *post_bias = a.ptr(8), *pre_weight = a.ptr(9), *pre_bias = a.ptr(10);
    void *h_out = a.ptr(11);
    const int64_t ldh_out = a.num(12);
    void *out = a.ptr(13);
    const int64_t ldn = a.num(14);
    void *stream = a.ptr(15);
    if (!a.ok) return nullptr;
    mmm_status st;
    Py_BEGIN_ALLOW_THREADS
    st = mmm_block_norm(&d, h, ldh, y, ldy, gate, ldgate, post_weight, post_bias, pre_weight, pre_bias, h_out, ldh_out, out, ldn, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

// epilogue_backward(M, N, dt, out_dtype, activation, dC, lddc, Z, ldz, dZ, lddz, dbias, workspace, workspace_bytes, stream)
PyObject *epilogue_backward(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    if (!arity("epilogue_backward", n, 15)) return nullptr;
    Args a{v};
    const int64_t M = a.num(0), N = a.num(1);
    const mmm_dtype dt = (mmm_dtype)a.num(2), out_dtype = (mmm_dtype)a.num(3);
    const int32_t activation = (int32_t)a.num(4);
    const void *dC = a.ptr(5);
    const int64_t lddc = a.num(6);
    const void *Z = a.ptr(7);
    const int64_t ldz = a.num(8);
    void *dZ = a.ptr(9);
    const int64_t lddz = a.num(10);
    float *dbias = static_cast<float *>(a.ptr(11));
    void *ws = a.ptr(12);
    const size_t bytes = (size_t)a.num(13);
    void *stream = a.ptr(14);
    if (!a.ok) return nullptr;
    mmm_status st;
    Py_BEGIN_ALLOW_THREADS
    st = mmm_epilogue_backward(M, N, dt, out_dtype, activation, dC, lddc, Z, ldz, dZ, lddz, dbias, ws, bytes, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

// matmul_backward(maps, dtype, X, ldx, Y, ldy, dC, lddc, dX, lddx, dY, lddy, accumulate, all_x, stream)
PyObject *matmul_backward(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    if (!arity("matmul_backward", n, 15)) return nullptr;
    Args a{v};
    const mmm_maps *maps = static_cast<const mmm_maps *>(a.ptr(0));
    const mmm_dtype dt = (mmm_dtype)a.num(1);
    const void *X = a.ptr(2);
    const int64_t ldx = a.num(3);
    const void *Y = a.ptr(4);
    const int64_t ldy = a.num(5);
    const void *dC = a.ptr(6);
    const int64_t lddc = a.num(7);
    void *dX = a.ptr(8);
    const int64_t lddx = a.num(9);
    float *dY = static_cast<float *>(a.ptr(10));
    const int64_t lddy = a.num(11);
    const int32_t acc = (int32_t)a.num(12), all_x = (int32_t)a.num(13);
    void *stream = a.ptr(14);
    if (!a.ok) return nullptr;
    mmm_status st;
    Py_BEGIN_ALLOW_THREADS
    st = mmm_matmul_backward(maps, dt, X, ldx, Y, ldy, dC, lddc, dX, lddx, dY, lddy, acc, all_x, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

// block_norm_backward(description, h_out, ldh_out, y, ldy, gate, ldgate, post_weight, post_bias, pre_weight, d_n, ldd_n, d_h_out, ldd_h_out, d_h, ldd_h,
// d_y, ldd_y, d_gate, ldd_gate, d_post_weight, d_post_bias, d_pre_weight, d_pre_bias, workspace, workspace_bytes, stream)
PyObject *block_norm_backward(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    if (!arity("block_norm_backward", n, 27)) return nullptr;
    mmm_block_norm_desc d;
    if (!description(v[0], d)) return nullptr;
    Args a{v};
    mmm_block_norm_grads g;
    g.h_out = a.ptr(1);
    g.ldh_out = a.num(2);
    g.y = a.ptr(3);
    g.ldy = a.num(4);
    g.gate_values = a.ptr(5);
    g.ldgate = a.num(6);
    g.post_weight = a.ptr(7);
    g.post_bias = a.ptr(8);
    g.pre_weight = a.ptr(9);
    g.d_n = a.ptr(10);
    g.ldd_n = a.num(11);
    g.d_h_out = a.ptr(12);
    g.ldd_h_out = a.num(13);
    g.d_h = a.ptr(14);
    g.ldd_h = a.num(15);
    g.d_y = a.ptr(16);
    g.ldd_y = a.num(17);
    g.d_gate = a.ptr(18);
    g.ldd_gate = a.num(19);
    g.d_post_weight = static_cast<float *>(a.ptr(20));
    g.d_post_bias = static_cast<float *>(a.ptr(21));
    g.d_pre_weight = static_cast<float *>(a.ptr(22));
    g.d_pre_bias = static_cast<float *>(a.ptr(23));
    void *ws = a.ptr(24);
    const size_t bytes = (size_t)a.num(25);
    void *stream = a.ptr(26);
    if (!a.ok) return nullptr;
    mmm_status st;
    Py_BEGIN_ALLOW_THREADS
    st = mmm_block_norm_backward(&d, &g, ws, bytes, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

// The address (a new reference) and the leading dimension of a matrix (0: of a vector) that has this shape, type and device and whose elements are
// neighbours; null where anything differs.
PyObject *located(PyObject *t, PyObject *want, PyObject *type, PyObject *where, long long &ld)
{
    static PyObject *const shape_name = PyUnicode_InternFromString("shape"), *const dtype_name = PyUnicode_InternFromString("dtype"),
                           *const device_name = PyUnicode_InternFromString("device"), *const stride_name = PyUnicode_InternFromString("stride"),
                           *const address_name = PyUnicode_InternFromString("data_ptr");
    ld = -1;
    PyObject *const shape = PyObject_GetAttr(t, shape_name), *const dtype = PyObject_GetAttr(t, dtype_name), *const device = PyObject_GetAttr(t, device_name);
    PyObject *stride = nullptr, *address = nullptr;
    if (shape != nullptr && device != nullptr && PyTuple_Check(shape) && PyTuple_Check(want) && dtype == type) {
        const Py_ssize_t dims = PyTuple_GET_SIZE(want);
        bool same = (dims == 1 || dims == 2) && PyTuple_GET_SIZE(shape) == dims;
        long long size[2] = {1, 1};
        for (Py_ssize_t i = 0; same && i < dims; ++i) {
            size[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(want, i));
            same = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, i)) == size[i];
        }
        if (same && PyObject_RichCompareBool(device, where, Py_EQ) == 1) stride = PyObject_CallMethodNoArgs(t, stride_name);
        if (stride != nullptr && PyTuple_Check(stride) && PyTuple_GET_SIZE(stride) == dims) {
            const long long last = PyLong_AsLongLong(PyTuple_GET_ITEM(stride, dims - 1)), first = PyLong_AsLongLong(PyTuple_GET_ITEM(stride, 0));
            if (last == 1 || size[dims - 1] <= 1) ld = dims == 1 ? 0 : size[0] > 1 || first > size[1] ? first : size[1];
        }
        if (ld >= 0) address = PyObject_CallMethodNoArgs(t, address_name);
    }
    Py_XDECREF(shape);
    Py_XDECREF(dtype);
    Py_XDECREF(device);
    Py_XDECREF(stride);
    if (address == nullptr) PyErr_Clear();
    return address;
}

// places(device, needed, tensor, shape, dtype, tensor, shape, dtype, ...): (address, leading dimension, address, leading dimension, ...) of all, None and 0 of a
// tensor that is None; the first `needed` have to be there.  Where something is wrong, the number of that tensor.
PyObject *places(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    if (n < 2 || (n - 2) % 3 != 0) {
        PyErr_SetString(PyExc_TypeError, "places takes a device, a number and three arguments for each tensor");
        return nullptr;
    }
    const Py_ssize_t tensors = (n - 2) / 3;
    const long long needed = PyLong_AsLongLong(v[1]);
    if (needed == -1 && PyErr_Occurred()) return nullptr;
    PyObject *const out = PyTuple_New(2 * tensors);
    if (out == nullptr) return nullptr;
    for (Py_ssize_t i = 0; i < tensors; ++i) {
        PyObject *const *const at = v + 2 + 3 * i;
        long long ld = 0;
        PyObject *address = nullptr;
        if (at[0] == Py_None && i >= needed) {
            Py_INCREF(Py_None);
            address = Py_None;
        } else if (at[0] != Py_None) {
            address = located(at[0], at[1], at[2], v[0], ld);
        }
        PyObject *const leading = address != nullptr ? PyLong_FromLongLong(ld) : nullptr;
        if (leading == nullptr) {
            Py_XDECREF(address);
            Py_DECREF(out);
            return PyErr_Occurred() ? nullptr : PyLong_FromSsize_t(i);
        }
        PyTuple_SET_ITEM(out, 2 * i, address);
        PyTuple_SET_ITEM(out, 2 * i + 1, leading);
    }
    return out;
}

PyMethodDef methods[] = {
    {"build_maps", (PyCFunction)(void (*)(void))build_maps, METH_FASTCALL, nullptr},
    {"matmul", (PyCFunction)(void (*)(void))matmul, METH_FASTCALL, nullptr},
    {"matmul_fused", (PyCFunction)(void (*)(void))matmul_fused, METH_FASTCALL, nullptr},
    {"matmul_epilogue", (PyCFunction)(void (*)(void))matmul_epilogue, METH_FASTCALL, nullptr},
    {"block_norm", (PyCFunction)(void (*)(void))block_norm, METH_FASTCALL, nullptr},
    {"epilogue_backward", (PyCFunction)(void (*)(void))epilogue_backward, METH_FASTCALL, nullptr},
    {"matmul_backward", (PyCFunction)(void (*)(void))matmul_backward, METH_FASTCALL, nullptr},
    {"block_norm_backward", (PyCFunction)(void (*)(void))block_norm_backward, METH_FASTCALL, nullptr},
    {"places", (PyCFunction)(void (*)(void))places, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_mmm_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}   // namespace

PyMODINIT_FUNC PyInit__mmm_native(void) { return PyModule_Create(&module); }
