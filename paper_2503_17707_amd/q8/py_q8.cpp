// Tensor arguments of the 8-bit linear layers' Python wrappers (binding.py), looked over
// and handed to the C entry points.
//
// A call of one token is as long as its host work, and an attribute of a tensor costs
// 50 to 100 ns to ask for in Python, a call's four to ten tensors 2 to 3.5 us.  Here the
// same conditions take a tenth of that (one row's norm, called in a row: 6.2 -> 4.1 us, a
// product of one token 6.5 -> 5.4).  A call that does not meet them returns LOOK: the
// wrapper then finds and names what is wrong.
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/pipeboost.h"
#include "../../include/pipeboost_ops.h"

namespace {

constexpr int LOOK = 1 << 20;  // no pb_status

decltype(&pb_op_norm_q8) norm_q8;
decltype(&pb_op_quant_q8) quant_q8;
decltype(&pb_op_gemm_q8) gemm_q8;

const at::Tensor* tensor(PyObject* o) { return THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr; }

bool here(const at::Tensor& t, at::ScalarType type, int device) {
    return t.scalar_type() == type && t.layout() == at::kStrided && t.is_cuda() && t.device().index() == device;
}

// A matrix of contiguous rows (a row of one element may have any stride inside).
struct Rows {
    void* p = nullptr;
    int64_t ld = 0;
    bool read(PyObject* o, at::ScalarType type, int64_t rows, int64_t cols, int device) {
        const at::Tensor* t = tensor(o);
        if (!t || !here(*t, type, device) || t->dim() != 2 || t->size(0) != rows || t->size(1) != cols ||
            (t->stride(1) != 1 && cols != 1))
            return false;
        p = t->data_ptr();
        ld = t->stride(0);
        return true;
    }
};

bool vector(PyObject* o, at::ScalarType type, int64_t n, int device, void*& p) {
    const at::Tensor* t = tensor(o);
    if (!t || !here(*t, type, device) || t->dim() != 1 || t->size(0) != n || !t->is_contiguous()) return false;
    p = t->data_ptr();
    return true;
}

// The device of a call and its stream; -1 where the first tensor is not on the current device.
// (device, stream): those of the stream that was given, (-1, 0) for the current one.
int device_of(const at::Tensor& t, PyObject* device, PyObject* stream, void*& s) {
    if (!t.is_cuda() || t.device().index() != c10::hip::current_device()) return -1;
    const long given = PyLong_AsLong(device);
    if (given < 0) {
        s = c10::hip::getCurrentHIPStream(t.device().index()).stream();
    } else {
        if (given != t.device().index()) return -1;
        s = PyLong_AsVoidPtr(stream);
    }
    return t.device().index();
}

at::ScalarType storage(long dtype) { return dtype == PB_F16 ? at::kHalf : at::kBFloat16; }

bool none(PyObject* o) { return o == Py_None; }

// dtype, layer, x, g, q, scale, delta, sum, b, out, eps, stream's device, stream
int norm(PyObject* const* a) {
    const long dtype = PyLong_AsLong(a[0]);
    const int layer = PyObject_IsTrue(a[1]);
    const float eps = (float)PyFloat_AsDouble(a[10]);
    const at::Tensor* x = tensor(a[2]);
    if (PyErr_Occurred()) return -1;
    if ((dtype != PB_BF16 && dtype != PB_F16) || !x || x->dim() != 2) return LOOK;
    void* stream;
    const int dev = device_of(*x, a[11], a[12], stream);
    if (PyErr_Occurred()) return -1;
    if (dev < 0 || none(a[4]) != none(a[5])) return LOOK;
    const at::ScalarType type = storage(dtype), xt = x->scalar_type();
    const int64_t rows = x->size(0), d = x->size(1);
    Rows rx, rdelta, rsum, rout, rq;
    void *g, *b = nullptr, *scale = nullptr;
    if ((xt != at::kFloat && xt != type) || !rx.read(a[2], xt, rows, d, dev) || !vector(a[3], type, d, dev, g) ||
        (!none(a[4]) && !(rq.read(a[4], at::kChar, rows, d, dev) && vector(a[5], at::kFloat, rows, dev, scale))) ||
        (!none(a[6]) && !rdelta.read(a[6], type, rows, d, dev)) || (!none(a[7]) && !rsum.read(a[7], xt, rows, d, dev)) ||
        (!none(a[8]) && !vector(a[8], type, d, dev, b)) || (!none(a[9]) && !rout.read(a[9], type, rows, d, dev)) ||
        rows > INT32_MAX || d > INT32_MAX)
        return LOOK;
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = norm_q8((int)dtype, layer, rx.p, rx.ld, xt == at::kFloat, rdelta.p, rdelta.ld, rsum.p, rsum.ld, g, b, eps, rout.p,
                 rout.ld, (int8_t*)rq.p, rq.ld, (float*)scale, (int)rows, (int)d, stream);
    Py_END_ALLOW_THREADS;
    return rc;
}

// dtype, x, q, scale, stream's device, stream
int quant(PyObject* const* a) {
    const long dtype = PyLong_AsLong(a[0]);
    const at::Tensor* x = tensor(a[1]);
    if (PyErr_Occurred()) return -1;
    if ((dtype != PB_BF16 && dtype != PB_F16) || !x || x->dim() != 2) return LOOK;
    void* stream;
    const int dev = device_of(*x, a[4], a[5], stream);
    if (PyErr_Occurred()) return -1;
    if (dev < 0) return LOOK;
    const at::ScalarType xt = x->scalar_type();
    const int64_t rows = x->size(0), cols = x->size(1);
    Rows rx, rq;
    void* scale;
    if ((xt != at::kFloat && xt != storage(dtype)) || !rx.read(a[1], xt, rows, cols, dev) ||
        !rq.read(a[2], at::kChar, rows, cols, dev) || !vector(a[3], at::kFloat, rows, dev, scale) || rows > INT32_MAX ||
        cols > INT32_MAX)
        return LOOK;
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = quant_q8((int)dtype, rx.p, rx.ld, xt == at::kFloat, (int8_t*)rq.p, rq.ld, (float*)scale, (int)rows, (int)cols,
                  stream);
    Py_END_ALLOW_THREADS;
    return rc;
}

// dtype, epi, X, sx, W, sw, bias, C, R, qscale, qcols, workspace, stream's device, stream
int gemm(PyObject* const* a) {
    const long dtype = PyLong_AsLong(a[0]), epi = PyLong_AsLong(a[1]), qcols = PyLong_AsLong(a[10]);
    const float qscale = (float)PyFloat_AsDouble(a[9]);
    const at::Tensor *X = tensor(a[2]), *W = tensor(a[4]);
    if (PyErr_Occurred()) return -1;
    if ((dtype != PB_BF16 && dtype != PB_F16) || epi < 0 || epi > 3 || !X || !W || X->dim() != 2 || W->dim() != 2) return LOOK;
    void* stream;
    const int dev = device_of(*X, a[12], a[13], stream);
    if (PyErr_Occurred()) return -1;
    if (dev < 0) return LOOK;
    const at::ScalarType type = storage(dtype);
    const bool wide = epi >= 2;
    const int64_t M = X->size(0), K = X->size(1), N = W->size(0);
    Rows rx, rw, out;
    void *sx, *sw, *bias = nullptr, *ws = nullptr;
    size_t ws_bytes = 0;
    if (!rx.read(a[2], at::kChar, M, K, dev) || !rw.read(a[4], at::kChar, N, K, dev) || !vector(a[3], at::kFloat, M, dev, sx) ||
        !vector(a[5], at::kFloat, N, dev, sw) || (!none(a[6]) && !vector(a[6], type, N, dev, bias)) ||
        !out.read(a[wide ? 8 : 7], wide ? at::kFloat : type, M, N, dev) || M > INT32_MAX || N > INT32_MAX || K > INT32_MAX ||
        qcols > INT32_MAX || qcols < INT32_MIN)
        return LOOK;
    if (!none(a[11])) {
        const at::Tensor* w = tensor(a[11]);
        if (!w || !here(*w, w->scalar_type(), dev) || !w->is_contiguous()) return LOOK;
        ws = w->data_ptr();
        ws_bytes = w->nbytes();
    }
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = gemm_q8((int)dtype, (int)epi, (const int8_t*)rx.p, rx.ld, (const float*)sx, (const int8_t*)rw.p, rw.ld,
                 (const float*)sw, bias, wide ? nullptr : out.p, wide ? (float*)out.p : nullptr, out.ld, (int)M, (int)N, (int)K,
                 qscale, (int)qcols, ws, ws_bytes, stream);
    Py_END_ALLOW_THREADS;
    return rc;
}

template <int (*F)(PyObject* const*), int N>
PyObject* call(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "%d arguments, not %zd", N, n);
        return nullptr;
    }
    int rc;
    try {
        rc = F(a);
    } catch (const std::exception& e) {  // (a tensor without storage)
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
    return PyErr_Occurred() ? nullptr : PyLong_FromLong(rc);
}

// The addresses of the C entry points in the library that binding.py has loaded.
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 3) {
        PyErr_SetString(PyExc_TypeError, "3 addresses");
        return nullptr;
    }
    norm_q8 = (decltype(norm_q8))PyLong_AsVoidPtr(a[0]);
    quant_q8 = (decltype(quant_q8))PyLong_AsVoidPtr(a[1]);
    gemm_q8 = (decltype(gemm_q8))PyLong_AsVoidPtr(a[2]);
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
}

PyMethodDef METHODS[] = {
    {"bind", (PyCFunction)(void (*)())bind, METH_FASTCALL, nullptr},
    {"norm", (PyCFunction)(void (*)())call<norm, 13>, METH_FASTCALL, nullptr},
    {"quant", (PyCFunction)(void (*)())call<quant, 6>, METH_FASTCALL, nullptr},
    {"gemm", (PyCFunction)(void (*)())call<gemm, 14>, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef MODULE = {PyModuleDef_HEAD_INIT, "pipeboost_q8_args", nullptr, -1, METHODS, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_pipeboost_q8_args() {
    PyObject* m = PyModule_Create(&MODULE);
    if (m && (PyModule_AddIntConstant(m, "LOOK", LOOK) < 0 || PyModule_AddStringConstant(m, "TORCH", PB_TORCH) < 0)) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
