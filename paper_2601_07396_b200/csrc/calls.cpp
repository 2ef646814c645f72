// The argument side of the 8-bit calls as a Python extension: a torch tensor's pointer, sizes, strides, type and device
// are read here in nanoseconds, where the interpreter takes 0.05-0.2 us for each -- 3 us of checks and 1.4 us of ctypes
// conversion beside kernels that can take less.  Nothing is computed here: the functions check what the C ABI cannot
// see (shapes against one another, device, contiguity), call it, and return its status code.  binding.py holds the
// public functions, loads this module next to the library and hands it the library's entry points.
#include <Python.h>

#include <cstdint>

#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/svdcache.h"

namespace {

using QuantizeFn = decltype(&svdcache_quantize_fp8);
using NormFn = decltype(&svdcache_residual_rmsnorm_fp8);
using GemmFn = decltype(&svdcache_gemm_fp8);
using StatusWordFn = decltype(&svdcache_gemm_fp8_status_word);
QuantizeFn g_quantize = nullptr;
NormFn g_norm = nullptr;
GemmFn g_gemm = nullptr;
StatusWordFn g_status_word = nullptr;

struct Refusal {};   // a Python error is set

[[noreturn]] void refuse(const char *what, const char *want) {
    PyErr_Format(PyExc_ValueError, "%s: %s", what, want);
    throw Refusal{};
}

const at::Tensor &tensor(PyObject *o, const char *what) {
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s: a tensor is expected", what);
        throw Refusal{};
    }
    return THPVariable_Unpack(o);
}

struct Matrix {
    void *p;
    int64_t rows, cols, ld;
};

// a matrix of contiguous rows on the device; torch gives a single row any stride
Matrix matrix(const at::Tensor &t, int device, const char *what) {
    if (t.dim() != 2 || !t.is_cuda() || t.get_device() != device) refuse(what, "a matrix on the same device is expected");
    const int64_t rows = t.size(0), cols = t.size(1);
    if (t.stride(1) != 1 && cols != 1) refuse(what, "contiguous rows are expected");
    return {t.data_ptr(), rows, cols, rows == 1 ? (cols + 15) / 16 * 16 : t.stride(0)};
}

struct Fp8 {
    void *q, *s;
    int64_t ld;
};

// Values as e4m3 or plain bytes, scales as E8M0 or plain bytes: other types of one byte (e5m2, int8, bool) would be read as
// what they are not.
bool holds_values(const at::Tensor &t) { return t.scalar_type() == at::kByte || t.scalar_type() == at::kFloat8_e4m3fn; }
bool holds_scales(const at::Tensor &t) { return t.scalar_type() == at::kByte || t.scalar_type() == at::kFloat8_e8m0fnu; }

// a matrix of at least `cols` columns, and its scale buffer
Fp8 fp8(PyObject *qo, PyObject *so, int64_t rows, int64_t cols, int device, const char *what) {
    const at::Tensor &q = tensor(qo, what), &s = tensor(so, what);
    const Matrix m = matrix(q, device, what);
    if (m.rows != rows || m.cols < cols || !holds_values(q)) refuse(what, "a byte (uint8 or float8_e4m3fn) for each element is expected");
    if (!s.is_cuda() || s.get_device() != device || !holds_scales(s) || !s.is_contiguous() ||
        s.numel() < (rows + 127) / 128 * ((cols + 511) / 512) * 512)
        refuse(what, "a scale buffer of svdcache_fp8_scale_bytes(rows, cols) bytes (uint8 or float8_e8m0fnu) is expected");
    return {m.p, s.data_ptr(), m.ld};
}

const float *vector(PyObject *o, int64_t n, int device, const char *what) {
    if (o == Py_None) return nullptr;
    const at::Tensor &t = tensor(o, what);
    if (t.scalar_type() != at::kFloat || t.dim() != 1 || t.size(0) != n || !t.is_cuda() || t.get_device() != device || !t.is_contiguous())
        refuse(what, "one fp32 value for each column on the same device is expected");
    return static_cast<const float *>(t.data_ptr());
}

// where a time-out is written: nothing else may lie there
int32_t *status_word(PyObject *o, int device) {
    if (o == Py_None) return nullptr;
    const at::Tensor &t = tensor(o, "status");
    if (t.scalar_type() != at::kInt || t.numel() < 1 || !t.is_cuda() || t.get_device() != device)
        refuse("status", "an int32 word on the same device is expected");
    return static_cast<int32_t *>(t.data_ptr());
}

int plain_type(const at::Tensor &t, const char *what) {
    if (t.scalar_type() == at::kFloat) return SVDCACHE_F32;
    if (t.scalar_type() == at::kBFloat16) return SVDCACHE_BF16;
    refuse(what, "fp32 or bf16 is expected");
}

int device_of(const at::Tensor &t, const char *what) {
    if (!t.is_cuda()) refuse(what, "a device matrix is expected");
    return (int)t.get_device();
}

// a number beyond int becomes its nearest, which the library refuses wherever an int is expected here
int dim32(int64_t n) { return n > INT32_MAX ? INT32_MAX : n < INT32_MIN ? INT32_MIN : (int)n; }

long long number(PyObject *o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Refusal{};
    return v;
}

// None: the current stream of the tensors' device
void *stream_of(PyObject *o, int device) {
    if (o == Py_None) return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
    return reinterpret_cast<void *>(static_cast<uintptr_t>(number(o)));
}

// the library launches on the current device: the tensors' one for the length of the call
template <typename F> PyObject *call(int device, F f) {
    const c10::cuda::CUDAGuard guard((c10::DeviceIndex)device);
    int rc = 0;
    PyThreadState *save = PyEval_SaveThread();
    rc = f();
    PyEval_RestoreThread(save);
    return PyLong_FromLong(rc);
}

// no exception of C++ passes into the interpreter
template <typename F> PyObject *guarded(Py_ssize_t n, Py_ssize_t want, F f) {
    if (n != want) {
        PyErr_Format(PyExc_TypeError, "%zd arguments are expected", want);
        return nullptr;
    }
    try {
        return f();
    } catch (const Refusal &) {
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
    }
    return nullptr;
}

// bind(quantize, norm, gemm, status_word): addresses of the library's functions
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 4, [&]() -> PyObject * {
        g_quantize = reinterpret_cast<QuantizeFn>(static_cast<uintptr_t>(number(a[0])));
        g_norm = reinterpret_cast<NormFn>(static_cast<uintptr_t>(number(a[1])));
        g_gemm = reinterpret_cast<GemmFn>(static_cast<uintptr_t>(number(a[2])));
        g_status_word = reinterpret_cast<StatusWordFn>(static_cast<uintptr_t>(number(a[3])));
        Py_RETURN_NONE;
    });
}

// quantize(X, Q, S, tile_rows, stream)
PyObject *quantize(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 5, [&] {
        const at::Tensor &x = tensor(a[0], "X");
        const int dev = device_of(x, "X"), type = plain_type(x, "X"), tile_rows = dim32(number(a[3]));
        const Matrix m = matrix(x, dev, "X");
        const Fp8 q = fp8(a[1], a[2], m.rows, m.cols, dev, "Q");
        void *stream = stream_of(a[4], dev);
        return call(dev, [&] { return g_quantize(m.p, m.rows, dim32(m.cols), m.ld, type, tile_rows, q.q, q.ld, q.s, stream); });
    });
}

// norm(H, X or None, H_out or None, weight or None, eps, Q, S, stream)
PyObject *norm(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 8, [&] {
        const at::Tensor &h = tensor(a[0], "H");
        const int dev = device_of(h, "H"), type = plain_type(h, "H");
        const Matrix m = matrix(h, dev, "H");
        Matrix side[2] = {{nullptr, 0, 0, 0}, {nullptr, 0, 0, 0}};
        for (int i = 0; i < 2; ++i) {
            if (a[1 + i] == Py_None) continue;
            const char *what = i ? "H_out" : "X";
            const at::Tensor &t = tensor(a[1 + i], what);
            side[i] = matrix(t, dev, what);
            if (side[i].rows != m.rows || side[i].cols != m.cols || t.scalar_type() != h.scalar_type()) refuse(what, "H's shape and type are expected");
        }
        const float *weight = vector(a[3], m.cols, dev, "weight");
        const double eps = PyFloat_AsDouble(a[4]);
        if (eps == -1.0 && PyErr_Occurred()) throw Refusal{};
        const Fp8 q = fp8(a[5], a[6], m.rows, m.cols, dev, "Q");
        void *stream = stream_of(a[7], dev);
        return call(dev, [&] {
            return g_norm(m.p, m.ld, side[0].p, side[0].ld, side[1].p, side[1].ld, weight, (float)eps, q.q, q.ld, q.s, m.rows, dim32(m.cols), type, stream);
        });
    });
}

// gemm(A, SA, B, SB, K, C, S_out or None, bias or None, act, status word or None: the library's own, stream)
PyObject *gemm(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 11, [&] {
        const at::Tensor &c = tensor(a[5], "C");
        const int dev = device_of(c, "C"), act = dim32(number(a[8]));
        const Matrix m = matrix(c, dev, "C");
        const long long K = number(a[4]);
        if (K < 0) refuse("K", "a count of columns is expected");
        const Fp8 A = fp8(a[0], a[1], m.rows, K, dev, "A"), B = fp8(a[2], a[3], m.cols, K, dev, "B");
        const float *bias = vector(a[7], m.cols, dev, "bias");
        int out = SVDCACHE_FP8;
        void *sc = nullptr;
        if (c.element_size() == 1) {
            if (a[6] == Py_None) refuse("S_out", "an 8-bit C needs a scale buffer");
            sc = fp8(a[5], a[6], m.rows, m.cols, dev, "C").s;
        } else {
            out = plain_type(c, "C");
        }
        int32_t *status = status_word(a[9], dev);
        void *stream = stream_of(a[10], dev);
        return call(dev, [&] {
            const int rc = status ? SVDCACHE_OK : g_status_word(&status);
            if (rc) return rc;
            return g_gemm(A.q, A.ld, A.s, B.q, B.ld, B.s, bias, act, m.p, m.ld, out, sc, m.rows, dim32(m.cols), dim32(K), status, stream);
        });
    });
}

PyMethodDef methods[] = {
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(bind)), METH_FASTCALL, nullptr},
    {"quantize", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(quantize)), METH_FASTCALL, nullptr},
    {"norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(norm)), METH_FASTCALL, nullptr},
    {"gemm", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(gemm)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&module); }
