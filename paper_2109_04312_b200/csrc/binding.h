// What the two halves of the native binding share: exceptions, checks of tensors, allocation (binding.cpp: calls on a plan;
// binding_cache.cpp: rotary positions and calls on a cache).
#pragma once
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <optional>

#include "mate.h"

namespace mate_binding {

extern PyObject *mate_error;  // exception class, called with (status, where)

struct Raised {};  // a Python exception is set

// Other Python threads run while a call may wait: the allocator for memory to become free, a launch for room in
// the queue, the first use of a plan on another stream for its upload.
struct NoGil {
    PyThreadState *state = PyEval_SaveThread();
    NoGil() = default;
    NoGil(const NoGil &) = delete;
    ~NoGil() { PyEval_RestoreThread(state); }
};

[[noreturn]] inline void fail(PyObject *type, const char *msg) {
    PyErr_SetString(type, msg);
    throw Raised();
}
[[noreturn]] inline void fail_named(PyObject *type, const char *format, const char *name) {
    PyErr_Format(type, format, name);
    throw Raised();
}
inline void check(int status, const char *where) {
    if (status == MATE_OK) return;
    PyObject *e = PyObject_CallFunction(mate_error, "is", status, where);
    if (e) {
        PyErr_SetObject(mate_error, e);
        Py_DECREF(e);
    }
    throw Raised();
}

inline const at::Tensor &tensor(PyObject *o, const char *name) {
    if (!THPVariable_Check(o)) fail_named(PyExc_ValueError, "%s must be a contiguous CUDA tensor", name);
    return THPVariable_Unpack(o);
}
inline void *dev(const at::Tensor &t, const char *name) {
    if (!t.is_cuda() || !t.is_contiguous()) fail_named(PyExc_ValueError, "%s must be a contiguous CUDA tensor", name);
    return t.data_ptr();
}
inline int dtype_code(const at::Tensor &t) {
    if (t.scalar_type() == at::kBFloat16) return MATE_BF16;
    if (t.scalar_type() == at::kFloat) return MATE_F32;
    PyErr_Format(PyExc_TypeError, "libmate takes bfloat16 or float32 tensors, got %s", c10::toString(t.scalar_type()));
    throw Raised();
}
inline float scale_of(PyObject *o, int64_t d) {
    if (o == Py_None) return (float)(1.0 / std::sqrt((double)d));
    const double s = PyFloat_AsDouble(o);
    if (s == -1.0 && PyErr_Occurred()) throw Raised();
    return (float)s;
}
inline unsigned flags_of(PyObject *o) {
    const unsigned long f = PyLong_AsUnsignedLongMask(o);
    if (PyErr_Occurred()) throw Raised();
    return (unsigned)f;
}
inline at::Tensor empty(c10::IntArrayRef size, at::ScalarType type, c10::Device device) {
    return at::Tensor(at::detail::empty_cuda(size, type, device, std::nullopt));
}

// A tensor that is read or written as `n` elements of a type has that type, and at least as many.
inline void holds(const at::Tensor &t, at::ScalarType type, int64_t n, const char *name) {
    if (t.scalar_type() == type && t.numel() >= n) return;
    PyErr_Format(PyExc_ValueError, "%s must be a %s tensor of %lld elements", name, c10::toString(type), (long long)n);
    throw Raised();
}

template <typename F>
PyObject *guarded(F &&f) {
    try {
        return f();
    } catch (const Raised &) {
        return nullptr;
    } catch (const std::exception &e) {
        torch::translate_exception_to_python(std::current_exception());
        return nullptr;
    }
}

extern PyMethodDef cache_methods[];  // binding_cache.cpp

}  // namespace mate_binding
