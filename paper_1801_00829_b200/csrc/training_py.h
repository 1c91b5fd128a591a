// What the parts of the CPython extension share: refusals, types, addresses of tensors, scratch, and how a function is offered to
// Python.
#pragma once

#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <cstring>
#include <map>
#include <string>
#include <utility>
#include <vector>
#include "fusedops_lm.h"

namespace fo_py {

inline PyObject *g_error = nullptr;        // FusedOpsError
inline PyObject *g_workspace = nullptr;    // f(GPU number, bytes) -> tensor: the current stream's scratch

struct Refused : std::exception {
    std::string text;
    explicit Refused(std::string t) : text(std::move(t)) {}
    const char *what() const noexcept override { return text.c_str(); }
};
struct Raised : std::exception {};   // a Python exception is set

inline void require(bool ok, const char *text)
{
    if (!ok) throw Refused(text);
}

inline int type_code(at::ScalarType t)
{
    switch (t) {
    case at::kDouble: return FO_F64;
    case at::kFloat: return FO_F32;
    case at::kBFloat16: return FO_BF16;
    case at::kHalf: return FO_F16;
    default: throw Refused(std::string("no kernel for ") + c10::toString(t));
    }
}

inline const at::Tensor *tensor_of(PyObject *o, const char *name)
{
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) throw Refused(std::string(name) + " is not a tensor");
    const at::Tensor &t = THPVariable_Unpack(o);
    // a view whose values are the negatives of what lies in memory (the imaginary part of a conjugate)
    if (t.is_neg()) throw Refused(std::string(name) + " is a negative view: resolve_neg() it first");
    return &t;
}

inline at::ScalarType dtype_of(PyObject *o, const char *name)
{
    if (!THPDtype_Check(o)) throw Refused(std::string(name) + " is not a dtype");
    return reinterpret_cast<THPDtype *>(o)->scalar_type;
}

// The address of a tensor of which `reach` elements from its first one on are used; its storage may have been resized.
inline void *data_of(const at::Tensor &t, int64_t reach, const char *name)
{
    if (reach <= 0) return nullptr;
    const c10::TensorImpl &impl = *t.unsafeGetTensorImpl();
    c10::StorageImpl &held = *impl.storage().unsafeGetStorageImpl();
    const size_t bytes = impl.dtype().itemsize(), at_byte = (size_t)impl.storage_offset() * bytes;
    if (held.nbytes() < at_byte + (size_t)reach * bytes)
        throw Refused(std::string(name) + ": the tensor's storage is smaller than the tensor");
    return static_cast<char *>(held.mutable_data()) + at_byte;
}

// The operators record no graph: a tensor that autograd follows would lose its gradient without a word.
inline void outside_graph(const at::Tensor &t, const char *name)
{
    if (t.requires_grad() && c10::GradMode::is_enabled())
        throw Refused(std::string(name) + " requires a gradient, and this call records none: call it under torch.no_grad(), or in an "
                                          "autograd.Function whose backward is the operator's gradient call");
}
// `t` was written: what autograd saved of it is no longer what it was.
inline void written(const at::Tensor &t)
{
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

inline bool is(PyObject *o, const char *text) { return PyUnicode_Check(o) && PyUnicode_CompareWithASCIIString(o, text) == 0; }

// Makes GPU `gpu` current for a call if another one is.
struct OnGpu {
    c10::DeviceIndex before;
    explicit OnGpu(c10::DeviceIndex gpu) : before(c10::cuda::current_device())
    {
        if (gpu == before) before = -1;
        else c10::cuda::set_device(gpu);
    }
    ~OnGpu()
    {
        if (before >= 0) c10::cuda::set_device(before);
    }
};

inline void check_status(int status, const char *name)
{
    if (status == FO_OK) return;
    PyObject *args = Py_BuildValue("(is)", status, name);
    PyObject *e = args ? PyObject_CallObject(g_error, args) : nullptr;
    Py_XDECREF(args);
    if (e) {
        PyErr_SetObject(g_error, e);
        Py_DECREF(e);
    }
    throw Raised();
}

inline PyObject *or_none(const at::Tensor &t)
{
    if (t.defined()) return THPVariable_Wrap(t);
    Py_RETURN_NONE;
}

inline at::Tensor new_workspace(c10::DeviceIndex gpu, size_t bytes)
{
    PyObject *o = PyObject_CallFunction(g_workspace, "in", (int)gpu, (Py_ssize_t)bytes);
    if (!o) throw Raised();
    const at::Tensor t = THPVariable_Unpack(o);
    Py_DECREF(o);
    return t;
}
// The stream's scratch; a call that is captured into a graph gets one of its own (binding.workspace).
inline at::Tensor workspace(c10::DeviceIndex gpu, cudaStream_t stream, size_t bytes)
{
    cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
    if (cudaStreamIsCapturing(stream, &capture) != cudaSuccess || capture != cudaStreamCaptureStatusNone)
        return new_workspace(gpu, bytes);
    static auto *cache = new std::map<std::pair<int, cudaStream_t>, at::Tensor>();      // outlives the interpreter
    at::Tensor &buf = (*cache)[{gpu, stream}];
    if (!buf.defined() || (size_t)buf.numel() < bytes) buf = new_workspace(gpu, bytes);
    return buf;
}

inline double number(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (PyErr_Occurred()) throw Raised();
    return v;
}
inline long long whole(PyObject *o)
{
    const long long v = PyLong_AsLongLong(o);
    if (PyErr_Occurred()) throw Raised();
    return v;
}

template <PyObject *(*IMPL)(PyObject *const *), int N>
inline PyObject *guarded(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "%d arguments are needed", N);
        return nullptr;
    }
    try {
        return IMPL(args);
    } catch (const Refused &e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const Raised &) {
    }
    return nullptr;
    END_HANDLE_TH_ERRORS
}
template <PyObject *(*IMPL)(PyObject *const *), int N>
PyMethodDef method(const char *name)
{
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&guarded<IMPL, N>)), METH_FASTCALL, nullptr};
}

}  // namespace fo_py
