// What the calls of the extension module share (host.cpp, host_kv.cpp, host_layer.cpp): how a Python object becomes memory and sizes, how new tensors
// are made, how a status becomes a result or an error.
#pragma once

#include <ATen/ATen.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/mxfp4.h"

namespace mxfp4_host {

inline PyObject* g_failed = nullptr;                // raises the error of a status code

// A tensor whose memory and sizes are what they say: exactly torch.Tensor (or Parameter) and no transform, mode or lazy bit.
inline const at::Tensor* plain(PyObject* o, at::ScalarType type, c10::Device device)
{
    static const uint64_t allowed =
        c10::DispatchKeySet({c10::DispatchKey::CUDA, c10::DispatchKey::AutogradCUDA, c10::DispatchKey::ADInplaceOrView,
                             c10::DispatchKey::AutocastCUDA}).raw_repr();
    if (!THPVariable_CheckExact(o))
        return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.defined() || (t.key_set().raw_repr() & ~allowed) != 0 || t.scalar_type() != type || t.device() != device ||
        !t.has_storage())
        return nullptr;
    return &t;
}

// A new tensor on the device: from the allocator behind torch.empty, without the way through the dispatcher, unless something on this
// thread wants to see it there (a transform; autocast and the keys that every thread has do not).  One row of
// 4096 x 4096, which the host bounds: 4.35 -> 4.17 us from call to call.
inline at::Tensor fresh(at::IntArrayRef size, at::ScalarType type, c10::Device device)
{
    static const uint64_t usual = (c10::default_included_set | c10::autocast_dispatch_keyset).raw_repr();
    if ((c10::impl::tls_local_dispatch_key_set().included_.raw_repr() & ~usual) != 0)
        return at::empty(size, at::TensorOptions().dtype(type).device(device));
    return at::Tensor(at::detail::empty_cuda(size, type, device, std::nullopt));
}

// What the binding's own checks take over: also a number that is none or too large, whose error they raise in their words.
inline PyObject* left()
{
    PyErr_Clear();
    Py_RETURN_NONE;
}

inline bool small(PyObject* o, int* v)                     // an int of the C interface as it stands
{
    int over = 0;
    const long long wide = PyLong_Check(o) ? PyLong_AsLongLongAndOverflow(o, &over) : 0;
    *v = (int)wide;
    return PyLong_Check(o) && over == 0 && wide == *v;
}

inline PyObject* finish(int rc, PyObject* (*wrap)(const at::Tensor*), const at::Tensor* out)
{
    if (rc == 0)
        return wrap(out);
    PyObject* raised = PyObject_CallFunction(g_failed, "i", rc);
    Py_XDECREF(raised);
    if (!PyErr_Occurred())
        PyErr_SetString(PyExc_RuntimeError, "mxfp4: status without an error");
    return nullptr;
}

inline PyObject* wrap_one(const at::Tensor* t) { return THPVariable_Wrap(t[0]); }

inline PyObject* wrap_list(const at::Tensor* t, int count)
{
    PyObject* tuple = PyTuple_New(count);
    for (int i = 0; tuple && i < count; ++i) {
        PyObject* item = THPVariable_Wrap(t[i]);
        if (!item) {
            Py_DECREF(tuple);
            return nullptr;
        }
        PyTuple_SET_ITEM(tuple, i, item);
    }
    return tuple;
}

inline PyObject* wrap_three(const at::Tensor* t) { return wrap_list(t, 3); }
inline PyObject* wrap_two(const at::Tensor* t) { return wrap_list(t, 2); }

// The module's functions that live in host_kv.cpp and host_layer.cpp.
extern PyMethodDef kv_methods[];
extern PyMethodDef layer_methods[];

}  // namespace mxfp4_host
