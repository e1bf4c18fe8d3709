// What the native parts of the Python binding share: checks and conversions of their arguments.
#pragma once

#include <ATen/FuncTorchTLS.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/python_cpp_function.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/jit/frontend/tracer.h>

#include "la.h"

extern PyObject *raw_stream;  // device index -> stream handle of its current stream (la_bind.cpp)
PyObject *init_layer(PyObject *, PyObject *const *x, Py_ssize_t n);  // la_bind_layer.cpp
extern PyMethodDef layer_methods[];

namespace {

struct Decline {};  // the Python function takes over; a Python exception may be set
inline void require(bool ok)
{
    if (!ok) throw Decline();
}

inline bool is_none(PyObject *o) { return o == Py_None; }
// Tensors and parameters; a subclass may answer is_contiguous, data_ptr and the rest in its own way, which
// the Python functions ask it for.
inline bool plain(PyObject *o) { return THPVariable_CheckExact(o); }
inline bool plain_or_none(PyObject *o) { return is_none(o) || plain(o); }
inline const at::Tensor &tensor(PyObject *o) { return THPVariable_Unpack(o); }
inline void *address(PyObject *o) { return is_none(o) ? nullptr : tensor(o).data_ptr(); }
inline size_t bytes(const at::Tensor &t) { return (size_t)t.numel() * t.element_size(); }

// Packed device tensors, all on one device (None is left out).
inline void check_packed(std::initializer_list<PyObject *> ts)
{
    const at::Tensor &ref = tensor(*ts.begin());
    for (PyObject *o : ts) {
        if (is_none(o)) continue;
        const at::Tensor &t = tensor(o);
        require(t.is_cuda() && t.is_contiguous() && t.get_device() == ref.get_device());
    }
}
inline void check_like(const at::Tensor &ref, std::initializer_list<PyObject *> ts)
{
    for (PyObject *o : ts)
        require(is_none(o) || (tensor(o).sizes() == ref.sizes() && tensor(o).scalar_type() == ref.scalar_type()));
}
inline void check_rows(const at::Tensor &ref, PyObject *g)
{
    if (is_none(g)) return;
    const at::Tensor &t = tensor(g);
    require(t.sizes() == ref.sizes().slice(0, 3) && t.scalar_type() == at::kFloat);
}
inline la_dtype dtype_code(const at::Tensor &t)
{
    require(t.scalar_type() == at::kFloat || t.scalar_type() == at::kBFloat16);
    return t.scalar_type() == at::kFloat ? LA_F32 : LA_BF16;
}
inline double real(PyObject *o)
{
    if (PyFloat_CheckExact(o)) return PyFloat_AS_DOUBLE(o);
    PyObject *f = PyNumber_Float(o);  // what float(o) gives
    require(f);
    const double x = PyFloat_AS_DOUBLE(f);
    Py_DECREF(f);
    return x;
}
inline float number(PyObject *o) { return (float)real(o); }
inline int truth(PyObject *o)
{
    const int x = PyObject_IsTrue(o);
    require(x >= 0);
    return x;
}
inline void *stream_of(PyObject *stream, const at::Tensor &ref)
{
    PyObject *h = is_none(stream) ? PyObject_CallFunction(raw_stream, "i", (int)ref.get_device())
                                  : PyObject_GetAttrString(stream, "cuda_stream");
    require(h);
    void *p = PyLong_AsVoidPtr(h);
    Py_DECREF(h);
    require(p || !PyErr_Occurred());
    return p;
}

// Runs body, which returns the library's status, on n arguments.  None: the Python function takes over.
template <typename Body>
PyObject *guarded(Py_ssize_t given, Py_ssize_t n, Body body)
{
    if (given != n) return PyErr_Format(PyExc_TypeError, "%zd arguments expected", n);
    try {
        return body();
    } catch (const Decline &) {
    } catch (const std::exception &) {
    }
    if (PyErr_Occurred() && !PyErr_ExceptionMatches(PyExc_Exception)) return nullptr;  // an interrupt
    PyErr_Clear();
    Py_RETURN_NONE;
}
template <typename Call>
PyObject *status(Call call)
{
    la_status s;
    Py_BEGIN_ALLOW_THREADS s = call();
    Py_END_ALLOW_THREADS return PyLong_FromLong(s);
}
inline bool ours(PyObject *const *a, int first, int last)
{
    if (!plain(a[first])) return false;
    for (int i = first + 1; i <= last; ++i)
        if (!plain_or_none(a[i])) return false;
    return true;
}

// The inputs of an autograd node in native code: plain tensors of one device, outside of modes, transforms and
// traces, which look for a Python function.  None is left out.
inline void check_inputs(const at::Tensor &ref, std::initializer_list<PyObject *> ts)
{
    for (PyObject *o : ts) {
        if (is_none(o)) continue;
        require(plain(o) && tensor(o).is_cuda() && tensor(o).get_device() == ref.get_device() &&
                !tensor(o)._fw_grad(0).defined());
        tensor(o).const_data_ptr();  // throws where there is no storage
    }
    require(!at::impl::torch_function_mode_enabled() && !c10::impl::TorchDispatchModeTLS::any_modes_set() &&
            !torch::jit::tracer::isTracing());
    if (const auto &transforms = at::functorch::functorchTLSAccessor())
        transforms->checkSupportsCppAutogradFunction();  // throws inside of vmap, grad and the like
}

inline at::Tensor buffer(size_t n, const at::Tensor &ref)
{
    return at::empty({(int64_t)(n < 256 ? 256 : n)}, ref.options().dtype(at::kByte));
}
inline void *current_stream(const at::Tensor &ref) { return c10::hip::getCurrentHIPStream(ref.get_device()).stream(); }

struct Status {  // what the library answered
    int rc;
};

}  // namespace
