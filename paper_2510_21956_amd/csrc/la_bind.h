// What the native parts of the Python binding share: checks and conversions of their arguments.
#pragma once

#include <ATen/FuncTorchTLS.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/functions/utils.h>
#include <torch/csrc/autograd/python_cpp_function.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/jit/frontend/tracer.h>

#include "la.h"

extern PyObject *raw_stream;  // device index -> stream handle of its current stream (la_bind.cpp)
PyObject *init_layer(PyObject *, PyObject *const *x, Py_ssize_t n);  // la_bind_layer.cpp
extern PyMethodDef layer_methods[];
PyObject *init_scan(PyObject *, PyObject *const *x, Py_ssize_t n);  // la_bind_scan.cpp
extern PyMethodDef scan_methods[];

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

// ---- what the autograd nodes of the operators around the attention share ----------------------------------------

using torch::autograd::AutogradContext;
using torch::autograd::variable_list;
typedef std::optional<at::Tensor> Maybe;

inline void *data(const at::Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }
inline void *data(const Maybe &t) { return t ? t->data_ptr() : nullptr; }
inline Maybe maybe(PyObject *o) { return is_none(o) ? Maybe() : Maybe(tensor(o)); }
inline Maybe packed(const Maybe &t) { return t ? Maybe(t->contiguous()) : t; }
inline at::Tensor kept(const Maybe &t) { return t ? *t : at::Tensor(); }

// A tensor as the kernels take it, like ref (device, type and, where given, sizes).
inline bool fits(const at::Tensor &t, const at::Tensor &ref, at::ScalarType type, at::IntArrayRef sizes)
{
    return !t.defined() || (t.is_cuda() && t.is_contiguous() && !t.unsafeGetTensorImpl()->is_python_dispatch() &&
                            t.get_device() == ref.get_device() && t.scalar_type() == type && t.sizes() == sizes);
}

// Gradients of gradients are not defined: where a graph of the backward pass is asked for, its results come out of a node
// that refuses, tied to all that they depend on (the operator's inputs and the incoming gradients), so that no
// derivative goes past it.
inline variable_list once(variable_list out, const variable_list &grads)
{
    using namespace torch::autograd;
    if (!at::GradMode::is_enabled()) return out;
    edge_list edges = collect_next_edges(grads);
    if (const auto node = get_current_node()) edges.insert(edges.end(), node->next_edges().begin(), node->next_edges().end());
    const auto refuse =
        std::make_shared<Error>("gradients of gradients are not defined for this operator", std::move(edges));
    for (at::Tensor &t : out)
        if (t.defined()) set_history(t = t.detach(), refuse);
    return out;
}

// Calls a backward pass in Python with `args` (a tuple, taken); its results, None where there is none.
inline variable_list from_python(PyObject *f, PyObject *args)
{
    PyObject *got = args ? PyObject_CallObject(f, args) : nullptr;
    Py_XDECREF(args);
    if (!got) {
        python_error e;
        e.persist();
        throw e;
    }
    variable_list out;
    for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(got); ++i) {
        PyObject *o = PyTuple_GET_ITEM(got, i);
        out.push_back(is_none(o) ? at::Tensor() : tensor(o));
    }
    Py_DECREF(got);
    return out;
}
inline PyObject *wrapped(const at::Tensor &t)
{
    if (t.defined()) return THPVariable_Wrap(t);
    Py_RETURN_NONE;
}
inline PyObject *tuple(const variable_list &ts)
{
    PyObject *out = PyTuple_New((Py_ssize_t)ts.size());
    for (size_t i = 0; out && i < ts.size(); ++i) PyTuple_SET_ITEM(out, (Py_ssize_t)i, wrapped(ts[i]));
    return out;
}

// Sizes that are the library's ints.
inline bool ints(std::initializer_list<int64_t> sizes)
{
    return std::max(sizes) < (int64_t)1 << 31;
}


// What a call has written: a node that saved it must not go on with the new values.
inline void written(std::initializer_list<PyObject *> ts)
{
    for (PyObject *o : ts)
        if (!is_none(o) && !tensor(o).is_inference()) tensor(o).unsafeGetTensorImpl()->bump_version();
}
// Takes the entry points' addresses x[0 .. n - 1].
inline bool addresses(PyObject *const *x, void **const *to, Py_ssize_t n)
{
    for (Py_ssize_t i = 0; i < n; ++i) {
        *to[i] = PyLong_AsVoidPtr(x[i]);
        if (!*to[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null address");
            return false;
        }
    }
    return true;
}

}  // namespace
