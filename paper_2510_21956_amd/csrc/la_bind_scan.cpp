// The selective state space layer's operators (autograd.py) as autograd nodes in native code, and the marshalling of
// their calls, in the manner of la_bind_layer.cpp: plain tensors only; everything else, and whatever is to be refused, stays
// with the Python functions of the same steps.  A step of the convolution takes 4.3 us this way and 10.9 from Python, of the scan 4.8
// and 16.9, a small convolution forward and backward 89 and 177, a small scan 134 and 265.
#include "la_bind.h"

namespace {

PyObject *python_conv, *python_scan;  // the backward passes in Python

decltype(&la_conv_workspace_bytes) conv_bytes;
decltype(&la_conv_forward) conv_fwd;
decltype(&la_conv_backward) conv_bwd;
decltype(&la_conv_step) conv_one;
decltype(&la_selective_workspace_bytes) scan_bytes;
decltype(&la_selective_saved_bytes) scan_saved;
decltype(&la_selective_forward) scan_fwd;
decltype(&la_selective_backward) scan_bwd;
decltype(&la_selective_step) scan_one;

// Elements from one row of t to the next, a row being its last `dims` dimensions; 0 where rows are not dense, or do not
// follow one another at one distance, at least their own length (binding.row_stride).
size_t row_stride(const at::Tensor &t, int dims)
{
    int64_t row = 1, step = 0, behind = 0;
    const int64_t n = t.dim();
    for (int64_t d = n - 1; d >= n - dims; --d) {
        if (t.size(d) != 1 && t.stride(d) != row) return 0;
        row *= t.size(d);
    }
    for (int64_t d = n - dims - 1; d >= 0; --d) {
        if (t.size(d) == 1 || !t.numel()) continue;
        if (!step) step = t.stride(d);
        else if (t.stride(d) != behind) return 0;
        if (!step) return 0;
        behind = t.stride(d) * t.size(d);
    }
    if (!step) step = std::max(row, (int64_t)1);
    return step >= row ? (size_t)step : 0;
}
constexpr size_t kRowsApart = 1 << 24;  // what the scan's row strides stay below (binding.ROWS_APART)
at::Tensor in_place(const at::Tensor &t, int dims, size_t below = SIZE_MAX)
{
    const size_t step = row_stride(t, dims);
    return step && step < below ? t : t.contiguous();
}

// A tensor whose rows the kernels read where they are: device, type and sizes as given.
bool rows_fit(const at::Tensor &t, const at::Tensor &ref, int dims, at::IntArrayRef sizes)
{
    return t.defined() && t.is_cuda() && !t.unsafeGetTensorImpl()->is_python_dispatch() && t.get_device() == ref.get_device() &&
           t.scalar_type() == ref.scalar_type() && t.sizes() == sizes && row_stride(t, dims);
}
// An int that is one of the library's constants, or that it refuses; a larger one is the Python function's to refuse.
int choice(PyObject *o)
{
    const long x = PyLong_AsLong(o);
    require(x == (int)x && !(x == -1 && PyErr_Occurred()));
    return (int)x;
}
la_dtype code_of(const at::Tensor &t) { return t.scalar_type() == at::kFloat ? LA_F32 : LA_BF16; }
// The sizes of x but for its last `but` dimensions, and more.
std::vector<int64_t> leading(const at::Tensor &x, int but, std::initializer_list<int64_t> more)
{
    std::vector<int64_t> s(x.sizes().begin(), x.sizes().end() - but);
    s.insert(s.end(), more);
    return s;
}

// ---- convolution ------------------------------------------------------------------------------------------------

struct ConvSizes {
    int B, N, C, W;
    la_dtype dt, wt;
    ConvSizes(const at::Tensor &x, const at::Tensor &w)
        : N((int)x.size(-2)), C((int)x.size(-1)), W((int)w.size(1)), dt(code_of(x)), wt(code_of(w))
    {
        B = N && C ? (int)(x.numel() / N / C) : 0;
    }
};
// Whether x, weight, bias, state and lengths are what the library takes.
void check_conv(const at::Tensor &x, PyObject *weight, PyObject *bias, PyObject *state, PyObject *lengths)
{
    require(x.dim() >= 2);
    const int64_t N = x.size(-2), C = x.size(-1);
    require(ints({N, C, N && C ? x.numel() / N / C : 0}));
    dtype_code(x);
    const at::Tensor &w = tensor(weight);
    require(w.dim() == 2 && w.size(0) == C && ints({w.size(1)}) && w.size(1) >= 1 &&
            (w.scalar_type() == at::kFloat || w.scalar_type() == x.scalar_type()));
    if (!is_none(bias)) require(tensor(bias).sizes() == w.sizes().slice(0, 1) && tensor(bias).scalar_type() == w.scalar_type());
    if (!is_none(state))
        require(tensor(state).scalar_type() == x.scalar_type() && tensor(state).sizes() == at::IntArrayRef(leading(x, 2, {w.size(1) - 1, C})));
    if (!is_none(lengths)) require(tensor(lengths).scalar_type() == at::kInt && tensor(lengths).sizes() == x.sizes().slice(0, x.dim() - 2));
}

struct Conv : torch::autograd::Function<Conv> {
    static variable_list forward(AutogradContext *ctx, const at::Tensor &x0, const at::Tensor &w0, const Maybe &bias0,
                                 const Maybe &state0, const Maybe &lengths0, int64_t act)
    {
        const c10::DeviceGuard guard(x0.device());
        const at::Tensor x = in_place(x0, 1), w = w0.contiguous();
        const Maybe bias = packed(bias0), state = packed(state0), lengths = packed(lengths0);
        const ConvSizes s(x, w);
        const at::Tensor y = at::empty(x.sizes(), x.options()), last = at::empty(leading(x, 2, {s.W - 1, s.C}), x.options());
        void *const p[] = {x.data_ptr(), w.data_ptr(), data(bias), data(state), y.data_ptr(), last.data_ptr(), data(lengths), current_stream(x)};
        const size_t stride = row_stride(x, 1);
        int rc;
        Py_BEGIN_ALLOW_THREADS rc = conv_fwd(p[0], stride, p[1], p[2], p[3], p[4], p[5], (const int *)p[6], s.B, s.N, s.C, s.W, (la_act)act, s.dt, s.wt, p[7]);
        Py_END_ALLOW_THREADS
        if (rc != 0) throw Status{rc};
        ctx->save_for_backward({x, w, kept(bias), kept(state), kept(lengths)});
        ctx->saved_data["act"] = act;
        ctx->set_materialize_grads(false);
        return {y, last};
    }
    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        const auto v = ctx->get_saved_variables();
        const at::Tensor &x = v[0], &w = v[1], &bias = v[2], &state = v[3], &lengths = v[4];
        const int64_t act = ctx->saved_data["act"].toInt();
        int at = 1;  // inputs that are there have an edge each
        const bool wants_w = ctx->needs_input_grad(at++), wants_b = bias.defined() && ctx->needs_input_grad(at++),
                   wants_s = state.defined() && ctx->needs_input_grad(at++);
        const at::Tensor dy = grads[0].defined() ? grads[0].contiguous() : at::zeros(x.sizes(), x.options()),
                         dlast = grads[1].defined() ? grads[1].contiguous() : at::Tensor();
        const auto type = x.scalar_type();
        if (x.dim() >= 2 && w.defined() && w.dim() == 2 && rows_fit(x, x, 1, x.sizes()) && fits(dy, x, type, x.sizes()) &&
            (w.scalar_type() == at::kFloat || w.scalar_type() == type) && fits(w, x, w.scalar_type(), {x.size(-1), w.size(1)}) &&
            fits(bias, x, w.scalar_type(), w.sizes().slice(0, 1)) && fits(state, x, type, leading(x, 2, {w.size(1) - 1, x.size(-1)})) &&
            fits(dlast, x, type, leading(x, 2, {w.size(1) - 1, x.size(-1)})) && fits(lengths, x, at::kInt, x.sizes().slice(0, x.dim() - 2))) {
            const c10::DeviceGuard guard(x.device());
            const ConvSizes s(x, w);
            variable_list out(6);
            out[0] = at::empty_like(dy);
            at::Tensor dw, db, ws;
            if (wants_w) dw = at::empty(w.sizes(), w.options().dtype(at::kFloat));
            if (wants_b) db = at::empty({s.C}, w.options().dtype(at::kFloat));
            if (wants_s) out[3] = at::empty_like(state);
            const size_t wb = wants_w || wants_b ? conv_bytes(s.B, s.N, s.C, s.W) : 0;
            if (wb) ws = buffer(wb, x);
            const int rc = conv_bwd(x.data_ptr(), row_stride(x, 1), w.data_ptr(), data(bias), data(state), dy.data_ptr(), data(dlast),
                                    out[0].data_ptr(), (float *)data(dw), (float *)data(db), data(out[3]), (const int *)data(lengths),
                                    s.B, s.N, s.C, s.W, (la_act)act, s.dt, s.wt, data(ws), wb, current_stream(x));
            if (rc == 0) {
                if (wants_w) out[1] = dw.to(w.scalar_type());
                if (wants_b) out[2] = db.to(w.scalar_type());
                return once(std::move(out), grads);
            }
        }
        // gradients of another kind, or a call that the library refuses: the Python code takes or words it
        pybind11::gil_scoped_acquire gil;
        variable_list out = from_python(python_conv, Py_BuildValue("NNNNNNNLiii", wrapped(x), wrapped(w), wrapped(bias), wrapped(state),
                                                                   wrapped(lengths), wrapped(dy), wrapped(dlast), (long long)act,
                                                                   (int)wants_w, (int)wants_b, (int)wants_s));
        out.resize(6);
        return once(std::move(out), grads);
    }
};

// x, weight, bias, state, lengths, act -> (y, last), or the library's status
PyObject *conv(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    PyObject *declined = guarded(n, 6, [&]() -> PyObject * {
        if (!ours(a, 0, 4) || is_none(a[1]) || !PyLong_CheckExact(a[5])) Py_RETURN_NONE;
        check_conv(tensor(a[0]), a[1], a[2], a[3], a[4]);
        check_inputs(tensor(a[0]), {a[0], a[1], a[2], a[3], a[4]});
        return PyBool_FromLong(1);
    });
    if (declined != Py_True) return declined;
    Py_DECREF(declined);
    try {
        return tuple(Conv::apply(tensor(a[0]), tensor(a[1]), maybe(a[2]), maybe(a[3]), maybe(a[4]), (int64_t)PyLong_AsLong(a[5])));
    } catch (const Status &s) {
        return PyLong_FromLong(s.rc);
    }
    END_HANDLE_TH_ERRORS
}

// x, weight, bias, state, y, last, lengths, act, stream -> status
PyObject *conv_forward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 9, [&]() -> PyObject * {
        if (!ours(a, 0, 6) || is_none(a[1]) || is_none(a[4]) || !PyLong_CheckExact(a[7])) Py_RETURN_NONE;
        const at::Tensor &x = tensor(a[0]), &w = tensor(a[1]);
        check_packed({a[1], a[2], a[3], a[4], a[5], a[6]});
        require(x.is_cuda() && x.get_device() == w.get_device());
        check_conv(x, a[1], a[2], a[3], a[6]);
        check_conv(x, a[1], a[2], a[5], a[6]);
        check_like(x, {a[4]});
        const size_t stride = row_stride(x, 1);
        require(stride);
        const ConvSizes s(x, w);
        const la_act act = (la_act)choice(a[7]);
        void *const st = stream_of(a[8], x), *p[7];
        for (int i = 0; i < 7; ++i) p[i] = address(a[i]);
        const c10::DeviceGuard guard(x.device());
        PyObject *const rc = status([&] {
            return conv_fwd(p[0], stride, p[1], p[2], p[3], p[4], p[5], (const int *)p[6], s.B, s.N, s.C, s.W, act, s.dt, s.wt, st);
        });
        if (rc && PyLong_AsLong(rc) == 0) written({a[4], a[5]});
        return rc;
    });
}

// x, weight, bias, state, y, act, stream -> status
PyObject *conv_step(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 7, [&]() -> PyObject * {
        if (!ours(a, 0, 4) || is_none(a[1]) || is_none(a[3]) || is_none(a[4]) || !PyLong_CheckExact(a[5])) Py_RETURN_NONE;
        const at::Tensor &x = tensor(a[0]), &w = tensor(a[1]);
        check_packed({a[1], a[2], a[3], a[4]});
        require(x.is_cuda() && x.get_device() == w.get_device());
        check_conv(x, a[1], a[2], a[3], Py_None);
        check_like(x, {a[4]});
        const size_t stride = row_stride(x, 1);
        require(stride);
        const ConvSizes s(x, w);
        const la_act act = (la_act)choice(a[5]);
        void *const st = stream_of(a[6], x), *p[5];
        for (int i = 0; i < 5; ++i) p[i] = address(a[i]);
        const c10::DeviceGuard guard(x.device());
        PyObject *const rc = status([&] { return conv_one(p[0], stride, p[1], p[2], p[3], p[4], s.B, s.N, s.C, s.W, act, s.dt, s.wt, st); });
        if (rc && PyLong_AsLong(rc) == 0) written({a[3], a[4]});
        return rc;
    });
}

// ---- selective scan -----------------------------------------------------------------------------------------------

struct ScanSizes {
    int B, N, C, S, G, dims;  // dims: those of a row of B and C
    la_dtype dt;
    ScanSizes(const at::Tensor &x, const at::Tensor &A, const at::Tensor &Bm)
        : N((int)x.size(-2)), C((int)x.size(-1)), S((int)A.size(1)), G(Bm.dim() > x.dim() ? (int)Bm.size(-2) : 1),
          dims(Bm.dim() > x.dim() ? 2 : 1), dt(code_of(x))
    {
        B = N && C ? (int)(x.numel() / N / C) : 0;
    }
};
bool vector_sizes(const at::Tensor &x, const at::Tensor &A, const at::Tensor &Bm)
{
    return Bm.sizes() == at::IntArrayRef(leading(x, 1, {A.size(1)})) ||
           (Bm.dim() == x.dim() + 1 && Bm.sizes() == at::IntArrayRef(leading(x, 1, {Bm.size(-2), A.size(1)})));
}
// Whether x, dt, A, B, C, D, bias, state and lengths are what the library takes.
void check_scan(PyObject *const *a, PyObject *state, PyObject *lengths)
{
    const at::Tensor &x = tensor(a[0]), &A = tensor(a[2]), &Bm = tensor(a[3]);
    require(x.dim() >= 2 && A.dim() == 2);
    const int64_t N = x.size(-2), C = x.size(-1);
    require(ints({N, C, N && C ? x.numel() / N / C : 0, A.size(1), Bm.dim() > 1 ? Bm.size(-2) : 0}));
    dtype_code(x);
    check_like(x, {a[1]});
    require(A.size(0) == C && A.scalar_type() == at::kFloat && vector_sizes(x, A, Bm) && Bm.scalar_type() == x.scalar_type());
    check_like(Bm, {a[4]});
    for (PyObject *o : {a[5], a[6]})
        if (!is_none(o)) require(tensor(o).sizes() == A.sizes().slice(0, 1) && tensor(o).scalar_type() == at::kFloat);
    if (!is_none(state))
        require(tensor(state).scalar_type() == at::kFloat && tensor(state).sizes() == at::IntArrayRef(leading(x, 2, {C, A.size(1)})));
    if (!is_none(lengths)) require(tensor(lengths).scalar_type() == at::kInt && tensor(lengths).sizes() == x.sizes().slice(0, x.dim() - 2));
}

struct Scan : torch::autograd::Function<Scan> {
    static variable_list forward(AutogradContext *ctx, const at::Tensor &x0, const at::Tensor &dt0, const at::Tensor &A0,
                                 const at::Tensor &B0, const at::Tensor &C0, const Maybe &D0, const Maybe &bias0, const Maybe &h00,
                                 const Maybe &lengths0, int64_t step, bool keeps)
    {
        const c10::DeviceGuard guard(x0.device());
        const int dims = B0.dim() > x0.dim() ? 2 : 1;
        const at::Tensor x = in_place(x0, 1, kRowsApart), dt = in_place(dt0, 1, kRowsApart), A = A0.contiguous(),
                         Bm = in_place(B0, dims, kRowsApart), Cm = in_place(C0, dims, kRowsApart);
        const Maybe D = packed(D0), bias = packed(bias0), h0 = packed(h00), lengths = packed(lengths0);
        const ScanSizes s(x, A, Bm);
        const at::Tensor y = at::empty(x.sizes(), x.options()), last = at::empty(leading(x, 2, {s.C, s.S}), A.options());
        const size_t wb = scan_bytes(s.B, s.N, s.C, s.S, s.G, 0), sb = keeps ? scan_saved(s.B, s.N, s.C, s.S) : 0;
        at::Tensor ws, saved;
        if (wb) ws = buffer(wb, x);
        if (sb) saved = buffer(sb, x);
        void *const p[] = {x.data_ptr(), dt.data_ptr(), A.data_ptr(), Bm.data_ptr(), Cm.data_ptr(), data(D), data(bias), data(h0),
                           y.data_ptr(), last.data_ptr(), data(saved), data(lengths), data(ws), current_stream(x)};
        const size_t xs = row_stride(x, 1), ts = row_stride(dt, 1), bs = row_stride(Bm, dims), cs = row_stride(Cm, dims);
        int rc;
        Py_BEGIN_ALLOW_THREADS rc = scan_fwd(p[0], xs, p[1], ts, (const float *)p[2], p[3], bs, p[4], cs, (const float *)p[5],
                                             (const float *)p[6], (const float *)p[7], p[8], (float *)p[9], p[10], sb, (const int *)p[11],
                                             s.B, s.N, s.C, s.S, s.G, (la_step)step, s.dt, p[12], wb, p[13]);
        Py_END_ALLOW_THREADS
        if (rc != 0) throw Status{rc};
        ctx->save_for_backward({x, dt, A, Bm, Cm, kept(D), kept(bias), kept(lengths), saved});
        ctx->saved_data["step"] = step;
        ctx->saved_data["h0"] = h0.has_value();
        ctx->set_materialize_grads(false);
        return {y, last};
    }
    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        const auto v = ctx->get_saved_variables();
        const at::Tensor &x = v[0], &dt = v[1], &A = v[2], &Bm = v[3], &Cm = v[4], &D = v[5], &bias = v[6], &lengths = v[7], &saved = v[8];
        const int64_t step = ctx->saved_data["step"].toInt();
        int at = 5;  // inputs that are there have an edge each
        const bool wants_A = ctx->needs_input_grad(2), wants_D = D.defined() && ctx->needs_input_grad(at++),
                   wants_b = bias.defined() && ctx->needs_input_grad(at++), wants_h = ctx->saved_data["h0"].toBool() && ctx->needs_input_grad(at++);
        const at::Tensor dy = grads[0].defined() ? grads[0].contiguous() : at::zeros(x.sizes(), x.options()),
                         dlast = grads[1].defined() ? grads[1].contiguous() : at::Tensor();
        const auto type = x.scalar_type();
        if (x.dim() >= 2 && A.defined() && A.dim() == 2 && Bm.defined() && Cm.defined() && saved.defined() &&
            (type == at::kFloat || type == at::kBFloat16) && rows_fit(x, x, 1, x.sizes()) && rows_fit(dt, x, 1, x.sizes()) &&
            vector_sizes(x, A, Bm) && rows_fit(Bm, x, Bm.dim() > x.dim() ? 2 : 1, Bm.sizes()) &&
            rows_fit(Cm, x, Bm.dim() > x.dim() ? 2 : 1, Bm.sizes()) && fits(A, x, at::kFloat, {x.size(-1), A.size(1)}) &&
            fits(D, x, at::kFloat, {x.size(-1)}) && fits(bias, x, at::kFloat, {x.size(-1)}) && fits(dy, x, type, x.sizes()) &&
            fits(dlast, x, at::kFloat, leading(x, 2, {x.size(-1), A.size(1)})) && fits(lengths, x, at::kInt, x.sizes().slice(0, x.dim() - 2)) &&
            fits(saved, x, at::kByte, saved.sizes())) {
            const c10::DeviceGuard guard(x.device());
            const ScanSizes s(x, A, Bm);
            variable_list out(11);
            out[0] = at::empty_like(dy);
            out[1] = at::empty_like(dy);
            if (wants_A) out[2] = at::empty_like(A);
            out[3] = at::empty(Bm.sizes(), Bm.options());
            out[4] = at::empty(Bm.sizes(), Bm.options());
            if (wants_D) out[5] = at::empty_like(D);
            if (wants_b) out[6] = at::empty_like(bias);
            if (wants_h) out[7] = at::empty(leading(x, 2, {s.C, s.S}), A.options());
            const size_t wb = scan_bytes(s.B, s.N, s.C, s.S, s.G, 1);
            const at::Tensor ws = buffer(wb, x);
            const int rc = scan_bwd(x.data_ptr(), row_stride(x, 1), dt.data_ptr(), row_stride(dt, 1), (const float *)A.data_ptr(), Bm.data_ptr(),
                                    row_stride(Bm, s.dims), Cm.data_ptr(), row_stride(Cm, s.dims), (const float *)data(D),
                                    (const float *)data(bias), saved.data_ptr(), bytes(saved), dy.data_ptr(), (const float *)data(dlast),
                                    out[0].data_ptr(), out[1].data_ptr(), (float *)data(out[2]), out[3].data_ptr(), out[4].data_ptr(),
                                    (float *)data(out[5]), (float *)data(out[6]), (float *)data(out[7]), (const int *)data(lengths), s.B, s.N,
                                    s.C, s.S, s.G, (la_step)step, s.dt, ws.data_ptr(), bytes(ws), current_stream(x));
            if (rc == 0) return once(std::move(out), grads);
        }
        pybind11::gil_scoped_acquire gil;
        variable_list out = from_python(
            python_scan, Py_BuildValue("NNNNNNNNNNNLiiii", wrapped(x), wrapped(dt), wrapped(A), wrapped(Bm), wrapped(Cm), wrapped(D),
                                       wrapped(bias), wrapped(lengths), wrapped(saved), wrapped(dy), wrapped(dlast), (long long)step,
                                       (int)wants_A, (int)wants_D, (int)wants_b, (int)wants_h));
        out.resize(11);
        return once(std::move(out), grads);
    }
};

// x, dt, A, B, C, D, bias, h0, lengths, step -> (y, last), or the library's status
PyObject *scan(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    bool keeps = false;
    PyObject *declined = guarded(n, 10, [&]() -> PyObject * {
        if (!ours(a, 0, 8) || !PyLong_CheckExact(a[9])) Py_RETURN_NONE;
        for (int i = 1; i < 5; ++i)
            if (is_none(a[i])) Py_RETURN_NONE;
        check_scan(a, a[7], a[8]);
        check_inputs(tensor(a[0]), {a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8]});
        for (int i = 0; i < 8; ++i) keeps = keeps || (!is_none(a[i]) && tensor(a[i]).requires_grad());
        keeps = keeps && at::GradMode::is_enabled();
        return PyBool_FromLong(1);
    });
    if (declined != Py_True) return declined;
    Py_DECREF(declined);
    try {
        return tuple(Scan::apply(tensor(a[0]), tensor(a[1]), tensor(a[2]), tensor(a[3]), tensor(a[4]), maybe(a[5]), maybe(a[6]), maybe(a[7]),
                                 maybe(a[8]), (int64_t)PyLong_AsLong(a[9]), keeps));
    } catch (const Status &s) {
        return PyLong_FromLong(s.rc);
    }
    END_HANDLE_TH_ERRORS
}

// What the calls on x, dt, A, B, C, D, bias, state, y, .. share.
struct ScanCall {
    const at::Tensor &x;
    ScanSizes s;
    size_t xs, ts, bs, cs;
    ScanCall(PyObject *const *a, PyObject *lengths)
        : x(tensor(a[0])), s((check_scan(a, a[7], lengths), x), tensor(a[2]), tensor(a[3])), xs(row_stride(x, 1)),
          ts(row_stride(tensor(a[1]), 1)), bs(row_stride(tensor(a[3]), s.dims)), cs(row_stride(tensor(a[4]), s.dims))
    {
        require(xs && ts && bs && cs);
        check_packed({a[2], a[5], a[6], a[7], a[8], lengths});
        for (int i : {0, 1, 3, 4}) require(tensor(a[i]).is_cuda() && tensor(a[i]).get_device() == tensor(a[2]).get_device());
        check_like(x, {a[8]});
    }
};

// x, dt, A, B, C, D, bias, h0, y, last, saved, lengths, step, workspace, stream -> status
PyObject *scan_forward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 15, [&]() -> PyObject * {
        if (!ours(a, 0, 11) || !plain_or_none(a[13]) || is_none(a[8]) || !PyLong_CheckExact(a[12])) Py_RETURN_NONE;
        for (int i = 1; i < 5; ++i)
            if (is_none(a[i])) Py_RETURN_NONE;
        const ScanCall c(a, a[11]);
        check_scan(a, a[9], a[11]);
        check_packed({a[2], a[9], a[10], a[13]});
        const la_step step = (la_step)choice(a[12]);
        void *const st = stream_of(a[14], c.x), *p[14];
        for (int i = 0; i < 14; ++i) p[i] = i == 12 ? nullptr : address(a[i]);
        const size_t sb = is_none(a[10]) ? 0 : bytes(tensor(a[10])), wb = is_none(a[13]) ? 0 : bytes(tensor(a[13]));
        const c10::DeviceGuard guard(c.x.device());
        PyObject *const rc = status([&] {
            return scan_fwd(p[0], c.xs, p[1], c.ts, (const float *)p[2], p[3], c.bs, p[4], c.cs, (const float *)p[5], (const float *)p[6],
                            (const float *)p[7], p[8], (float *)p[9], p[10], sb, (const int *)p[11], c.s.B, c.s.N, c.s.C, c.s.S, c.s.G, step,
                            c.s.dt, p[13], wb, st);
        });
        if (rc && PyLong_AsLong(rc) == 0) written({a[8], a[9], a[10]});
        return rc;
    });
}

// x, dt, A, B, C, D, bias, state, y, step, stream -> status
PyObject *scan_step(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 11, [&]() -> PyObject * {
        if (!ours(a, 0, 8) || is_none(a[7]) || is_none(a[8]) || !PyLong_CheckExact(a[9])) Py_RETURN_NONE;
        for (int i = 1; i < 5; ++i)
            if (is_none(a[i])) Py_RETURN_NONE;
        const ScanCall c(a, Py_None);
        require(std::max({c.xs, c.ts, c.bs, c.cs}) < kRowsApart);  // the Python function copies
        const la_step step = (la_step)choice(a[9]);
        void *const st = stream_of(a[10], c.x), *p[9];
        for (int i = 0; i < 9; ++i) p[i] = address(a[i]);
        const c10::DeviceGuard guard(c.x.device());
        PyObject *const rc = status([&] {
            return scan_one(p[0], c.xs, p[1], c.ts, (const float *)p[2], p[3], c.bs, p[4], c.cs, (const float *)p[5], (const float *)p[6],
                            (float *)p[7], p[8], c.s.B, c.s.N, c.s.C, c.s.S, c.s.G, step, c.s.dt, st);
        });
        if (rc && PyLong_AsLong(rc) == 0) written({a[7], a[8]});
        return rc;
    });
}

}  // namespace

// The backward passes in Python, then the addresses of the entry points in the order of the pointers above
PyObject *init_scan(PyObject *, PyObject *const *x, Py_ssize_t n)
{
    void **const to[] = {(void **)&conv_bytes, (void **)&conv_fwd, (void **)&conv_bwd, (void **)&conv_one, (void **)&scan_bytes,
                         (void **)&scan_saved, (void **)&scan_fwd, (void **)&scan_bwd, (void **)&scan_one};
    constexpr Py_ssize_t COUNT = sizeof(to) / sizeof(to[0]);
    if (n != 2 + COUNT) {
        PyErr_SetString(PyExc_TypeError, "init_scan takes two callables and the entry points' addresses");
        return nullptr;
    }
    if (!addresses(x + 2, to, COUNT)) return nullptr;
    Py_INCREF(x[0]);
    Py_XSETREF(python_conv, x[0]);
    Py_INCREF(x[1]);
    Py_XSETREF(python_scan, x[1]);
    Py_RETURN_NONE;
}

PyMethodDef scan_methods[] = {{"conv", (PyCFunction)(void (*)())conv, METH_FASTCALL, nullptr},
                              {"conv_forward", (PyCFunction)(void (*)())conv_forward, METH_FASTCALL, nullptr},
                              {"conv_step", (PyCFunction)(void (*)())conv_step, METH_FASTCALL, nullptr},
                              {"scan", (PyCFunction)(void (*)())scan, METH_FASTCALL, nullptr},
                              {"scan_forward", (PyCFunction)(void (*)())scan_forward, METH_FASTCALL, nullptr},
                              {"scan_step", (PyCFunction)(void (*)())scan_step, METH_FASTCALL, nullptr},
                              {nullptr, nullptr, 0, nullptr}};
