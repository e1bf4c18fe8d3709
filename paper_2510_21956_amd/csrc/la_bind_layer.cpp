// The operators around the attention (autograd.py) as autograd nodes in native code, and the marshalling of their
// small calls, in the manner of la_bind.cpp: plain tensors only; everything else, and whatever is to be refused,
// stays with the Python functions of the same steps.  Through Python and here, us, nearly all of it host: rms_norm
// on 5003 rows of 771, fp32, forward and backward 121 and 62; attention with checkpoints on 1 slice of 256 rows,
// D = 16, 235 and 91; rms_norm_quantised on 8 rows 17 and 7.0; a step of a recurrence 8.3 and 4.0.
#include "la_bind.h"

namespace {

PyObject *python_recurrence, *python_norm, *python_checkpointed;  // the backward passes in Python

decltype(&la_recurrence_workspace_bytes) rec_bytes;
decltype(&la_recurrence_forward) rec_forward;
decltype(&la_recurrence_backward) rec_backward;
decltype(&la_recurrence_step) rec_step;
decltype(&la_pack_tensors) pack_tensors;
decltype(&la_unpack_rows) unpack_rows;
decltype(&la_rmsnorm_workspace_bytes) norm_bytes;
decltype(&la_rmsnorm_forward) norm_forward;
decltype(&la_rmsnorm_backward) norm_backward;
decltype(&la_forward_traced) att_forward, att_forward_qknorm;
decltype(&la_forward_save) att_save, att_save_qknorm;
decltype(&la_backward_saved) att_backward, att_backward_qknorm;
decltype(&la_workspace_bytes) att_bytes;
decltype(&la_saved_state_bytes) att_saved_bytes;

// ---- gated recurrence -----------------------------------------------------------------------------------------

struct Sequences {
    int B, N, C;
    la_dtype dt;
    explicit Sequences(const at::Tensor &x)
        : N((int)x.size(-2)), C((int)x.size(-1)), dt(x.scalar_type() == at::kFloat ? LA_F32 : LA_BF16)
    {
        B = N && C ? (int)(x.numel() / N / C) : 0;
    }
};
bool ints_of_sequences(const at::Tensor &x)
{
    const int64_t N = x.size(-2), C = x.size(-1);
    return ints({N, C, N && C ? x.numel() / N / C : 0});
}
std::vector<int64_t> state_sizes(const at::Tensor &x)
{
    std::vector<int64_t> s(x.sizes().begin(), x.sizes().end() - 2);
    s.push_back(x.size(-1));
    return s;
}

struct Recurrence : torch::autograd::Function<Recurrence> {
    static variable_list forward(AutogradContext *ctx, const at::Tensor &x0, const at::Tensor &g0, const Maybe &state0,
                                 const Maybe &lengths0, int64_t gate)
    {
        const c10::DeviceGuard guard(x0.device());
        const at::Tensor x = x0.contiguous(), g = g0.contiguous();
        const Maybe h0 = packed(state0), lengths = packed(lengths0);
        const Sequences s(x);
        const at::Tensor h = at::empty_like(x), last = at::empty(state_sizes(x), x.options().dtype(at::kFloat));
        const size_t wb = rec_bytes(s.B, s.N, s.C, s.dt, 0);
        at::Tensor ws;
        if (wb) ws = buffer(wb, x);
        void *const p[] = {x.data_ptr(), g.data_ptr(), data(h0), h.data_ptr(), last.data_ptr(), data(lengths), data(ws),
                           current_stream(x)};
        int rc;
        Py_BEGIN_ALLOW_THREADS rc = rec_forward(p[0], p[1], (const float *)p[2], p[3], (float *)p[4], (const int *)p[5],
                                                s.B, s.N, s.C, (la_gate)gate, s.dt, p[6], wb, p[7]);
        Py_END_ALLOW_THREADS
        if (rc != 0) throw Status{rc};
        ctx->save_for_backward({x, g, kept(h0), h, kept(lengths)});
        ctx->saved_data["gate"] = gate;
        ctx->set_materialize_grads(false);
        return {h, last};
    }
    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        const auto v = ctx->get_saved_variables();
        const at::Tensor &x = v[0], &g = v[1], &h0 = v[2], &h = v[3], &lengths = v[4];
        const int64_t gate = ctx->saved_data["gate"].toInt();
        const bool wants_h0 = h0.defined() && ctx->needs_input_grad(2);
        const at::Tensor dh = grads[0].defined() ? grads[0].contiguous() : at::zeros_like(x),
                         dlast = grads[1].defined() ? grads[1].contiguous() : at::Tensor();
        const auto type = x.scalar_type();
        if (x.defined() && fits(x, x, type, x.sizes()) && fits(g, x, type, x.sizes()) && fits(h, x, type, x.sizes()) &&
            fits(dh, x, type, x.sizes()) && fits(h0, x, at::kFloat, state_sizes(x)) &&
            fits(dlast, x, at::kFloat, state_sizes(x)) &&
            fits(lengths, x, at::kInt, x.sizes().slice(0, x.dim() - 2))) {
            const c10::DeviceGuard guard(x.device());
            const Sequences s(x);
            variable_list out(5);
            out[0] = at::empty_like(x);
            out[1] = at::empty_like(x);
            if (wants_h0) out[2] = at::empty_like(h0);
            const size_t wb = rec_bytes(s.B, s.N, s.C, s.dt, 1);
            at::Tensor ws;
            if (wb) ws = buffer(wb, x);
            const int rc = rec_backward(x.data_ptr(), g.data_ptr(), (const float *)data(h0), h.data_ptr(), dh.data_ptr(),
                                        (const float *)data(dlast), out[0].data_ptr(), out[1].data_ptr(),
                                        (float *)data(out[2]), (const int *)data(lengths), s.B, s.N, s.C, (la_gate)gate,
                                        s.dt, data(ws), wb, current_stream(x));
            if (rc == 0) return once(std::move(out), grads);
        }
        // gradients of another kind, or a call that the library refuses: the Python code takes or words it
        pybind11::gil_scoped_acquire gil;
        variable_list out = from_python(python_recurrence, Py_BuildValue("NNNNNNNLi", wrapped(x), wrapped(g), wrapped(h0),
                                                                         wrapped(h), wrapped(lengths), wrapped(dh),
                                                                         wrapped(dlast), (long long)gate, (int)wants_h0));
        out.resize(5);
        return once(std::move(out), grads);
    }
};

// x, gates, h0, lengths, gate -> (h, last), or the library's status
PyObject *recurrence(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    PyObject *declined = guarded(n, 5, [&]() -> PyObject * {
        if (!ours(a, 0, 3) || is_none(a[1]) || !PyLong_CheckExact(a[4])) Py_RETURN_NONE;
        const at::Tensor &x = tensor(a[0]);
        require(x.dim() >= 2 && ints_of_sequences(x));
        dtype_code(x);
        check_like(x, {a[1]});
        check_inputs(x, {a[0], a[1], a[2], a[3]});
        require(is_none(a[2]) || (tensor(a[2]).scalar_type() == at::kFloat && tensor(a[2]).sizes() == at::IntArrayRef(state_sizes(x))));
        require(is_none(a[3]) ||
                (tensor(a[3]).scalar_type() == at::kInt && tensor(a[3]).sizes() == x.sizes().slice(0, x.dim() - 2)));
        return PyBool_FromLong(1);
    });
    if (declined != Py_True) return declined;
    Py_DECREF(declined);
    try {
        return tuple(Recurrence::apply(tensor(a[0]), tensor(a[1]), maybe(a[2]), maybe(a[3]), (int64_t)PyLong_AsLong(a[4])));
    } catch (const Status &s) {
        return PyLong_FromLong(s.rc);
    }
    END_HANDLE_TH_ERRORS
}

// x, gates, h, state, gate, stream -> status
PyObject *recurrence_step(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 6, [&]() -> PyObject * {
        for (int i = 0; i < 4; ++i)
            if (!plain(a[i])) Py_RETURN_NONE;
        const at::Tensor &x = tensor(a[0]), &state = tensor(a[3]);
        require(x.dim() >= 2 && ints_of_sequences(x) && PyLong_CheckExact(a[4]));
        check_packed({a[0], a[1], a[2], a[3]});
        check_like(x, {a[1], a[2]});
        dtype_code(x);
        require(state.scalar_type() == at::kFloat && state.sizes() == at::IntArrayRef(state_sizes(x)));
        const Sequences s(x);
        const la_gate gate = (la_gate)PyLong_AsLong(a[4]);
        void *const st = stream_of(a[5], x), *const p[] = {address(a[0]), address(a[1]), address(a[2]), address(a[3])};
        const c10::DeviceGuard guard(x.device());
        PyObject *const rc = status([&] { return rec_step(p[0], p[1], p[2], (float *)p[3], s.B, s.N, s.C, gate, s.dt, st); });
        if (rc && PyLong_AsLong(rc) == 0)  // a node that saved what was written must not go on with the new values
            for (int i : {2, 3})
                if (!tensor(a[i]).is_inference()) tensor(a[i]).unsafeGetTensorImpl()->bump_version();
        return rc;
    });
}

// ---- rows in 8 bits -------------------------------------------------------------------------------------------

std::vector<int64_t> power_sizes(at::IntArrayRef sizes)
{
    std::vector<int64_t> s(sizes.begin(), sizes.end());
    s.back() = (s.back() + 31) / 32;
    return s;
}
at::Tensor codes_for(at::IntArrayRef sizes, int64_t code, const at::Tensor &ref)
{
    return at::empty(sizes, ref.options().dtype(code == LA_E4M3 ? at::kFloat8_e4m3fn : at::kChar));
}
at::Tensor powers_for(at::IntArrayRef sizes, const at::Tensor &ref)
{
    return at::empty(power_sizes(sizes), ref.options().dtype(at::kFloat8_e8m0fnu));
}

// ---- norm -----------------------------------------------------------------------------------------------------

la_dtype weight_code(const at::Tensor &w) { return !w.defined() || w.scalar_type() == at::kFloat ? LA_F32 : LA_BF16; }

struct NormOut {
    at::Tensor y, powers, total, kept, kept_powers, rstd;
};
// One call of la_rmsnorm_forward: y in `ycode` (or -1: as x), the sum also in `kcode` (or -1), rstd where it is wanted.
// The interpreter lock is held.
NormOut run_norm(const at::Tensor &x, const Maybe &residual, const Maybe &weight, double eps, int64_t ycode, int64_t kcode,
                 bool with_rstd)
{
    NormOut o;
    o.y = ycode < 0 ? at::empty_like(x) : codes_for(x.sizes(), ycode, x);
    if (ycode >= 0) o.powers = powers_for(x.sizes(), x);
    if (residual) o.total = at::empty_like(x);
    if (kcode >= 0) o.kept = codes_for(x.sizes(), kcode, x), o.kept_powers = powers_for(x.sizes(), x);
    if (with_rstd) o.rstd = at::empty(x.sizes().slice(0, x.dim() - 1), x.options().dtype(at::kFloat));
    const int C = (int)x.size(-1);
    const size_t rows = C ? x.numel() / C : 0;
    const la_dtype dt = x.scalar_type() == at::kFloat ? LA_F32 : LA_BF16, wt = weight_code(kept(weight));
    void *const p[] = {x.data_ptr(), data(residual), data(weight), o.y.data_ptr(), data(o.powers), data(o.total),
                       data(o.kept), data(o.kept_powers), data(o.rstd), current_stream(x)};
    int rc;
    Py_BEGIN_ALLOW_THREADS rc = norm_forward(p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], (float *)p[8], rows, C,
                                             (float)eps, dt, wt, ycode < 0 ? dt : (la_dtype)ycode,
                                             kcode < 0 ? LA_E4M3 : (la_dtype)kcode, p[9]);
    Py_END_ALLOW_THREADS
    if (rc != 0) throw Status{rc};
    return o;
}

struct RmsNorm : torch::autograd::Function<RmsNorm> {
    static variable_list forward(AutogradContext *ctx, const at::Tensor &x0, const Maybe &residual0, const Maybe &weight0,
                                 double eps, int64_t code)
    {
        const c10::DeviceGuard guard(x0.device());
        const at::Tensor x = x0.contiguous();
        const Maybe residual = packed(residual0), weight = packed(weight0);
        const NormOut o = run_norm(x, residual, weight, eps, -1, code, true);
        ctx->save_for_backward({code >= 0 ? o.kept : residual ? o.total : x, o.kept_powers, kept(weight), o.rstd});
        ctx->saved_data["code"] = code;
        ctx->saved_data["residual"] = residual.has_value();
        ctx->set_materialize_grads(false);
        if (residual) return {o.y, o.total};
        return {o.y};
    }
    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        const bool residual = ctx->saved_data["residual"].toBool();
        const bool wants_res = residual && ctx->needs_input_grad(1);
        variable_list out(5);
        if (!grads[0].defined()) {  // the sum alone was used
            out[0] = grads.size() > 1 ? grads[1] : at::Tensor();
            if (wants_res) out[1] = out[0];
            return out;
        }
        const auto v = ctx->get_saved_variables();
        const at::Tensor &total = v[0], &powers = v[1], &weight = v[2], &rstd = v[3];
        const int64_t code = ctx->saved_data["code"].toInt();
        const bool wants_w = weight.defined() && ctx->needs_input_grad(residual ? 2 : 1);
        const at::Tensor dy = grads[0].contiguous(),
                         dtotal = grads.size() > 1 && grads[1].defined() ? grads[1].contiguous() : at::Tensor();
        const auto type = dy.scalar_type();
        const auto sizes = total.sizes();
        if (sizes.size() && (type == at::kFloat || type == at::kBFloat16) && fits(dy, total, type, sizes) &&
            fits(dtotal, total, type, sizes) &&
            fits(total, total, code < 0 ? type : code == LA_E4M3 ? at::kFloat8_e4m3fn : at::kChar, sizes) &&
            fits(powers, total, at::kFloat8_e8m0fnu, power_sizes(sizes)) && (code < 0) == !powers.defined() &&
            fits(rstd, total, at::kFloat, sizes.slice(0, sizes.size() - 1)) &&
            fits(weight, total, weight.defined() && weight.scalar_type() != type ? at::kFloat : type, sizes.slice(sizes.size() - 1))) {
            const c10::DeviceGuard guard(dy.device());
            const int C = (int)dy.size(-1);
            const size_t rows = dy.numel() / C;
            at::Tensor dx = at::empty_like(dy), dw, ws;
            size_t wb = 0;
            if (wants_w) {
                dw = at::empty({C}, dy.options().dtype(at::kFloat));
                wb = norm_bytes(rows, C);
                ws = buffer(wb, dy);
            }
            const la_dtype dt = type == at::kFloat ? LA_F32 : LA_BF16;
            const int rc = norm_backward(total.data_ptr(), data(powers), data(weight), (const float *)rstd.data_ptr(),
                                         dy.data_ptr(), data(dtotal), dx.data_ptr(), (float *)data(dw), rows, C, dt,
                                         weight_code(weight), code < 0 ? dt : (la_dtype)code, data(ws), wb, current_stream(dy));
            if (rc == 0) {
                out[0] = dx;
                if (wants_res) out[1] = dx;
                if (wants_w) out[2] = dw.to(weight.scalar_type());
                return once(std::move(out), grads);
            }
        }
        pybind11::gil_scoped_acquire gil;
        out = from_python(python_norm, Py_BuildValue("NNNNNNLii", wrapped(total), wrapped(powers), wrapped(weight),
                                                     wrapped(rstd), wrapped(dy), wrapped(dtotal), (long long)code,
                                                     (int)wants_res, (int)wants_w));
        out.resize(5);
        return once(std::move(out), grads);
    }
};

// Whether x, weight and residual are what the library takes.
void check_norm(PyObject *x0, PyObject *weight, PyObject *residual)
{
    require(plain(x0) && plain_or_none(weight) && plain_or_none(residual));
    const at::Tensor &x = tensor(x0);
    require(x.dim() >= 1 && ints({x.size(-1)}));
    dtype_code(x);
    check_like(x, {residual});
    check_inputs(x, {x0, weight, residual});
    require(is_none(weight) || (tensor(weight).sizes() == x.sizes().slice(x.dim() - 1) &&
                                (tensor(weight).scalar_type() == at::kFloat || tensor(weight).scalar_type() == x.scalar_type())));
}

// x, weight, residual, eps, code (-1: none) -> (y) or (y, total), or the library's status
PyObject *norm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    double eps = 0;
    PyObject *declined = guarded(n, 5, [&]() -> PyObject * {
        check_norm(a[0], a[1], a[2]);
        require(PyLong_CheckExact(a[4]) && !THPVariable_Check(a[3]));
        eps = real(a[3]);
        return PyBool_FromLong(1);
    });
    if (declined != Py_True) return declined;
    Py_DECREF(declined);
    try {
        return tuple(RmsNorm::apply(tensor(a[0]), maybe(a[2]), maybe(a[1]), eps, (int64_t)PyLong_AsLong(a[4])));
    } catch (const Status &s) {
        return PyLong_FromLong(s.rc);
    }
    END_HANDLE_TH_ERRORS
}

// x, weight, residual, eps, code -> (codes, scales) or (codes, scales, total), or the library's status
PyObject *norm_quantised(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 5, [&]() -> PyObject * {
        check_norm(a[0], a[1], a[2]);
        require(PyLong_CheckExact(a[4]));
        const double eps = real(a[3]);
        const int64_t code = PyLong_AsLong(a[4]);
        require(code == LA_E4M3 || code == LA_I8);
        const at::AutoDispatchBelowADInplaceOrView plainly;  // no graph
        const c10::DeviceGuard guard(tensor(a[0]).device());
        try {
            const at::Tensor x = tensor(a[0]).contiguous();
            const NormOut o = run_norm(x, packed(maybe(a[2])), packed(maybe(a[1])), eps, code, -1, false);
            return o.total.defined() ? tuple({o.y, o.powers, o.total}) : tuple({o.y, o.powers});
        } catch (const Status &s) {
            return PyLong_FromLong(s.rc);
        }
    });
}

// ---- attention with checkpoints -------------------------------------------------------------------------------

struct Checkpointed : torch::autograd::Function<Checkpointed> {
    static at::Tensor forward(AutogradContext *ctx, const at::Tensor &Q0, const at::Tensor &K0, const at::Tensor &V0, double a,
                              double b, bool causal, bool norm, int64_t code)
    {
        const c10::DeviceGuard guard(Q0.device());
        const at::Tensor Q = Q0.contiguous(), K = K0.contiguous(), V = V0.contiguous();
        const int B = Q.size(0), H = Q.size(1), N = Q.size(2), D = Q.size(3);
        const la_dtype dt = dtype_code(Q);
        const at::Tensor O = at::empty_like(Q), ws = buffer(att_bytes(B, H, N, D, dt, causal, 0), Q);
        const at::Tensor codes = codes_for({3, B, H, N, D}, code, Q), powers = powers_for({3, B, H, N, D}, Q);
        const size_t rows = (size_t)B * H * N, step = rows * D, pstep = rows * ((D + 31) / 32), wb = bytes(ws);
        const void *const x[] = {Q.data_ptr(), K.data_ptr(), V.data_ptr()};
        char *const c = (char *)codes.data_ptr(), *const p = (char *)powers.data_ptr();
        void *const cs[] = {c, c + step, c + 2 * step}, *const ps[] = {p, p + pstep, p + 2 * pstep};
        void *const o = O.data_ptr(), *const w = ws.data_ptr(), *const st = current_stream(Q);
        int rc;
        Py_BEGIN_ALLOW_THREADS rc = (norm ? att_forward_qknorm : att_forward)(
            x[0], x[1], x[2], o, nullptr, B, H, N, D, (float)a, (float)b, causal, dt, w, wb, st, nullptr);
        if (rc == 0) rc = pack_tensors(3, x, cs, ps, rows, D, dt, (la_dtype)code, st);
        Py_END_ALLOW_THREADS
        if (rc != 0) throw Status{rc};
        ctx->save_for_backward({codes, powers});
        ctx->saved_data["a"] = a;
        ctx->saved_data["b"] = b;
        ctx->saved_data["causal"] = causal;
        ctx->saved_data["norm"] = norm;
        ctx->saved_data["code"] = code;
        ctx->saved_data["float"] = dt == LA_F32;
        return O;
    }
    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        auto &d = ctx->saved_data;
        const auto v = ctx->get_saved_variables();
        const at::Tensor &codes = v[0], &powers = v[1], dO = grads[0].contiguous();
        const double a = d["a"].toDouble(), b = d["b"].toDouble();
        const bool causal = d["causal"].toBool(), norm = d["norm"].toBool();
        const int64_t code = d["code"].toInt();
        const la_dtype dt = d["float"].toBool() ? LA_F32 : LA_BF16;
        const auto type = dt == LA_F32 ? at::kFloat : at::kBFloat16;
        variable_list out(8);
        if (codes.dim() == 5 && fits(codes, codes, code == LA_E4M3 ? at::kFloat8_e4m3fn : at::kChar, codes.sizes()) &&
            fits(powers, codes, at::kFloat8_e8m0fnu, power_sizes(codes.sizes())) &&
            fits(dO, codes, type, codes.sizes().slice(1))) {
            const c10::DeviceGuard guard(dO.device());
            const int B = dO.size(0), H = dO.size(1), N = dO.size(2), D = dO.size(3);
            const size_t rows = (size_t)B * H * N;
            for (int i = 0; i < 3; ++i) out[i] = at::empty_like(dO);
            // one workspace for both passes, which follow one another on the stream
            const size_t wb = std::max(att_bytes(B, H, N, D, dt, causal, 0), att_bytes(B, H, N, D, dt, causal, 1)),
                         ns = att_saved_bytes(B, H, N, D, dt, causal), tb = rows * D * dO.element_size();
            // Q, K, V side by side, O, g, the hand-over and the workspace in one allocation
            const size_t sizes[] = {3 * tb, tb, rows * 4, ns, std::max(wb, (size_t)256)};
            size_t at[5], total = 0;
            for (int i = 0; i < 5; ++i) at[i] = total, total += (sizes[i] + 255) / 256 * 256;
            const at::Tensor room = buffer(total, dO);
            char *const base = (char *)room.data_ptr(), *const q = base, *const k = q + tb, *const vv = k + tb;
            void *const O = base + at[1], *const saved = ns ? base + at[3] : nullptr, *const ws = base + at[4];
            float *const g = (float *)(base + at[2]);
            void *const st = current_stream(dO);
            int rc = unpack_rows(codes.data_ptr(), powers.data_ptr(), q, 3 * rows, D, (la_dtype)code, dt, st);
            if (rc == 0)
                rc = (norm ? att_save_qknorm : att_save)(q, k, vv, O, g, B, H, N, D, (float)a, (float)b, causal, dt, ws, wb, saved,
                                                         ns, st, nullptr);
            if (rc == 0)
                rc = (norm ? att_backward_qknorm : att_backward)(
                    q, k, vv, O, g, dO.data_ptr(), out[0].data_ptr(), out[1].data_ptr(), out[2].data_ptr(), B, H, N, D, (float)a,
                    (float)b, causal, dt, ws, wb, saved, ns, st, nullptr);
            if (rc == 0) return once(std::move(out), grads);
        }
        pybind11::gil_scoped_acquire gil;
        out = from_python(python_checkpointed,
                          Py_BuildValue("NNNddiiLi", wrapped(codes), wrapped(powers), wrapped(dO), a, b, (int)causal, (int)norm,
                                        (long long)code, (int)(dt == LA_F32)));
        out.resize(8);
        return once(std::move(out), grads);
    }
};

// Q, K, V, a, b, causal, normalise, code -> O, or the library's status
PyObject *checkpointed(PyObject *, PyObject *const *x, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    double a = 0, b = 0;
    PyObject *declined = guarded(n, 8, [&]() -> PyObject * {
        for (int i = 0; i < 3; ++i)
            if (!plain(x[i])) Py_RETURN_NONE;
        const at::Tensor &Q = tensor(x[0]);
        require(Q.dim() == 4 && Q.is_cuda() && PyLong_CheckExact(x[7]));
        dtype_code(Q);
        check_like(Q, {x[1], x[2]});
        check_inputs(Q, {x[0], x[1], x[2]});
        for (int i = 3; i < 7; ++i) require(!THPVariable_Check(x[i]));
        a = real(x[3]);
        b = real(x[4]);
        return PyBool_FromLong(1);
    });
    if (declined != Py_True) return declined;
    Py_DECREF(declined);
    const int causal = PyObject_IsTrue(x[5]), norm = PyObject_IsTrue(x[6]);
    if (PyErr_Occurred()) return nullptr;
    try {
        return THPVariable_Wrap(Checkpointed::apply(tensor(x[0]), tensor(x[1]), tensor(x[2]), a, b, causal != 0, norm != 0,
                                                    (int64_t)PyLong_AsLong(x[7])));
    } catch (const Status &s) {
        return PyLong_FromLong(s.rc);
    }
    END_HANDLE_TH_ERRORS
}

}  // namespace

// The backward passes in Python, then the addresses of the entry points in the order of the pointers above
PyObject *init_layer(PyObject *, PyObject *const *x, Py_ssize_t n)
{
    PyObject **const calls[] = {&python_recurrence, &python_norm, &python_checkpointed};
    void **const to[] = {(void **)&rec_bytes, (void **)&rec_forward, (void **)&rec_backward, (void **)&rec_step,
                         (void **)&pack_tensors, (void **)&unpack_rows, (void **)&norm_bytes, (void **)&norm_forward,
                         (void **)&norm_backward, (void **)&att_forward, (void **)&att_forward_qknorm, (void **)&att_save,
                         (void **)&att_save_qknorm, (void **)&att_backward, (void **)&att_backward_qknorm,
                         (void **)&att_bytes, (void **)&att_saved_bytes};
    constexpr Py_ssize_t COUNT = sizeof(to) / sizeof(to[0]);
    if (n != 3 + COUNT) {
        PyErr_SetString(PyExc_TypeError, "init_layer takes three callables and the entry points' addresses");
        return nullptr;
    }
    for (Py_ssize_t i = 0; i < COUNT; ++i) {
        *to[i] = PyLong_AsVoidPtr(x[3 + i]);
        if (!*to[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null address");
            return nullptr;
        }
    }
    for (int i = 0; i < 3; ++i) {
        Py_INCREF(x[i]);
        Py_XSETREF(*calls[i], x[i]);
    }
    Py_RETURN_NONE;
}

PyMethodDef layer_methods[] = {{"recurrence", (PyCFunction)(void (*)())recurrence, METH_FASTCALL, nullptr},
                               {"recurrence_step", (PyCFunction)(void (*)())recurrence_step, METH_FASTCALL, nullptr},
                               {"norm", (PyCFunction)(void (*)())norm, METH_FASTCALL, nullptr},
                               {"norm_quantised", (PyCFunction)(void (*)())norm_quantised, METH_FASTCALL, nullptr},
                               {"checkpointed", (PyCFunction)(void (*)())checkpointed, METH_FASTCALL, nullptr},
                               {nullptr, nullptr, 0, nullptr}};
