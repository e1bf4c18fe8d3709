"""torch.autograd wrapper over the C ABI (the paper's plug-and-play module, Sec. 6).

Plumbing only: it allocates the outputs, the workspaces and the hand-over buffer with
torch, keeps the set {Q, K, V, O, g} of Sec. 3.2 (plus the forward pass's running sums at
the segment boundaries) for the backward pass, and calls la_forward_save /
la_backward_saved; for plain tensors outside of modes, transforms and traces by a node of the same steps in
native code (binding.attention).  Every arithmetic step runs in the HIP library; there is no fallback.
Gradients are with respect to the Q, K, V handed in; with ``normalize_qk`` the rows of Q and
K are scaled to unit length inside the kernels (Sec. 3.3) and the gradients are those for the
raw rows.  a and b are constants.

The operators around the attention follow below it in the same manner: gated_recurrence, rms_norm, and
rows in 8 bits (pack_rows, unpack_rows, rms_norm_quantised, the ``checkpoint`` of linear_attention and
rms_norm); behind them a selective state space layer's: causal_conv, selective_scan.

Every call can be captured into a graph, a training step too: run it a few times on the stream that will capture,
let go of the results (no eager graph of the same leaves may be alive while a backward pass is captured: torch
then joins streams inside the capture), and take the gradients from torch.autograd.grad.
"""
import functools

import torch

from . import binding as _b


def _code(t):
    return _b.LA_F32 if t.dtype == torch.float32 else _b.LA_BF16


def _bytes(n, device):
    return torch.empty(max(int(n), 256), dtype=torch.uint8, device=device)


def _once(backward):
    """``backward`` gets the saved tensors as a call that unpacks them one time, whatever hooks they went through.
    Gradients of gradients are not defined: where a graph of the backward pass is asked for, results that depend on them
    come out of a node that refuses, tied to the incoming gradients and the tensors that were kept."""
    @functools.wraps(backward)
    def refusing(ctx, *grads):
        kept = []

        def saved():
            if not kept:
                kept.append(ctx.saved_tensors)
            return kept[0]
        with torch.no_grad():
            out = backward(ctx, saved, *grads)
        if not kept or not torch.is_grad_enabled():
            return out
        ends = [t.detach().requires_grad_(True) for t in out if t is not None]
        ties = [t for t in (*kept[0], *grads) if t is not None and t.requires_grad]
        refuse = torch._C._functions.DelayedError(b"gradients of gradients are not defined for this operator",
                                                  len(ends) + len(ties))
        ends = refuse(*ends, *ties)
        ends = iter((ends,) if isinstance(ends, torch.Tensor) else ends)
        return tuple(None if t is None else next(ends) for t in out)
    return refusing


class LinearAttentionFunction(torch.autograd.Function):
    """O = LA(Q, K, V) with kernel f(x) = a + b x; Q, K, V: [B, H, N, D] device tensors."""

    @staticmethod
    def forward(ctx, Q, K, V, a, b, causal, normalize_qk=False):
        Q, K, V = Q.contiguous(), K.contiguous(), V.contiguous()
        B, H, N, D = Q.shape
        dt = _code(Q)
        O = torch.empty_like(Q)
        G = torch.empty((B, H, N), dtype=torch.float32, device=Q.device)
        ws = _bytes(_b.la_workspace_bytes(B, H, N, D, dt, causal, 0), Q.device)
        ns = _b.la_saved_state_bytes(B, H, N, D, dt, causal)
        saved = _bytes(ns, Q.device) if ns else None
        fwd = _b.la_forward_qknorm_save if normalize_qk else _b.la_forward_save
        fwd(Q, K, V, O, G, a, b, causal, ws, saved)
        ctx.save_for_backward(Q, K, V, O, G)
        ctx.la_saved = saved
        ctx.la_args = (float(a), float(b), bool(causal), bool(normalize_qk))
        return O

    @staticmethod
    def backward(ctx, dO):
        return (*python_backward(*ctx.saved_tensors, dO, ctx.la_saved, *ctx.la_args), None, None, None, None)


def python_backward(Q, K, V, O, G, dO, saved, a, b, causal, normalize_qk):
    B, H, N, D = Q.shape
    dO = dO.contiguous()
    dQ, dK, dV = torch.empty_like(Q), torch.empty_like(Q), torch.empty_like(Q)
    ws = _bytes(_b.la_workspace_bytes(B, H, N, D, _code(Q), causal, 1), Q.device)
    bwd = _b.la_backward_qknorm_saved if normalize_qk else _b.la_backward_saved
    bwd(Q, K, V, O, G, dO, dQ, dK, dV, a, b, causal, ws, saved)
    return dQ, dK, dV


class CheckpointedAttentionFunction(torch.autograd.Function):
    """The same with Q, K, V kept in 8 bits and nothing else: the backward pass unpacks them, runs the
    forward pass again on what they stand for, and returns the gradients there."""

    @staticmethod
    def forward(ctx, Q, K, V, a, b, causal, normalize_qk, code):
        Q, K, V = Q.contiguous(), K.contiguous(), V.contiguous()
        B, H, N, D = Q.shape
        dt = _code(Q)
        O = torch.empty_like(Q)
        ws = _bytes(_b.la_workspace_bytes(B, H, N, D, dt, causal, 0), Q.device)
        (_b.la_forward_qknorm if normalize_qk else _b.la_forward)(Q, K, V, O, None, a, b, causal, ws)
        codes, scales = _eight_bits(Q, code, 3)
        _b.la_pack_tensors([Q, K, V], list(codes), list(scales), code)
        ctx.save_for_backward(codes, scales)
        ctx.la_args = (float(a), float(b), bool(causal), bool(normalize_qk), code, Q.dtype == torch.float32)
        return O

    @staticmethod
    @_once
    def backward(ctx, saved, dO):
        return (*checkpointed_backward(*saved(), dO.contiguous(), *ctx.la_args), None, None, None, None, None)


def checkpointed_backward(codes, scales, dO, a, b, causal, normalize_qk, code, single):
    Q, K, V = unpack_rows(codes, scales, code, torch.float32 if single else torch.bfloat16)
    B, H, N, D = Q.shape
    dt = _code(Q)
    O, G = torch.empty_like(Q), torch.empty((B, H, N), dtype=torch.float32, device=Q.device)
    ws = _bytes(_b.la_workspace_bytes(B, H, N, D, dt, causal, 0), Q.device)
    ns = _b.la_saved_state_bytes(B, H, N, D, dt, causal)
    saved = _bytes(ns, Q.device) if ns else None
    fwd = _b.la_forward_qknorm_save if normalize_qk else _b.la_forward_save
    fwd(Q, K, V, O, G, a, b, causal, ws, saved)
    return python_backward(Q, K, V, O, G, dO, saved, a, b, bool(causal), bool(normalize_qk))


def linear_attention(Q, K, V, a=1.0, b=0.5, causal=True, normalize_qk=False, checkpoint=None):
    """Differentiable linear attention on [B, H, N, D] float32 or bfloat16 device tensors;
    ``normalize_qk`` scales the rows of Q and K to unit length inside the kernels (D <= 128).

    ``checkpoint`` "e4m3" or "int8" keeps Q, K, V for the backward pass in 8 bits (3.1 bytes an element of Q
    instead of 8 in bfloat16, 16 in float32; la_pack_rows of include/la.h): the gradients are then those at the
    values that the 8 bits stand for, and the backward pass runs the forward pass again."""
    if checkpoint is not None:
        code = _b.eight_bit_code(checkpoint)
        if Q.shape != K.shape or Q.shape != V.shape:
            raise ValueError("shape mismatch")
        O = _b.in_native_code("checkpointed", "la_forward_save" if normalize_qk else "la_forward", Q, K, V, a, b, causal, normalize_qk, code)
        if O is not None:
            return O
        return CheckpointedAttentionFunction.apply(Q, K, V, a, b, causal, normalize_qk, code)
    O = _b.attention(Q, K, V, a, b, causal, normalize_qk)
    if O is not None:
        return O
    return LinearAttentionFunction.apply(Q, K, V, a, b, causal, normalize_qk)


def pack_rows(x, code):
    """x [..., C] in 8 bits: codes (float8_e4m3fn or int8) and the powers of two of 32 neighbours
    (float8_e8m0fnu); ``code`` "e4m3", "int8", LA_E4M3 or LA_I8.  Not differentiable."""
    code = _b.eight_bit_code(code) if isinstance(code, str) else code
    x = x.detach().contiguous()
    codes, scales = _eight_bits(x, code)
    _b.la_pack_rows(x, codes, scales, code)
    return codes, scales


def unpack_rows(codes, scales, code, dtype):
    """The values that pack_rows' codes stand for, as ``dtype`` (float32 or bfloat16)."""
    code = _b.eight_bit_code(code) if isinstance(code, str) else code
    codes, scales = codes.contiguous(), scales.contiguous()
    x = torch.empty(codes.shape, dtype=dtype, device=codes.device)
    _b.la_unpack_rows(codes, scales, x, code)
    return x


def _eight_bits(x, code, *count):
    """Room for x's codes and powers (for `count` tensors like x)."""
    kind = torch.float8_e4m3fn if code == _b.LA_E4M3 else torch.int8
    groups = (*count, *_b.powers_shape(x.shape))
    return (torch.empty((*count, *x.shape), dtype=kind, device=x.device),
            torch.empty(groups, dtype=torch.float8_e8m0fnu, device=x.device))


_GATES = {"value": _b.LA_GATE_VALUE, "sigmoid": _b.LA_GATE_SIGMOID}


class GatedRecurrenceFunction(torch.autograd.Function):
    """h_t = f_t h_{t-1} + u_t (la_recurrence_forward); x, gates: [..., N, C] device tensors."""

    @staticmethod
    def forward(ctx, x, gates, h0, lengths, gate):
        x, gates = x.contiguous(), gates.contiguous()
        h0 = h0 if h0 is None else h0.contiguous()
        lengths = lengths if lengths is None else lengths.contiguous()
        h = torch.empty_like(x)
        last = torch.empty((*x.shape[:-2], x.shape[-1]), dtype=torch.float32, device=x.device)
        _b.la_recurrence_forward(x, gates, h0, h, last, lengths, gate, _recurrence_room(x, 0))
        ctx.save_for_backward(x, gates, h0, h, lengths)
        ctx.la_gate = gate
        ctx.set_materialize_grads(False)
        return h, last

    @staticmethod
    @_once
    def backward(ctx, saved, dh, dlast):
        x = saved()[0]
        dh = torch.zeros_like(x) if dh is None else dh.contiguous()
        dlast = dlast if dlast is None else dlast.contiguous()
        return (*recurrence_backward(*saved(), dh, dlast, ctx.la_gate, ctx.needs_input_grad[2]), None, None)


def recurrence_backward(x, gates, h0, h, lengths, dh, dlast, gate, wants_h0):
    dx, dgates = torch.empty_like(x), torch.empty_like(x)
    dh0 = torch.empty_like(h0) if wants_h0 else None
    _b.la_recurrence_backward(x, gates, h0, h, dh, dlast, dx, dgates, dh0, lengths, gate, _recurrence_room(x, 1))
    return dx, dgates, dh0


def _recurrence_room(x, is_backward):
    N, C = x.shape[-2:]
    n = _b.la_recurrence_workspace_bytes(x.numel() // (N * C) if x.numel() else 0, N, C, _code(x), is_backward)
    return _bytes(n, x.device) if n else None


def gated_recurrence(x, gates, h0=None, lengths=None, gate="sigmoid"):
    """Differentiable gated linear recurrence along the second to last dimension of x, gates [..., N, C]
    (float32 or bfloat16 device tensors): h_t = f_t h_{t-1} + u_t with

      gate "sigmoid":  f_t = sigmoid(gates_t), u_t = (1 - f_t) x_t;   gate "value":  f_t = gates_t, u_t = x_t.

    h0 [..., C] float32: the state before the first row (None: zeros).  lengths [...] int32: rows from there
    on are padding, zero in every output.  Returns h like x and the state after the last row, [..., C] float32,
    from which la_recurrence_step goes on."""
    if gate not in _GATES:
        raise ValueError("gates are %s, got %r" % (" and ".join(map(repr, _GATES)), gate))
    out = _b.in_native_code("recurrence", "la_recurrence_forward", x, gates, h0, lengths, _GATES[gate])
    if out is not None:
        return out
    return GatedRecurrenceFunction.apply(x, gates, h0, lengths, _GATES[gate])


class RmsNormFunction(torch.autograd.Function):
    """y = w s rstd, s = x + residual (la_rmsnorm_forward); x: [..., C] device tensors."""

    @staticmethod
    def forward(ctx, x, residual, weight, eps, code):
        x = x.contiguous()
        residual = residual if residual is None else residual.contiguous()
        weight = weight if weight is None else weight.contiguous()
        y = torch.empty_like(x)
        total = None if residual is None else torch.empty_like(x)
        rstd = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
        kept, kscales = (None, None) if code is None else _eight_bits(x, code)
        _b.la_rmsnorm_forward(x, residual, weight, y, None, total, kept, kscales, rstd, eps, None, code)
        ctx.save_for_backward((x if total is None else total) if code is None else kept, kscales, weight, rstd)
        ctx.la_code = code
        ctx.set_materialize_grads(False)
        return y, total

    @staticmethod
    @_once
    def backward(ctx, saved, dy, dtotal):
        if dy is None:  # the sum alone was used
            return dtotal, dtotal if ctx.needs_input_grad[1] else None, None, None, None
        dtotal = dtotal if dtotal is None else dtotal.contiguous()
        return (*norm_backward(*saved(), dy.contiguous(), dtotal, -1 if ctx.la_code is None else ctx.la_code,
                               ctx.needs_input_grad[1], ctx.needs_input_grad[2]), None, None)


def norm_backward(total, scales, weight, rstd, dy, dtotal, code, wants_residual, wants_weight):
    dx = torch.empty_like(dy)
    dw = ws = None
    if wants_weight:
        C = dy.shape[-1]
        dw = torch.empty(C, dtype=torch.float32, device=dy.device)
        ws = _bytes(_b.la_rmsnorm_workspace_bytes(dy.numel() // C, C), dy.device)
    _b.la_rmsnorm_backward(total, scales, weight, rstd, dy, dtotal, dx, dw, ws, None if code < 0 else code)
    return dx, dx if wants_residual else None, dw if dw is None else dw.to(weight.dtype)


def rms_norm(x, weight=None, residual=None, eps=1e-6, checkpoint=None):
    """Differentiable root-mean-square norm of the rows of x [..., C] (float32 or bfloat16 device tensors),
    with ``residual`` added first: s = x + residual, y = weight s / sqrt(mean(s^2) + eps); weight [C] float32
    or x's type (None: ones).  Returns y, or (y, s) where there is a residual.

    ``checkpoint`` "e4m3" or "int8" keeps s in 8 bits for the backward pass, which then goes by those."""
    code = None if checkpoint is None else _b.eight_bit_code(checkpoint)
    out = _b.in_native_code("norm", "la_rmsnorm_forward", x, weight, residual, eps, -1 if code is None else code)
    if out is None:
        out = RmsNormFunction.apply(x, residual, weight, float(eps), code)
    return out[0] if residual is None else out


def rms_norm_quantised(x, weight=None, residual=None, eps=1e-6, code="e4m3"):
    """rms_norm with y in 8 bits, for a matrix product on 8-bit operands: codes like x (float8_e4m3fn or
    int8) and scales [..., ceil(C / 32)] (float8_e8m0fnu), and s where there is a residual.  Not differentiable."""
    code = _b.eight_bit_code(code)
    out = _b.in_native_code("norm_quantised", "la_rmsnorm_forward", x, weight, residual, eps, code)
    if out is not None:
        return out
    x = x.detach().contiguous()
    residual = residual if residual is None else residual.detach().contiguous()
    weight = weight if weight is None else weight.detach().contiguous()
    codes, scales = _eight_bits(x, code)
    total = None if residual is None else torch.empty_like(x)
    _b.la_rmsnorm_forward(x, residual, weight, codes, scales, total, None, None, None, eps, code)
    return (codes, scales) if residual is None else (codes, scales, total)


# ---- the selective state space layer ----------------------------------------------------------

def _rows_in_place(t, dims=1, below=1 << 62):
    """t as the kernels take it: rows that are dense and at one distance, less than `below` elements, else a copy."""
    return t if t is None or (_b.row_stride(t, dims) or below) < below else t.contiguous()


def _dense(t):
    return t if t is None else t.contiguous()


class CausalConvFunction(torch.autograd.Function):
    """y_t = act(bias + sum_j w_j x_{t-(W-1)+j}) (la_conv_forward); x: [..., N, C] device tensors."""

    @staticmethod
    def forward(ctx, x, weight, bias, state, lengths, act):
        x, weight, bias, state, lengths = _rows_in_place(x), *map(_dense, (weight, bias, state, lengths))
        if x.dim() < 2 or weight.dim() != 2:
            raise ValueError("x must be [..., N, C] and the weight [C, taps]")
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        last = torch.empty((*x.shape[:-2], weight.shape[1] - 1, x.shape[-1]), dtype=x.dtype, device=x.device)
        _b.la_conv_forward(x, weight, bias, state, y, last, lengths, act)
        ctx.save_for_backward(x, weight, bias, state, lengths)
        ctx.la_act = act
        ctx.set_materialize_grads(False)
        return y, last

    @staticmethod
    @_once
    def backward(ctx, saved, dy, dlast):
        x = saved()[0]
        dy = torch.zeros(x.shape, dtype=x.dtype, device=x.device) if dy is None else dy.contiguous()
        return (*conv_backward(*saved(), dy, _dense(dlast), ctx.la_act, *ctx.needs_input_grad[1:4]), None, None)


def conv_backward(x, weight, bias, state, lengths, dy, dlast, act, wants_weight, wants_bias, wants_state):
    dx = torch.empty_like(dy)
    dw = torch.empty(weight.shape, dtype=torch.float32, device=x.device) if wants_weight else None
    db = torch.empty(weight.shape[:1], dtype=torch.float32, device=x.device) if wants_bias else None
    ds = torch.empty_like(state) if wants_state else None
    ws = None
    if wants_weight or wants_bias:
        N, C = x.shape[-2:]
        ws = _bytes(_b.la_conv_workspace_bytes(x.numel() // (N * C) if x.numel() else 0, N, C, weight.shape[1]), x.device)
    _b.la_conv_backward(x, weight, bias, state, dy, dlast, dx, dw, db, ds, lengths, act, ws)
    return dx, dw if dw is None else dw.to(weight.dtype), db if db is None else db.to(bias.dtype), ds


_ACTS = {"none": _b.LA_ACT_NONE, "silu": _b.LA_ACT_SILU}
_STEPS = {"value": _b.LA_STEP_VALUE, "softplus": _b.LA_STEP_SOFTPLUS}


def causal_conv(x, weight, bias=None, state=None, lengths=None, activation="silu"):
    """Differentiable causal convolution along the second to last dimension of x [..., N, C] (float32 or bfloat16 device
    tensors; a part of wider rows is read where it is), one filter of 2 to 8 taps a channel:
    y_t = act(bias + sum_j weight[:, j] x_{t-(W-1)+j}), activation "silu" or "none"; weight [C, W] and bias [C] float32 or x's type.

    state [..., W - 1, C] like x: the rows before the first (None: zeros).  lengths [...] int32: rows from there on are
    padding, zero in every output.  Returns y like x and the last W - 1 rows of every sequence, from which la_conv_step and another
    call's state go on."""
    if activation not in _ACTS:
        raise ValueError("activations are %s, got %r" % (" and ".join(map(repr, _ACTS)), activation))
    out = _b.in_native_code("conv", "la_conv_forward", x, weight, bias, state, lengths, _ACTS[activation])
    if out is not None:
        return out
    return CausalConvFunction.apply(x, weight, bias, state, lengths, _ACTS[activation])


class SelectiveScanFunction(torch.autograd.Function):
    """h_t = exp(d_t A) h_{t-1} + d_t x_t B_t, y_t = C_t h_t + D x_t (la_selective_forward); x: [..., N, C] device tensors."""

    @staticmethod
    def forward(ctx, x, dt, A, B, C, D, bias, h0, lengths, step, keeps):
        dims = 1 if B.dim() == x.dim() else 2
        x, dt, B, C = (_rows_in_place(t, k, _b.ROWS_APART) for t, k in ((x, 1), (dt, 1), (B, dims), (C, dims)))
        A, D, bias, h0, lengths = map(_dense, (A, D, bias, h0, lengths))
        sizes = _scan_sizes(x, A, B)
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        last = torch.empty((*x.shape[:-2], *A.shape), dtype=torch.float32, device=x.device)
        saved = _bytes(_b.la_selective_saved_bytes(*sizes[:4]), x.device) if keeps else None
        n = _b.la_selective_workspace_bytes(*sizes, 0)
        _b.la_selective_forward(x, dt, A, B, C, D, bias, h0, y, last, saved, lengths, step, _bytes(n, x.device) if n else None)
        ctx.save_for_backward(x, dt, A, B, C, D, bias, lengths, saved)
        ctx.la_step = step
        ctx.set_materialize_grads(False)
        return y, last

    @staticmethod
    @_once
    def backward(ctx, saved, dy, dlast):
        x = saved()[0]
        dy = torch.zeros(x.shape, dtype=x.dtype, device=x.device) if dy is None else dy.contiguous()
        wants = ctx.needs_input_grad
        return (*scan_backward(*saved(), dy, _dense(dlast), ctx.la_step, wants[2], *wants[5:8]), None, None, None)


def _scan_sizes(x, A, B):
    if x.dim() < 2 or A.dim() != 2 or B.dim() not in (x.dim(), x.dim() + 1):
        raise ValueError("x must be [..., N, C], A [C, states], B and C [..., N, states] or [..., N, groups, states]")
    N, C = x.shape[-2:]
    return x.numel() // (N * C) if x.numel() else 0, N, C, A.shape[1], B.shape[-2] if B.dim() > x.dim() else 1


def scan_backward(x, dt, A, B, C, D, bias, lengths, saved, dy, dlast, step, wants_A, wants_D, wants_bias, wants_h0):
    sizes = _scan_sizes(x, A, B)
    dx, ddt = torch.empty_like(dy), torch.empty_like(dy)
    dB, dC = (torch.empty(B.shape, dtype=B.dtype, device=x.device) for _ in range(2))
    dA = torch.empty_like(A) if wants_A else None
    dD = torch.empty_like(D) if wants_D else None
    db = torch.empty_like(bias) if wants_bias else None
    dh0 = torch.empty((*x.shape[:-2], *A.shape), dtype=torch.float32, device=x.device) if wants_h0 else None
    ws = _bytes(_b.la_selective_workspace_bytes(*sizes, 1), x.device)
    _b.la_selective_backward(x, dt, A, B, C, D, bias, saved, dy, dlast, dx, ddt, dA, dB, dC, dD, db, dh0, lengths, step, ws)
    return dx, ddt, dA, dB, dC, dD, db, dh0


def selective_scan(x, dt, A, B, C, D=None, bias=None, h0=None, lengths=None, step="softplus"):
    """Differentiable selective state space scan along the second to last dimension of x, dt [..., N, C] (float32 or bfloat16
    device tensors), with A [C, S] float32 and B, C [..., N, S], or [..., N, G, S] for G groups of channels, like x; all but A may be
    parts of wider rows, which are read where they are (copied where they lie 2^24 elements apart or more):

      h_t = exp(d_t A) h_{t-1} + d_t x_t B_t,  y_t = sum over the states C_t h_t + D x_t,  with
      step "softplus":  d_t = log(1 + exp(dt_t + bias));   step "value":  d_t = dt_t + bias.

    D, bias [C] float32 (None: zeros).  h0 [..., C, S] float32: the state before the first row (None: zeros).  lengths [...]
    int32: rows from there on are padding, zero in every output.  Returns y like x and the state after the last row, [..., C, S]
    float32, from which la_selective_step goes on.  For the backward pass it keeps its inputs and the states of every 16th row."""
    if step not in _STEPS:
        raise ValueError("steps are %s, got %r" % (" and ".join(map(repr, _STEPS)), step))
    out = _b.in_native_code("scan", "la_selective_forward", x, dt, A, B, C, D, bias, h0, lengths, _STEPS[step])
    if out is not None:
        return out
    keeps = torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (x, dt, A, B, C, D, bias, h0))
    return SelectiveScanFunction.apply(x, dt, A, B, C, D, bias, h0, lengths, _STEPS[step], keeps)
