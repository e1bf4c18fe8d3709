"""Host-only checks of the short convolution and the selective scan: their formulas, and what is refused."""
import ctypes

import pytest
import torch

import paper_2510_21956_amd as la
from paper_2510_21956_amd import binding
from selective_reference import Scan64, conv64, conv_backward64
from test_binding import DeviceTensor

NULL, SHAPE, UNSUPPORTED, ALIGN, WORKSPACE, ALIAS = 1, 2, 3, 4, 5, 7


def differences(loss, inputs, grads, step=1e-5, off=1e-7):
    """grads against differences of the loss, 64 bits: errors of the step's square and of 2^-52 / step times the loss."""
    for name, t in inputs.items():
        for i in range(t.numel()):
            e = torch.zeros(t.numel(), dtype=torch.float64)
            e[i] = step
            e = e.reshape(t.shape)
            diff = (loss(**{**inputs, name: t + e}) - loss(**{**inputs, name: t - e})) / (2 * step)
            assert abs(diff - grads[name].reshape(-1)[i]) <= off, (name, i)


@pytest.mark.parametrize("act", ["silu", "none"])
@pytest.mark.parametrize("lengths", [None, [5, 0], [1, 2]])
def test_convolution_gradients_are_the_formulas(act, lengths):
    gen = torch.Generator().manual_seed(3)
    r = lambda *s: torch.randn(*s, dtype=torch.float64, generator=gen)  # noqa: E731
    B, N, C, W = 2, 5, 2, 4
    n = None if lengths is None else torch.tensor(lengths)
    ins = {"x": r(B, N, C), "w": r(C, W), "bias": r(C), "state": r(B, W - 1, C)}
    dy, dlast = r(B, N, C), r(B, W - 1, C)

    def loss(x, w, bias, state):
        y, last, _ = conv64(x, w, bias, state, n, act)
        return (y * dy).sum() + (last * dlast).sum()
    got, _ = conv_backward64(*ins.values(), dy, dlast, n, act)
    differences(loss, ins, dict(zip(ins, got)))


@pytest.mark.parametrize("step", ["softplus", "value"])
@pytest.mark.parametrize("lengths", [None, [4, 0]])
def test_scan_gradients_are_the_formulas(step, lengths):
    gen = torch.Generator().manual_seed(4)
    r = lambda *s: torch.randn(*s, dtype=torch.float64, generator=gen)  # noqa: E731
    B, N, C, S, G = 2, 4, 4, 3, 2
    n = None if lengths is None else torch.tensor(lengths)
    ins = {"x": r(B, N, C), "dt": r(B, N, C), "A": -torch.exp(r(C, S)), "Bm": r(B, N, G, S), "Cm": r(B, N, G, S), "D": r(C),
           "bias": r(C), "h0": r(B, C, S)}
    if step == "value":
        ins["dt"] = torch.exp(ins["dt"]) + 2 * ins["bias"].abs().max()
    dy, dlast = r(B, N, C), r(B, C, S)

    def loss(**t):
        s = Scan64(**t, lengths=n, step=step)
        return (s.y * dy).sum() + (s.last * dlast).sum()
    got, _ = Scan64(**ins, lengths=n, step=step).backward(dy, dlast)
    names = {"x": "x", "dt": "dt", "A": "A", "Bm": "B", "Cm": "C", "D": "D", "bias": "bias", "h0": "h0"}
    differences(loss, ins, {k: got[v] for k, v in names.items()})


# ---- refusals -----------------------------------------------------------------------------------

@pytest.fixture(scope="module")
def lib():
    return la.load_library()


def _addresses(n):
    """Made-up device addresses, far apart."""
    return [ctypes.c_void_p(0x10000000 + (k << 36)) for k in range(n)]


def test_convolution_refusals(lib):
    p = _addresses(16)
    V = ctypes.c_void_p

    def fwd(X=p[0], xs=65, W=p[1], bias=None, st=None, Y=p[2], last=None, n=None, B=2, N=300, C=65, taps=4, act=1, dt=1, wt=0):
        return lib.la_conv_forward(X, xs, W, bias, st, Y, last, n, B, N, C, taps, act, dt, wt, None)

    def bwd(X=p[0], xs=65, W=p[1], bias=None, st=None, dY=p[2], dlast=None, dX=p[3], dW=p[4], db=p[5], ds=None, n=None, B=2, N=300, C=65,
            taps=4, act=1, dt=1, wt=0, ws=p[6], size=1 << 30):
        return lib.la_conv_backward(X, xs, W, bias, st, dY, dlast, dX, dW, db, ds, n, B, N, C, taps, act, dt, wt, ws, size, None)

    def step(X=p[0], xs=65, W=p[1], bias=None, S=p[7], Y=p[2], B=2, T=1, C=65, taps=4, act=1, dt=1, wt=0):
        return lib.la_conv_step(X, xs, W, bias, S, Y, B, T, C, taps, act, dt, wt, None)
    for call, rows in ((fwd, "N"), (bwd, "N"), (step, "T")):
        for bad in ({"B": 0}, {rows: 0}, {"C": -1}, {"taps": 1}, {"taps": 9}, {"xs": 64}, {rows: (1 << 30) + 1, "B": 1},
                    {"B": 1 << 20, rows: 1 << 20}, {"B": 1 << 15, rows: 16, "C": 1 << 17, "xs": 1 << 17}):
            assert call(**bad) == SHAPE, (call, bad)
        for bad in ({"dt": 2}, {"wt": 2}, {"dt": 0, "wt": 1}, {"act": 2}, {"act": -1}):
            assert call(**bad) == UNSUPPORTED, bad
        for name in ("X", "W"):
            assert call(**{name: None}) == NULL and call(**{name: V(p[8].value + 1)}) == ALIGN
        assert call(bias=V(p[8].value + 2)) == ALIGN
    assert fwd(Y=None) == NULL and fwd(Y=V(p[2].value + 1)) == ALIGN and fwd(n=V(p[8].value + 2)) == ALIGN
    assert fwd(Y=p[0]) == ALIAS and fwd(last=p[2]) == ALIAS and fwd(st=p[8], last=p[8]) == ALIAS and fwd(W=V(p[2].value + 8)) == ALIAS
    assert fwd(xs=200, Y=V(p[0].value + 140)) == ALIAS  # beside x, within its rows' reach
    for name in ("dY", "dX"):
        assert bwd(**{name: None}) == NULL and bwd(**{name: V(p[8].value + 1)}) == ALIGN
    assert bwd(dX=p[2]) == ALIAS and bwd(dW=p[1]) == ALIAS and bwd(dlast=p[8], ds=p[8]) == ALIAS and bwd(db=V(p[5].value + 2)) == ALIGN
    for bad in ({"ws": None}, {"size": 64}, {"ws": V(p[6].value + 16)}):
        assert bwd(**bad) == WORKSPACE, bad
    assert bwd(ws=V(p[3].value + 256)) == ALIAS
    assert step(S=None) == NULL and step(Y=None) == NULL and step(S=p[0]) == ALIAS and step(Y=p[7]) == ALIAS and step(S=V(p[7].value + 1)) == ALIGN


def test_scan_refusals(lib):
    p = _addresses(24)
    V = ctypes.c_void_p

    def head(X=p[0], xs=66, Dt=p[1], ts=66, A=p[2], Bm=p[3], bs=32, Cm=p[4], cs=32, D=None, bias=None):
        return (X, xs, Dt, ts, A, Bm, bs, Cm, cs, D, bias)

    def fwd(h0=None, Y=p[5], last=None, saved=None, ss=0, n=None, B=2, N=300, C=66, S=16, G=2, step=1, dt=1, ws=p[6], size=1 << 30, **h):
        return lib.la_selective_forward(*head(**h), h0, Y, last, saved, ss, n, B, N, C, S, G, step, dt, ws, size, None)

    def bwd(saved=p[7], ss=1 << 30, dY=p[5], dlast=None, dX=p[8], dDt=p[9], dA=p[10], dB=p[11], dC=p[12], dD=None, db=None, dh0=None, n=None,
            B=2, N=300, C=66, S=16, G=2, step=1, dt=1, ws=p[6], size=1 << 30, **h):
        return lib.la_selective_backward(*head(**h), saved, ss, dY, dlast, dX, dDt, dA, dB, dC, dD, db, dh0, n, B, N, C, S, G, step, dt, ws,
                                         size, None)

    def one(state=p[7], Y=p[5], B=2, T=1, C=66, S=16, G=2, step=1, dt=1, **h):
        return lib.la_selective_step(*head(**h), state, Y, B, T, C, S, G, step, dt, None)
    for call, rows in ((fwd, "N"), (bwd, "N"), (one, "T")):
        for bad in ({"B": 0}, {rows: 0}, {"C": 0}, {"S": 0}, {"S": 129, "bs": 400, "cs": 400}, {"G": 0}, {"G": 4}, {"xs": 65}, {"ts": 0},
                    {"bs": 31}, {"cs": 31}, {"xs": 1 << 24}, {"cs": 1 << 24}, {rows: (1 << 30) + 1, "B": 1}, {"B": 1 << 20, rows: 1},
                    {"B": 1 << 19, rows: 1 << 17}):
            assert call(**bad) == SHAPE, (call, bad)
        for bad in ({"dt": 2}, {"step": 2}, {"step": -1}):
            assert call(**bad) == UNSUPPORTED, bad
        for name in ("X", "Dt", "A", "Bm", "Cm"):
            assert call(**{name: None}) == NULL and call(**{name: V(p[14].value + 1)}) == ALIGN
        assert call(D=V(p[14].value + 2)) == ALIGN and call(bias=V(p[14].value + 2)) == ALIGN
    # 300 rows of two chains are cut into segments: a workspace is needed
    assert lib.la_selective_workspace_bytes(2, 300, 66, 16, 2, 0) > 0
    for call in (fwd, bwd):
        for bad in ({"ws": None}, {"size": 0}, {"ws": V(p[6].value + 16)}):
            assert call(**bad) == WORKSPACE, bad
        assert call(n=V(p[14].value + 2)) == ALIGN
    assert fwd(Y=None) == NULL and fwd(Y=p[0]) == ALIAS and fwd(h0=p[14], last=p[14]) == ALIAS and fwd(ws=p[5]) == ALIAS
    assert fwd(saved=p[7], ss=64) == WORKSPACE and fwd(saved=V(p[7].value + 16), ss=1 << 30) == WORKSPACE and fwd(saved=p[5], ss=1 << 30) == ALIAS
    for name in ("dY", "dX", "dDt", "dB", "dC"):
        assert bwd(**{name: None}) == NULL and bwd(**{name: V(p[14].value + 1)}) == ALIGN
    assert bwd(saved=None) == WORKSPACE and bwd(ss=64) == WORKSPACE and bwd(dX=p[5]) == ALIAS and bwd(dB=p[3]) == ALIAS
    assert bwd(dA=p[2]) == ALIAS and bwd(dlast=p[14], dh0=p[14]) == ALIAS and bwd(dD=V(p[14].value + 2)) == ALIGN and bwd(dC=p[11]) == ALIAS
    assert one(state=None) == NULL and one(Y=None) == NULL and one(state=p[0]) == ALIAS and one(Y=p[7]) == ALIAS


def test_sizes_of_buffers(lib):
    assert lib.la_conv_workspace_bytes(2, 300, 65, 1) == 0 and lib.la_conv_workspace_bytes(0, 300, 65, 4) == 0
    for B, N, C, W in ((1, 1, 1, 2), (8, 2048, 2048, 4), (3, 1201, 771, 3), (1, 131072, 64, 8)):
        n = lib.la_conv_workspace_bytes(B, N, C, W)
        # a share of (W + 1) C floats for 64 rows or more of a workgroup's 512 channels, of four runs of 16 rows at least
        assert n % 256 == 0 and 0 < n <= (B * ((N + 15) // 16) + 1) * (W + 1) * C * 4 + 256
    assert lib.la_selective_workspace_bytes(1, 1, 1, 129, 1, 0) == 0 and lib.la_selective_saved_bytes(1, 0, 1, 1) == 0
    for B, N, C, S, G in ((1, 1, 1, 1, 1), (8, 2048, 2048, 16, 1), (3, 1003, 771, 20, 3), (1, 65536, 1536, 16, 1), (2, 50, 64, 128, 1)):
        kept = lib.la_selective_saved_bytes(B, N, C, S)
        assert kept % 256 == 0 and 0 <= kept - B * ((N + 15) // 16) * C * S * 4 < 256
        assert lib.la_selective_workspace_bytes(B, N, C, S, G, 0) <= B * (N // 32 + 1) * C * (S + 1) * 4 + 1024
        assert lib.la_selective_workspace_bytes(B, N, C, S, G, 1) > 0


def _stand_in(t):
    d = DeviceTensor(t)
    d.stride = t.stride
    return d


def test_row_strides():
    x = torch.zeros(3, 5, 40)
    assert binding.row_stride(x) == 40 and binding.row_stride(x[..., 3:20]) == 40 and binding.row_stride(x[:, :1, :7]) == 200
    assert binding.row_stride(x[:, 1:, :]) is None and binding.row_stride(x[..., ::2]) is None  # a gap between sequences; within rows
    assert binding.row_stride(x[:1, 1:, :]) == 40 and binding.row_stride(x[:, :1, :].expand(3, 5, 40)) is None
    assert binding.row_stride(x[..., :24].unflatten(-1, (4, 6)), 2) == 40 and binding.row_stride(x.unflatten(-1, (4, 10))[..., :6], 2) is None
    assert binding.row_stride(x.transpose(0, 1)) is None and binding.row_stride(torch.zeros(1, 1, 7)[..., :5]) == 5
    assert binding.row_stride(torch.zeros(2, 3, 8)[..., :1]) == 8


def test_binding_refuses_other_shapes_and_types(lib):
    """What the Python functions refuse before the library is asked (stand-ins for device tensors)."""
    D = lambda *s, t=torch.bfloat16: _stand_in(torch.zeros(*s, dtype=t))  # noqa: E731
    F = torch.float32
    x, w = D(2, 8, 16), D(16, 4, t=F)
    ok = (x, w, D(16, t=F), D(2, 3, 16), D(2, 8, 16), D(2, 3, 16), D(2, t=torch.int32), 1)
    for k, bad in ((0, D(16)), (0, _stand_in(torch.zeros(2, 16, 8, dtype=torch.bfloat16).transpose(1, 2))), (1, D(15, 4, t=F)), (1, D(16, t=F)),
                   (1, D(16, 4, t=torch.float16)), (1, None), (2, D(16)), (2, D(15, t=F)), (3, D(2, 4, 16)), (3, D(2, 3, 16, t=F)),
                   (4, D(2, 8, 15)), (4, None), (4, D(2, 8, 16, t=F)), (5, D(3, 16)), (6, D(2, t=F)), (6, D(3, t=torch.int32)),
                   (4, _stand_in(torch.zeros(2, 8, 32, dtype=torch.bfloat16)[..., ::2]))):
        a = list(ok)
        a[k] = bad
        with pytest.raises((ValueError, TypeError)):
            la.la_conv_forward(*a)
    with pytest.raises((ValueError, TypeError)):
        la.la_conv_step(x, w, None, None, D(2, 8, 16), 1)
    for k in (0, 5, 6, 7):
        a = [x, w, None, None, D(2, 8, 16), None, D(2, 8, 16), D(16, 4, t=F), D(16, t=F), None, None, 1, None]
        a[{0: 0, 5: 6, 6: 7, 7: 8}[k]] = D(3, 3)
        with pytest.raises((ValueError, TypeError)):
            la.la_conv_backward(*a)
    A, Bm = D(16, 4, t=F), D(2, 8, 4)
    ok = (x, D(2, 8, 16), A, Bm, D(2, 8, 4), D(16, t=F), D(16, t=F), D(2, 16, 4, t=F), D(2, 8, 16), D(2, 16, 4, t=F), None, None, 1, None)
    for k, bad in ((0, D(16)), (1, D(2, 8, 15)), (1, None), (2, D(15, 4, t=F)), (2, D(16, 4)), (2, None), (3, D(2, 8, 5)), (3, D(2, 7, 4)),
                   (3, D(2, 8, 4, t=F)), (3, None), (4, D(2, 8, 1, 4)), (4, None), (5, D(16)), (6, D(15, t=F)), (7, D(2, 4, 16, t=F)), (7, D(2, 16, 4)),
                   (8, D(2, 8, 17)), (8, None), (9, D(2, 16, t=F)), (11, D(2))):
        a = list(ok)
        a[k] = bad
        with pytest.raises((ValueError, TypeError)):
            la.la_selective_forward(*a)
    with pytest.raises((ValueError, TypeError)):
        la.la_selective_step(*ok[:7], None, D(2, 8, 16), 1)
    grads = [D(2, 8, 16), None, D(2, 8, 16), D(2, 8, 16), D(16, 4, t=F), D(2, 8, 4), D(2, 8, 4), None, None, None]  # dy .. dh0
    for k, bad in ((0, D(2, 8, 17)), (0, None), (2, None), (3, D(2, 9, 16)), (4, D(4, 16, t=F)), (5, D(2, 8, 1, 4)), (6, None), (7, D(15, t=F)),
                   (8, D(16)), (9, D(2, 16, 5, t=F)), (1, D(2, 16, 4))):
        a = list(grads)
        a[k] = bad
        with pytest.raises((ValueError, TypeError)):
            la.la_selective_backward(*ok[:7], D(1 << 16, t=torch.uint8), *a, None, 1, None)


def test_sizes_beyond_32_bits_are_refused(lib):
    """Sizes that a C int would cut off to ones the library takes."""
    D = lambda *s, t=torch.bfloat16: _stand_in(torch.empty(*s, dtype=t, device="meta"))  # noqa: E731
    F, big = torch.float32, (1 << 32) + 64
    for s in ((1, big, 1), (big, 1, 1), (1, 1, big)):
        x = D(*s)
        w, A, state = D(s[2], 4, t=F), D(s[2], 1, t=F), D(s[0], s[2], 1, t=F)
        Bm = D(s[0], s[1], 1)
        with pytest.raises(ValueError, match="2\\^31"):
            la.la_conv_forward(x, w, None, None, x, None, None, 1)
        with pytest.raises(ValueError, match="2\\^31"):
            la.la_conv_step(x, w, None, D(s[0], 3, s[2]), x, 1)
        with pytest.raises(ValueError, match="2\\^31"):
            la.la_selective_forward(x, x, A, Bm, Bm, None, None, None, x, None, None, None, 1, None)
        with pytest.raises(ValueError, match="2\\^31"):
            la.la_selective_step(x, x, A, Bm, Bm, None, None, state, x, 1)
        assert la.la_selective_workspace_bytes(*s, 1, 1, 0) == 0 and la.la_conv_workspace_bytes(*s, 4) == 0
        assert la.la_selective_saved_bytes(*s, 1) == 0


def test_wrappers_refuse_unknown_names_and_host_tensors():
    x, w, A, B = torch.zeros(2, 8, 16), torch.zeros(16, 4), torch.zeros(16, 4), torch.zeros(2, 8, 4)
    for call in (lambda: la.causal_conv(x, w, activation="gelu"), lambda: la.selective_scan(x, x, A, B, B, step="exp"),
                 lambda: la.causal_conv(x, w), lambda: la.selective_scan(x, x, A, B, B), lambda: la.selective_scan(x[0, 0], x, A, B, B)):
        with pytest.raises(ValueError):
            call()
