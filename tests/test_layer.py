"""Host-only checks of the operators around the attention: their formulas, and what is refused."""
import ctypes

import pytest
import torch

import paper_2510_21956_amd as la
from layer_reference import kept64, norm64, norm_backward64, pack64, recurrence64, recurrence_backward64
from test_binding import DeviceTensor


@pytest.mark.parametrize("gate", ["value", "sigmoid"])
@pytest.mark.parametrize("lengths", [None, [5, 0]])
def test_recurrence_gradients_are_the_formulas(gate, lengths):
    """The formulas of the backward pass against differences, 64 bits: step 1e-5, errors of its square and
    of 2^-52 / 1e-5."""
    gen = torch.Generator().manual_seed(3)
    r = lambda *s: torch.randn(*s, dtype=torch.float64, generator=gen)
    B, N, C = 2, 7, 3
    x, g, h0, dh, dlast = r(B, N, C), torch.sigmoid(r(B, N, C)), r(B, C), r(B, N, C), r(B, C)
    n = None if lengths is None else torch.tensor(lengths)

    def loss(x, g, h0):
        h, last, _, _ = recurrence64(x, g, h0, n, gate)
        return (h * dh).sum() + (last * dlast).sum()
    h = recurrence64(x, g, h0, n, gate)[0]
    got = recurrence_backward64(x, g, h0, h, dh, dlast, n, gate)[:3]
    for k, (t, d) in enumerate(zip((x, g, h0), got)):
        for i in range(t.numel()):
            e = torch.zeros(t.numel(), dtype=torch.float64)
            e[i] = 1e-5
            e = e.reshape(t.shape)
            a = [x, g, h0]
            up, down = a.copy(), a.copy()
            up[k], down[k] = t + e, t - e
            diff = (loss(*up) - loss(*down)) / 2e-5
            assert abs(diff - d.reshape(-1)[i]) <= 1e-8, (k, i)


@pytest.mark.parametrize("weighted", [True, False])
def test_norm_gradients_are_the_formulas(weighted):
    gen = torch.Generator().manual_seed(4)
    r = lambda *s: torch.randn(*s, dtype=torch.float64, generator=gen).requires_grad_(True)
    s, w, dy, ds = r(5, 11), r(11), r(5, 11), r(5, 11)
    y = norm64(s, w if weighted else None, 1e-3)[0]
    want = torch.autograd.grad((y * dy).sum() + (s * ds).sum(), (s, w) if weighted else (s,))
    rstd = norm64(s, None, 1e-3)[1]
    got = norm_backward64(s, rstd, w if weighted else None, dy, ds)
    for a, b in zip(got, want):
        assert (a - b).abs().max() <= 1e-12


def test_eight_bits_by_hand():
    """The blocks of a row written out: ties to even, the largest magnitude at and above what fits, a short
    group, zeros."""
    row = torch.zeros(1, 70)
    row[0, 0], row[0, 1], row[0, 2], row[0, 3] = 448.0, 17.0, 19.0, 2.0 ** -10   # power 0: steps of 2 from 16 on
    row[0, 32], row[0, 33] = 449.0, 1.0                                        # power 1
    row[0, 64] = 1.0                                                           # 2^-8 256
    v, k = pack64(row, "e4m3")
    assert k.tolist() == [[0, 1, -8]]
    assert v[0, 0, :4].tolist() == [448.0, 16.0, 20.0, 0.0] and v[0, 1, :2].tolist() == [224.0, 0.5] and v[0, 2, 0] == 256.0
    row = torch.zeros(1, 70)
    row[0, 64] = 1.0
    row[0, 0], row[0, 1], row[0, 32], row[0, 33] = 127.0 / 64, 2.5 / 64, 128.0 / 64, 3.0 / 64
    v, k = pack64(row, "int8")
    assert k.tolist() == [[0, 1, 0]]
    assert (64 * v[0, 0, :2]).tolist() == [127.0, 2.0] and (64 * v[0, 1, :2]).tolist() == [64.0, 2.0] and 64 * v[0, 2, 0] == 64.0
    x = torch.randn(7, 100, generator=torch.Generator().manual_seed(5))
    for code in ("e4m3", "int8"):
        y = kept64(x, code)
        assert torch.equal(y, y.bfloat16().double())  # eight bits are a bfloat16
        most = torch.nn.functional.pad(x.abs(), (0, 28)).reshape(7, 4, 32).amax(2, keepdim=True).expand(-1, -1, 32)
        most = most.reshape(7, 128)[:, :100].double()
        # half a step: 1/16 of a value, or 1/128 of the group's power, which is at most its largest magnitude
        assert ((y - x.double()).abs() <= (torch.maximum(x.double().abs() / 16, most * 2.0 ** -15) if code == "e4m3"
                                           else most / 64)).all()


# ---- refusals -----------------------------------------------------------------------------------

@pytest.fixture(scope="module")
def lib():
    return la.load_library()


def _addresses(n):
    """Made-up device addresses, far apart."""
    return [ctypes.c_void_p(0x10000000 + (k << 36)) for k in range(n)]


NULL, UNSUPPORTED, SHAPE, ALIGN, WORKSPACE, ALIAS = 1, 3, 2, 4, 5, 7


def test_recurrence_refusals(lib):
    p = _addresses(12)
    V = ctypes.c_void_p

    def fwd(X=p[0], G=p[1], h0=None, H=p[2], last=None, n=None, B=2, N=300, C=65, gate=1, dt=1, ws=p[3], size=1 << 30):
        return lib.la_recurrence_forward(X, G, h0, H, last, n, B, N, C, gate, dt, ws, size, None)

    def bwd(X=p[0], G=p[1], h0=None, H=p[2], dH=p[4], dlast=None, dX=p[5], dG=p[6], dh0=None, n=None, B=2, N=300, C=65,
            gate=1, dt=1, ws=p[3], size=1 << 30):
        return lib.la_recurrence_backward(X, G, h0, H, dH, dlast, dX, dG, dh0, n, B, N, C, gate, dt, ws, size, None)

    def step(X=p[0], G=p[1], H=p[2], S=p[7], B=2, T=1, C=65, gate=1, dt=1):
        return lib.la_recurrence_step(X, G, H, S, B, T, C, gate, dt, None)
    for call in (fwd, bwd):
        for bad in ({"B": 0}, {"N": 0}, {"C": -1}, {"B": 1 << 20, "N": 1 << 20}, {"B": 1 << 23, "N": 1, "C": 1}, {"N": (1 << 30) + 1, "B": 1, "C": 1}):
            assert call(**bad) == SHAPE, bad
        for bad in ({"dt": 2}, {"dt": 7}, {"gate": 2}, {"gate": -1}):
            assert call(**bad) == UNSUPPORTED, bad
        for name in ("X", "G", "H"):
            assert call(**{name: None}) == NULL
            assert call(**{name: V(p[8].value + 1)}) == ALIGN
        assert call(h0=V(p[8].value + 2)) == ALIGN and call(n=V(p[8].value + 2)) == ALIGN
        for bad in ({"ws": None}, {"size": 0}, {"ws": V(p[3].value + 16)}):
            assert call(**bad) == WORKSPACE, bad
        assert call(ws=V(p[2].value + 256)) == ALIAS
    assert fwd(H=p[0]) == ALIAS and fwd(H=V(p[1].value + 2)) == ALIAS
    assert fwd(h0=p[8], last=p[8]) == ALIAS and fwd(n=p[2]) == ALIAS
    for name in ("dH", "dX", "dG"):
        assert bwd(**{name: None}) == NULL
    assert bwd(dX=p[4]) == ALIAS and bwd(dG=p[5]) == ALIAS and bwd(dh0=p[8], dlast=p[8]) == ALIAS
    assert bwd(dh0=V(p[8].value + 1)) == ALIGN and bwd(dlast=V(p[8].value + 1)) == ALIGN
    for bad in ({"B": 0}, {"T": 0}, {"C": 0}):
        assert step(**bad) == SHAPE
    assert step(gate=3) == UNSUPPORTED and step(dt=3) == UNSUPPORTED
    for name in ("X", "G", "H", "S"):
        assert step(**{name: None}) == NULL
    assert step(S=V(p[7].value + 2)) == ALIGN and step(H=p[0]) == ALIAS and step(S=p[1]) == ALIAS


def test_recurrence_workspace_sizes(lib):
    for bad in ((0, 1, 1, 0, 0), (1, 0, 1, 0, 0), (1, 1, 0, 0, 0), (1, 1, 1, 2, 0), (1 << 23, 1, 1, 0, 0)):
        assert lib.la_recurrence_workspace_bytes(*bad) == 0
    for B, N, C in ((1, 1, 1), (1, 131072, 2048), (64, 300, 7), (3, 5003, 771), (8, 1, 2048), (5000, 4000, 64)):
        for dt in (0, 1):
            for back in (0, 1):
                n = lib.la_recurrence_workspace_bytes(B, N, C, dt, back)
                assert n % 256 == 0 and n <= B * N * C + 65536  # a share of the tensors (9 or 11 bytes an element)


def test_rows_refusals(lib):
    p = _addresses(16)
    V = ctypes.c_void_p

    def pack(X=p[0], c=p[1], s=p[2], rows=10, C=70, dt=1, code=2):
        return lib.la_pack_rows(X, c, s, rows, C, dt, code, None)

    def unpack(X=p[0], c=p[1], s=p[2], rows=10, C=70, dt=1, code=2):
        return lib.la_unpack_rows(c, s, X, rows, C, code, dt, None)
    for call in (pack, unpack):
        assert call(rows=0) == SHAPE and call(C=0) == SHAPE and call(rows=1 << 30, C=1 << 20) == SHAPE
        assert call(dt=2) == UNSUPPORTED and call(code=0) == UNSUPPORTED and call(code=4) == UNSUPPORTED
        for name in "Xcs":
            assert call(**{name: None}) == NULL
        assert call(X=V(p[0].value + 1)) == ALIGN
        assert call(X=V(p[1].value + 600)) == ALIAS and call(s=p[0]) == ALIAS

    def fwd(X=p[0], R=None, W=p[1], Y=p[2], Ys=None, S=None, K=None, Ks=None, rstd=p[3], rows=10, C=70, dt=1, wt=0, yt=1,
            kt=2):
        return lib.la_rmsnorm_forward(X, R, W, Y, Ys, S, K, Ks, rstd, rows, C, 1e-6, dt, wt, yt, kt, None)
    assert fwd(rows=0) == SHAPE and fwd(C=0) == SHAPE and fwd(C=16385) == SHAPE
    assert fwd(dt=2) == UNSUPPORTED and fwd(wt=2) == UNSUPPORTED and fwd(dt=0, yt=0, wt=1) == UNSUPPORTED
    assert fwd(yt=0) == UNSUPPORTED and fwd(K=p[4], Ks=p[5], kt=1) == UNSUPPORTED
    for bad in ({"X": None}, {"Y": None}, {"R": p[4]}, {"S": p[4]}, {"K": p[4]}, {"Ks": p[4]}, {"Ys": p[4]}, {"yt": 2}):
        assert fwd(**bad) == NULL, bad
    assert fwd(X=V(p[0].value + 1)) == ALIGN and fwd(W=V(p[1].value + 2)) == ALIGN and fwd(rstd=V(p[3].value + 2)) == ALIGN
    assert fwd(Y=p[0]) == ALIAS and fwd(R=p[4], S=p[0]) == ALIAS and fwd(R=p[4], S=V(p[4].value + 2)) == ALIAS
    assert fwd(W=p[2]) == ALIAS and fwd(rstd=p[2]) == ALIAS

    def bwd(S=p[0], Ss=None, W=p[1], rstd=p[3], dY=p[4], dS=None, dX=p[5], dW=p[6], rows=10, C=70, dt=1, wt=0, st=1, ws=p[7],
            size=1 << 20):
        return lib.la_rmsnorm_backward(S, Ss, W, rstd, dY, dS, dX, dW, rows, C, dt, wt, st, ws, size, None)
    assert bwd(rows=0) == SHAPE and bwd(C=16385) == SHAPE and bwd(dt=3) == UNSUPPORTED and bwd(st=0) == UNSUPPORTED
    for bad in ({"S": None}, {"rstd": None}, {"dY": None}, {"dX": None}, {"st": 2}, {"Ss": p[8]}, {"W": None}):
        assert bwd(**bad) == NULL, bad
    for bad in ({"ws": None}, {"size": 64}, {"ws": V(p[7].value + 16)}):
        assert bwd(**bad) == WORKSPACE, bad
    assert bwd(dX=p[4]) == ALIAS and bwd(dX=p[0]) == ALIAS and bwd(dW=p[1]) == ALIAS and bwd(ws=V(p[5].value - 256)) == ALIAS
    assert bwd(dY=V(p[4].value + 1)) == ALIGN and bwd(dW=V(p[6].value + 2)) == ALIGN
    assert lib.la_rmsnorm_workspace_bytes(0, 5) == 0 and lib.la_rmsnorm_workspace_bytes(5, 16385) == 0
    assert 0 < lib.la_rmsnorm_workspace_bytes(1 << 29, 1024) <= 1 << 24


def test_binding_refuses_other_shapes_and_types(lib):
    """What the Python functions refuse before the library is asked (stand-ins for device tensors)."""
    D = lambda *s, t=torch.bfloat16: DeviceTensor(torch.zeros(*s, dtype=t))
    F = torch.float32
    x, st = D(2, 8, 16), D(2, 16, t=F)
    ok = (x, D(2, 8, 16), None, D(2, 8, 16), st, None, 1, None)
    for k, bad in ((1, D(2, 8, 15)), (1, D(2, 8, 16, t=F)), (3, D(8, 2, 16)), (2, D(2, 16)), (2, D(2, 15, t=F)), (4, D(16, t=F)),
                   (5, D(2, t=F)), (5, D(3, t=torch.int32)), (1, None), (3, None),
                   (1, DeviceTensor(torch.zeros(2, 16, 8, dtype=torch.bfloat16).transpose(1, 2)))):
        a = list(ok)
        a[k] = bad
        with pytest.raises((ValueError, TypeError)):
            la.la_recurrence_forward(*a)
    with pytest.raises(TypeError):
        la.la_recurrence_step(D(2, 8, 16, t=torch.float16), D(2, 8, 16, t=torch.float16), D(2, 8, 16, t=torch.float16), st, 0)
    with pytest.raises(ValueError):
        la.la_recurrence_backward(x, x, None, x, None, None, x, x, None, None, 0, None)
    with pytest.raises(ValueError):
        la.la_recurrence_step(D(16), D(16), D(16), D(16, t=F), 0)  # no rows
    r, c, s = D(4, 70), D(4, 70, t=torch.uint8), D(4, 3, t=torch.uint8)
    for a in ((r, D(4, 70), s, 2), (r, c, D(4, 2, t=torch.uint8), 2), (r, c, s, 0), (r, c, None, 2), (D(4, 70, t=torch.float16), c, s, 3)):
        with pytest.raises((ValueError, TypeError)):
            la.la_pack_rows(*a)
    w, rs = D(70, t=F), D(4, t=F)
    for a in ((r, r, w, r, None, None, None, None, rs, 1e-6), (r, None, D(69), r, None, None, None, None, rs, 1e-6),
              (r, None, D(70, t=torch.float16), r, None, None, None, None, rs, 1e-6),
              (r, None, w, r, s, None, None, None, rs, 1e-6), (r, None, w, r, None, None, c, s, rs, 1e-6),
              (r, None, w, r, None, None, None, None, D(5, t=F), 1e-6), (r, None, w, r, s, None, None, None, rs, 1e-6, 2)):
        with pytest.raises((ValueError, TypeError)):
            la.la_rmsnorm_forward(*a)
    for a in ((r, None, w, rs, D(4, 71), None, r, None, None), (r, s, w, rs, r, None, r, None, None),
              (c, s, w, rs, r, None, r, None, None), (r, None, None, rs, r, None, r, w, None),
              (r, None, w, rs, r, None, r, D(70), None), (r, None, w, None, r, None, r, None, None)):
        with pytest.raises((ValueError, TypeError)):
            la.la_rmsnorm_backward(*a)


def test_sizes_beyond_32_bits_are_refused(lib):
    """Sizes that a C int would cut off to ones the library takes."""
    D = lambda *s, t=torch.bfloat16: DeviceTensor(torch.empty(*s, dtype=t, device="meta"))
    F, big = torch.float32, (1 << 32) + 64
    for s in ((1, big, 1), (big, 1, 1), (1, 1, big)):
        x, state = D(*s), D(s[0], s[2], t=F)
        with pytest.raises(ValueError, match="2\\^31"):
            la.la_recurrence_forward(x, x, None, x, state, None, 1, None)
        with pytest.raises(ValueError, match="2\\^31"):
            la.la_recurrence_backward(x, x, None, x, x, None, x, x, None, None, 1, None)
        with pytest.raises(ValueError, match="2\\^31"):
            la.la_recurrence_step(x, x, x, state, 1)
        assert la.la_recurrence_workspace_bytes(*s, la.LA_BF16, 0) == 0
    x, rs, powers, codes = D(1, big), D(1, t=F), D(1, big // 32, t=torch.uint8), D(1, big, t=torch.uint8)
    for call in (lambda: la.la_pack_rows(x, codes, powers, la.LA_I8), lambda: la.la_unpack_rows(codes, powers, x, la.LA_I8),
                 lambda: la.la_pack_tensors([x], [codes], [powers], la.LA_I8),
                 lambda: la.la_rmsnorm_forward(x, None, None, x, None, None, None, None, rs, 1e-6),
                 lambda: la.la_rmsnorm_backward(x, None, None, rs, x, None, x, None, None)):
        with pytest.raises(ValueError, match="2\\^31"):
            call()
    assert la.la_rmsnorm_workspace_bytes(1, big) == 0


def test_wrappers_refuse_unknown_names():
    x = torch.zeros(2, 8, 16)
    for call in (lambda: la.gated_recurrence(x, x, gate="tanh"), lambda: la.rms_norm(x, checkpoint="int4"),
                 lambda: la.rms_norm_quantised(x, code="bf16"), lambda: la.pack_rows(x, "fp8"),
                 lambda: la.linear_attention(x, x, x, checkpoint="fp8")):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: la.gated_recurrence(x, x), lambda: la.rms_norm(x), lambda: la.pack_rows(x, "int8"),
                 lambda: la.rms_norm_quantised(x)):  # host tensors: there is no fallback
        with pytest.raises(ValueError):
            call()
