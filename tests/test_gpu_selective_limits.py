"""The short convolution and the selective scan where their tests against the definition do not go: long segments, layouts of many
chains, infinities, rows that lie far apart."""
import math

import pytest
import torch

import paper_2510_21956_amd as la
from layer_reference import U
from paper_2510_21956_amd import binding
from selective_reference import Scan64, conv_backward64
from test_gpu_selective import check, draw

pytestmark = pytest.mark.gpu
F = torch.float32


def poison(*shape, dtype=F):
    return torch.full(shape, float("nan"), dtype=dtype, device="cuda")


def room(n):
    return torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") if n else None


def rand(*shape, seed=0, dtype=F):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def test_states_carried_through_long_segments():
    """One state, inputs of zero, equal steps: h_t = h0 exp(A d (t + 1)) and dx_t = d B dlast exp(A d (N - 1 - t)), looked at where a
    segment starts, forward, and ends, backward.  There a value has gone through k segments, each exp(A sum d), z = A sum d = -1/4:
    the sum's 10 U, A's roundings and the product's 3 U of |z|, the exponential and the product with the state 3 U; then a row's
    exponential and the read-out's products, 8 U."""
    N, C, S, segs = 256 * 1232, 64, 1, 256
    words = la.la_selective_workspace_bytes(1, N, C, S, 1, 0) // 4
    assert words == segs * C * (S + 1)  # what a segment makes of zero states, and its sum of d
    assert la.la_selective_workspace_bytes(1, N, C, S, 1, 1) // 4 == segs * C * (2 * S + 3) + N // 16 * 64
    rows = N // segs
    d = torch.tensor(0.01)
    x, dt = torch.zeros(1, N, C, device="cuda"), d.cuda().expand(1, N, C).contiguous()
    A = torch.full((C, S), -0.25 / (0.01 * rows), device="cuda")
    Bm, Cm = rand(1, N, S, seed=1), rand(1, N, S, seed=2)
    h0, dlast = rand(1, C, S, seed=3), rand(1, C, S, seed=4)
    y, last = poison(1, N, C), poison(1, C, S)
    saved = room(la.la_selective_saved_bytes(1, N, C, S))
    la.la_selective_forward(x, dt, A, Bm, Cm, None, None, h0, y, last, saved, None, la.LA_STEP_VALUE,
                            room(la.la_selective_workspace_bytes(1, N, C, S, 1, 0)))
    z = A.double()[:, 0] * d.double().item()  # of a row
    k = torch.arange(segs, dtype=torch.float64, device="cuda").unsqueeze(1)
    allowed = (k * (13 / 4 + 3) + 8) * U
    starts = torch.arange(segs, device="cuda") * rows
    want = Cm[0, starts].double() * h0[0, :, 0].double() * torch.exp(z * (starts + 1.0).unsqueeze(1))
    assert ((y[0, starts].double() - want).abs() <= allowed * want.abs()).all()
    dx, ddt, dB, dC = poison(1, N, C), poison(1, N, C), poison(1, N, S), poison(1, N, S)
    la.la_selective_backward(x, dt, A, Bm, Cm, None, None, saved, x, dlast, dx, ddt, None, dB, dC, None, None, None, None, la.LA_STEP_VALUE,
                             room(la.la_selective_workspace_bytes(1, N, C, S, 1, 1)))
    ends = N - 1 - starts
    want = d.double().item() * Bm[0, ends].double() * dlast[0, :, 0].double() * torch.exp(z * (N - 1.0 - ends).unsqueeze(1))
    assert ((dx[0, ends].double() - want).abs() <= allowed * want.abs()).all()


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("streams", [False, True])
def test_tokens_out_of_a_long_batch(monkeypatch, native, streams):
    """One row of each of two sequences whose rows lie 2^24 elements apart, or a little less: what its copy gives, bit for bit."""
    la.load_library()
    if not native:
        monkeypatch.setattr(binding, "_native", None)
    C, S = 2048, 16
    A, D, bias = -torch.exp(rand(C, S, seed=1)), rand(C, seed=2), rand(C, seed=3)
    for rows in (8192, 8191):
        hidden = torch.empty(2, rows, C, dtype=torch.bfloat16, device="cuda")
        proj = torch.empty(2, rows * 8, 256, dtype=torch.bfloat16, device="cuda")
        x, dt, B, Cm = hidden[:, 5:6], hidden[:, 900:901], proj[:, 3:4, 7:7 + S], proj[:, 9:10, 100:100 + 2 * S].unflatten(2, (2, S))
        for k, t in enumerate((x, dt, B, Cm)):
            t.copy_(rand(*t.shape, seed=10 + k, dtype=t.dtype))
        Cm, B2 = Cm[:, :, 0], Cm
        stream = torch.cuda.Stream() if streams else None
        if streams:
            stream.wait_stream(torch.cuda.current_stream())
        for b, c in ((B, Cm), (B2, B2)):
            got = []
            for place in (lambda t: t, lambda t: t.contiguous()):
                state, y = rand(2, C, S, seed=20), poison(2, 1, C, dtype=x.dtype)
                if streams:
                    torch.cuda.current_stream().synchronize()
                la.la_selective_step(place(x), place(dt), A, place(b), place(c), D, bias, state, y, la.LA_STEP_SOFTPLUS, stream=stream)
                if streams:
                    torch.cuda.current_stream().wait_stream(stream)
                leaves = [t.detach().requires_grad_(True) for t in (x, dt, b, c)]
                z, last = la.selective_scan(*(place(t) for t in leaves[:2]), A, *(place(t) for t in leaves[2:]), D, bias, rand(2, C, S, seed=20))
                grads = torch.autograd.grad([z, last], leaves, [rand(2, 1, C, seed=21, dtype=x.dtype), rand(2, C, S, seed=22)])
                got.append([state, y, z, last, *grads])
            assert all(torch.equal(p, q) for p, q in zip(*got)) and torch.isfinite(got[0][1]).all()
            assert torch.equal(got[0][0], got[0][3])


def test_more_channels_than_a_launch_has_threads():
    """One row of 2^30 channels in all, eight taps, and the rows to carry on: 2^32 threads in two launches and more.  y is the
    last tap's product, `last` zeros and the row itself."""
    B, C, W = 2, 1 << 29, 8
    x = torch.randn(B, 1, C, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(C, W, dtype=torch.bfloat16, device="cuda")
    y = poison(B, 1, C, dtype=x.dtype)
    last = poison(B, W - 1, C, dtype=x.dtype)
    la.la_conv_forward(x, w, None, None, y, last, None, la.LA_ACT_NONE)
    assert torch.equal(y, x)
    for b in range(B):
        assert torch.equal(last[b, -1], x[b, 0])
        for j in range(W - 2):
            assert not last[b, j].any()


def test_sums_of_more_channels_than_a_launch_has():
    """dw and dbias of 2^28 channels and some more: one row's, dy x and dy."""
    C = (1 << 28) + 65
    x, dy = torch.randn(1, 1, C, device="cuda"), torch.randn(1, 1, C, device="cuda")
    w = torch.ones(C, 2, device="cuda")
    dx, dw, db = poison(1, 1, C), poison(C, 2), poison(C)
    la.la_conv_backward(x, w, None, None, dy, None, dx, dw, db, None, None, la.LA_ACT_NONE, room(la.la_conv_workspace_bytes(1, 1, C, 2)))
    assert torch.equal(dx, dy) and torch.equal(db, dy[0, 0]) and torch.equal(dw[:, 1], (x * dy)[0, 0]) and not dw[:, 0].any()


def as_defined(got, want, off, name):
    """NaN where the definition has NaN, infinities where it has them, what is finite within its bounds (where infinities spoil a
    bound, nothing is asked)."""
    got, want = got.cpu().double(), want.double()
    assert torch.equal(got.isnan(), want.isnan()), (name, "NaN", int(got.isnan().sum()), int(want.isnan().sum()))
    assert torch.equal(got == math.inf, want == math.inf) and torch.equal(got == -math.inf, want == -math.inf), name
    known = want.isfinite() & off.isfinite()
    assert ((got - want).abs() <= off + U * want.abs())[known].all(), name


INFINITE = ["x", "last x", "dt", "B", "C", "h0", "dy", "dlast"]
# places behind the last state: one piece and segments, few sequences and many
PLACES = [(2, 32, 64, 1, 1), (2, 32, 64, 3, 1), (1, 32, 64, 5, 1), (1, 48, 64, 9, 1), (1, 32, 64, 13, 1), (1, 32, 128, 20, 2), (1, 320, 64, 20, 1),
          (1, 32, 64, 40, 1), (1, 16, 64, 50, 1), (1, 16, 64, 70, 1), (1, 16, 64, 100, 1), (260, 16, 64, 14, 1)]
# lanes behind the last channel
LANES = [(2, 32, 5, 2, 1), (2, 32, 70, 3, 1), (1, 32, 66, 8, 2), (1, 48, 70, 16, 1), (1, 32, 130, 20, 2), (1, 304, 8, 20, 1), (300, 16, 8, 14, 1), (1, 16, 66, 64, 1),
         (1, 16, 66, 128, 1), (2, 192, 8, 100, 1)]
# rows behind a tile's last
ROWS = [(2, 40, 5, 1, 1), (2, 40, 70, 3, 1), (1, 19, 64, 5, 1), (1, 37, 66, 8, 2), (1, 40, 64, 9, 1), (1, 24, 64, 13, 1), (1, 33, 70, 16, 1), (1, 40, 130, 20, 2),
        (1, 300, 8, 20, 1), (1, 21, 64, 40, 1), (1, 21, 64, 50, 1), (1, 21, 66, 64, 1), (1, 19, 64, 70, 1), (1, 19, 66, 128, 1), (1, 211, 8, 100, 1)]


@pytest.mark.parametrize("what", INFINITE)
@pytest.mark.parametrize("B,N,C,S,G", PLACES + LANES + ROWS)
def test_infinities_are_those_of_the_definition(B, N, C, S, G, what):
    """One infinite value.  Everything else is positive, so that sums over states keep the infinity's sign: what has no value of its
    own, places behind the last state, lanes behind the last channel, rows behind a tile's last, must not turn it into NaN."""
    gen = torch.Generator().manual_seed(N + C + S)
    r = lambda *s: torch.rand(*s, generator=gen) + 0.5  # noqa: E731
    x, dt, A, Bm, Cm, D = r(B, N, C), r(B, N, C) / 8, -r(C, S) / 4, r(B, N, G, S), r(B, N, G, S), r(C)
    h0, dy, dlast, step = r(B, C, S), r(B, N, C), r(B, C, S), "value"
    at = {"x": (x, N // 2), "last x": (x, N - 1), "dt": (dt, N // 2), "B": (Bm, N // 2), "C": (Cm, N // 2), "dy": (dy, N // 2)}
    if what in at:
        t, row = at[what]
        t[B - 1, row].view(-1)[-1] = math.inf
    else:
        (h0 if what == "h0" else dlast)[B - 1, C - 1, S - 1] = math.inf
    ref = Scan64(x[-1:], dt[-1:], A, Bm[-1:], Cm[-1:], D, None, h0[-1:], None, step)
    dev = [t.cuda() for t in (x, dt, A, Bm, Cm, D)]
    y, last, saved = poison(B, N, C), poison(B, C, S), room(la.la_selective_saved_bytes(B, N, C, S))
    la.la_selective_forward(*dev, None, h0.cuda(), y, last, saved, None, la.LA_STEP_VALUE, room(la.la_selective_workspace_bytes(B, N, C, S, G, 0)))
    as_defined(y[-1:], ref.y, ref.Ey, "y")
    as_defined(last[-1:], ref.last, ref.Elast, "last")
    state, z = h0.cuda(), poison(B, N, C)
    la.la_selective_step(*dev, None, state, z, la.LA_STEP_VALUE)
    as_defined(z[-1:], ref.y, ref.Ey, "y in steps")
    as_defined(state[-1:], ref.last, ref.Elast, "state in steps")
    out = [poison(*s) for s in ((B, N, C), (B, N, C), (C, S), Bm.shape, Bm.shape, (C,), (C,), (B, C, S))]
    la.la_selective_backward(*dev, None, saved, dy.cuda(), dlast.cuda(), *out, None, la.LA_STEP_VALUE,
                             room(la.la_selective_workspace_bytes(B, N, C, S, G, 1)))
    want, off = ref.backward(dy[-1:], dlast[-1:])
    for k, got in zip(("x", "dt", "A", "B", "C", "D", "bias", "h0"), out):
        if got.shape[0] == B and got.dim() > 1 and k != "A":
            as_defined(got[-1:], want[k], off[k], "d" + k)
        elif B == 1:
            as_defined(got, want[k], off[k], "d" + k)


@pytest.mark.parametrize("S", [5, 16, 20])
def test_an_infinite_state_through_many_segments(S):
    """A state that is infinite stays so, however little the decays of a segment's rows leave together: exp(-5) a row."""
    N, C = 4000, 8
    ones = lambda *s: torch.ones(*s, device="cuda")  # noqa: E731
    x, A, Bm, h0 = ones(1, N, C), -ones(C, S), ones(1, N, S), ones(1, C, S)
    h0[0, 3, 1] = math.inf
    y, last = poison(1, N, C), poison(1, C, S)
    la.la_selective_forward(x, 5 * x, A, Bm, Bm, None, None, h0, y, last, None, None, la.LA_STEP_VALUE,
                            room(la.la_selective_workspace_bytes(1, N, C, S, 1, 0)))
    assert (y[0, :, 3] == math.inf).all() and last[0, 3, 1] == math.inf
    rest = [c for c in range(C) if c != 3]
    assert torch.isfinite(y[0, :, rest]).all() and int(torch.isfinite(last).sum()) == C * S - 1


@pytest.mark.parametrize("dtype", [F, torch.bfloat16])
@pytest.mark.parametrize("W", [2, 3, 4, 8])
@pytest.mark.parametrize("value", [math.inf, math.nan])
def test_weights_that_are_no_numbers_leave_padding_alone(W, dtype, value):
    """An infinite tap or one that is NaN reaches the gradients of the rows that it has a share in: padding stays zero, and of a sequence without rows
    the carried rows' gradient is what comes back."""
    N, C = 70, 9
    gen = torch.Generator().manual_seed(W)
    r = lambda *s: torch.rand(*s, generator=gen).to(dtype) + 0.5  # noqa: E731
    lengths = torch.tensor([N, 0, 1, 5, 33, 64], dtype=torch.int32)
    B = len(lengths)
    x, state, dy, dlast, w = r(B, N, C), r(B, W - 1, C), r(B, N, C), r(B, W - 1, C), r(C, W).float()
    w[2, 0] = w[4, W - 1] = w[6, W // 2] = value
    out = [poison(B, N, C, dtype=dtype), poison(C, W), poison(C), poison(B, W - 1, C, dtype=dtype)]
    la.la_conv_backward(*(t.cuda() for t in (x, w)), None, *(t.cuda() for t in (state, dy, dlast)), *out, lengths.cuda(), la.LA_ACT_NONE,
                        room(la.la_conv_workspace_bytes(B, N, C, W)))
    want, off = conv_backward64(x, w, None, state, dy, dlast, lengths, "none")
    half = 0 if dtype == F else 2.0 ** -8
    for k, got, a, e in zip(("dx", "dw", "dbias", "dstate"), out, want, off):
        as_defined(got, a, e + (half * a.abs() if k in ("dx", "dstate") else 0), k)
    for b, n in enumerate(lengths.tolist()):
        assert not out[0][b, n:].any()
    assert torch.equal(out[3][1].cpu(), dlast[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,N,C,S", [(300, 35, 8, 16), (300, 33, 8, 13), (300, 18, 8, 9), (270, 20, 66, 7), (300, 40, 5, 24), (300, 20, 8, 30), (300, 20, 8, 2)])
def test_many_short_sequences(B, N, C, S, dtype):
    """More sequences than compute units: one piece each, from the caller's states on, and four states a wave where few sequences have two."""
    assert la.la_selective_workspace_bytes(B, N, C, S, 1, 0) == 0
    lengths = torch.randint(-1, N + 2, (B,), generator=torch.Generator().manual_seed(B + S), dtype=torch.int32)
    ins = draw(B, N, C, S, 1, dtype, "softplus", S)
    check(*ins, lengths, "softplus")
    check(*ins, None, "softplus")


def serving_calls(native, monkeypatch):
    """What the calls of a serving program write, every optional argument there and missing."""
    out = []
    with monkeypatch.context() as m:
        if not native:
            m.setattr(binding, "_native", None)
        bf = torch.bfloat16
        x, w, b, n = rand(2, 20, 40, dtype=bf), rand(40, 4, seed=1), rand(40, seed=2), torch.tensor([20, 7], dtype=torch.int32, device="cuda")
        A, B, D = -torch.exp(rand(40, 6, seed=4)), rand(2, 20, 2, 6, seed=5, dtype=bf), rand(40, seed=6)
        ws = room(max(256, la.la_selective_workspace_bytes(2, 20, 40, 6, 2, 0)))
        for full in (False, True):
            y, last = poison(2, 20, 40, dtype=bf), poison(2, 3, 40, dtype=bf) if full else None
            state = rand(2, 3, 40, seed=3, dtype=bf)
            la.la_conv_forward(x, w, b if full else None, state if full else None, y, last, n if full else None, la.LA_ACT_SILU)
            token = poison(2, 2, 40, dtype=bf)
            la.la_conv_step(x[:, :2].contiguous(), w, b if full else None, state, token, la.LA_ACT_NONE if full else la.LA_ACT_SILU)
            out += [y, last, state, token]
            y, last, h = poison(2, 20, 40, dtype=bf), poison(2, 40, 6) if full else None, rand(2, 40, 6, seed=7)
            la.la_selective_forward(x, x, A, B, B, D if full else None, b if full else None, h if full else None, y, last, None, n if full else None,
                                    la.LA_STEP_SOFTPLUS, ws)
            token = poison(2, 3, 40, dtype=bf)
            part, B3 = x[:, :3].contiguous(), B[:, :3].contiguous()
            la.la_selective_step(part, part, A, B3, B3, D if full else None, b if full else None, h, token,
                                 la.LA_STEP_SOFTPLUS if full else la.LA_STEP_VALUE)
            out += [y, last, h, token]
    return out


def test_native_calls_write_what_calls_from_python_write(monkeypatch):
    la.load_library()
    assert binding._native is not None
    native, python = serving_calls(True, monkeypatch), serving_calls(False, monkeypatch)
    for k, (a, c) in enumerate(zip(native, python)):
        assert (a is None) == (c is None) and (a is None or (torch.equal(a, c) and torch.isfinite(a).all())), k


def test_native_refusals_in_the_words_of_python(monkeypatch):
    la.load_library()
    x, w, A, B, D = rand(4, 8, 16), rand(16, 4), rand(16, 5), rand(4, 8, 5), rand(16)
    none = torch.zeros((), device="cuda")

    def said():
        words = []
        for bad in (lambda: la.causal_conv(x, w[:3]), lambda: la.causal_conv(x, w, D[:2]), lambda: la.causal_conv(x, w, D, x), lambda: la.causal_conv(x, w, lengths=D),
                    lambda: la.causal_conv(x, w[:, :1]), lambda: la.causal_conv(x.half(), w), lambda: la.causal_conv(none, w), lambda: la.causal_conv(x, none),
                    lambda: la.selective_scan(x, x[:2], A, B, B), lambda: la.selective_scan(x, none, A, B, B), lambda: la.selective_scan(x, x, A, B, none),
                    lambda: la.selective_scan(x, x, A.half(), B, B), lambda: la.selective_scan(x, x, A, B, B, D, None, D),
                    lambda: la.la_conv_step(x, w, None, x, x, 1), lambda: la.la_conv_step(x, w, None, D, x, 1),
                    lambda: la.la_selective_step(x, x, A, B, B, None, None, D, x, 1), lambda: la.la_selective_step(x, x, A, B, B, D, None, rand(4, 16, 5), x[:2], 1),
                    lambda: la.la_selective_step(x, none, A, B, B, None, None, rand(4, 16, 5), x, 1)):
            with pytest.raises((ValueError, TypeError, la.LaError)) as e:
                bad()
            words.append("%s: %s" % (type(e.value).__name__, e.value))
        return words
    native = said()
    with monkeypatch.context() as m:
        m.setattr(binding, "_native", None)
        assert said() == native


def test_constants_beyond_32_bits_in_native_code():
    x, w, y = rand(2, 8, 16), rand(16, 4), poison(2, 8, 16)
    A, B, h = rand(16, 4), rand(2, 8, 4), rand(2, 16, 4)
    for value in ((1 << 32) + 1, 1 << 70):
        for call in (lambda: la.la_conv_forward(x, w, None, None, y, None, None, value), lambda: la.la_conv_step(x, w, None, rand(2, 3, 16), y, value),
                     lambda: la.la_selective_forward(x, x, A, B, B, None, None, None, y, None, None, None, value, None),
                     lambda: la.la_selective_step(x, x, A, B, B, None, None, h, y, value)):
            with pytest.raises(ValueError, match="constants"):
                call()
    assert y.isnan().all()
