"""Gated linear recurrences against the definition in 64 bits (tests/layer_reference.py), within bounds that
count roundings."""
import pytest
import torch

import paper_2510_21956_amd as la
from layer_reference import STEPS, U, half, recurrence64, recurrence_backward64, within

pytestmark = pytest.mark.gpu
GATE = {"value": la.LA_GATE_VALUE, "sigmoid": la.LA_GATE_SIGMOID}
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


def draw(B, N, C, dtype, gate, seed, spread=2.0):
    """x, gates, h0, dh, dlast on the host; every 50th row or so starts anew."""
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen)
    g = r(B, N, C) * spread + 1.0
    g[torch.rand(B, N, generator=gen) < 0.02] = -float("inf")
    if gate == "value":
        g = torch.sigmoid(g) * torch.where(torch.rand(B, N, C, generator=gen) < 0.1, -1.0, 1.0)
    td = TYPE[dtype]
    return r(B, N, C).to(td), g.to(td), r(B, C), r(B, N, C).to(td), r(B, C)


def poison(*shape, dtype):
    return torch.full(shape, float("nan"), dtype=dtype, device="cuda")


def room(x, back):
    B, N, C = x.shape
    n = la.la_recurrence_workspace_bytes(B, N, C, la.LA_F32 if x.dtype == torch.float32 else la.LA_BF16, back)
    return torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") if n else None


def forward(x, g, h0, lengths, gate, ws=None):
    h, last = poison(*x.shape, dtype=x.dtype), poison(x.shape[0], x.shape[2], dtype=torch.float32)
    la.la_recurrence_forward(x, g, h0, h, last, lengths, GATE[gate], ws if ws is not None else room(x, 0))
    return h, last


def backward(x, g, h0, h, dh, dlast, lengths, gate, ws=None):
    dx, dg = poison(*x.shape, dtype=x.dtype), poison(*x.shape, dtype=x.dtype)
    dh0 = poison(x.shape[0], x.shape[2], dtype=torch.float32)
    la.la_recurrence_backward(x, g, h0, h, dh, dlast, dx, dg, dh0, lengths, GATE[gate], ws if ws is not None else room(x, 1))
    return dx, dg, dh0


def up(*ts):
    return [None if t is None else t.cuda() for t in ts]


SHAPES = [(1, 1, 1), (2, 1, 64), (3, 2, 65), (1, 33, 2), (2, 257, 130), (2, 1000, 771), (1, 5000, 16), (5, 64, 2048),
          (1, 3001, 48), (70, 40, 3), (1, 700, 128), (2, 2049, 63), (1, 1, 5000)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gate", ["value", "sigmoid"])
@pytest.mark.parametrize("B,N,C", SHAPES)
def test_against_the_definition(B, N, C, gate, dtype):
    """Forward and backward with a state carried in and out.  The backward pass gets the reference's h, rounded
    to the stored type, so that it is compared with the formulas at the very values it reads."""
    x, g, h0, dh, dlast = draw(B, N, C, dtype, gate, B * 1000 + N + C)
    h, last = forward(*up(x, g, h0), None, gate)
    want, wlast, E, Elast = recurrence64(x, g, h0, None, gate)
    within(h, want, E, x.dtype)
    within(last, wlast, Elast, torch.float32)
    stored = want.to(x.dtype)
    got = backward(*up(x, g, h0, stored, dh, dlast), None, gate)
    dx, dg, dh0, Ex, Eg, E0 = recurrence_backward64(x, g, h0, stored, dh, dlast, None, gate)
    for a, b, e, t in zip(got, (dx, dg, dh0), (Ex, Eg, E0), (x.dtype, x.dtype, torch.float32)):
        within(a, b, e, t)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,N,C", [(65, 300, 16), (5, 500, 20), (3, 1500, 32), (2, 129, 8), (33, 17, 5), (9, 400, 4), (7, 257, 64)])
def test_heads_that_share_a_wave(B, N, C, dtype):
    """Narrow sequences side by side in a wave, some waves not full; the same with lengths, which take a wave each."""
    x, g, h0, dh, dlast = draw(B, N, C, dtype, "sigmoid", B + N + C)
    h, last = forward(*up(x, g, h0), None, "sigmoid")
    want, wlast, E, Elast = recurrence64(x, g, h0, None, "sigmoid")
    within(h, want, E, x.dtype)
    within(last, wlast, Elast, torch.float32)
    n = torch.full((B,), N, dtype=torch.int32)
    h2, last2 = forward(*up(x, g, h0), n.cuda(), "sigmoid")
    within(h2, want, E, x.dtype)
    within(last2, wlast, Elast, torch.float32)
    stored = want.to(x.dtype)
    ref = recurrence_backward64(x, g, h0, stored, dh, dlast, None, "sigmoid")
    for lengths in (None, n.cuda()):
        got = backward(*up(x, g, h0, stored, dh, dlast), lengths, "sigmoid")
        for a, b, e, t in zip(got, ref[:3], ref[3:], (x.dtype, x.dtype, torch.float32)):
            within(a, b, e, t)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gate", ["value", "sigmoid"])
@pytest.mark.parametrize("N,C,lengths", [(300, 65, [300, 0, 17, 1, 299]), (2500, 64, [1, 2500, 1300, 0, 40]), (40, 7, [0, 0, -3, 99, 5])])
def test_padded_batches(N, C, lengths, gate, dtype):
    """Rows behind a sequence's end hold NaN: none is read, zeros are written there; lengths outside 0 .. N
    are taken as the nearer of the two.  Without a carried state and its gradient."""
    x, g, _, dh, _ = draw(5, N, C, dtype, gate, N)
    n = torch.tensor(lengths, dtype=torch.int32)
    for t in (x, g, dh):
        for b, k in enumerate(lengths):
            t[b, max(0, k):] = float("nan")
    clean = [torch.nan_to_num(t) if t is not g else torch.where(torch.isnan(g), torch.zeros_like(g), g) for t in (x, g, dh)]
    h, last = forward(*up(x, g), None, n.cuda(), gate)
    want, wlast, E, Elast = recurrence64(clean[0], clean[1], None, n, gate)
    within(h, want, E, x.dtype)
    within(last, wlast, Elast, torch.float32)
    stored = want.to(x.dtype)
    held = stored.clone()
    for b, k in enumerate(lengths):
        held[b, max(0, k):] = float("nan")
    got = backward(*up(x, g, None, held, dh), None, n.cuda(), gate)
    ref = recurrence_backward64(clean[0], clean[1], None, stored, clean[2], None, n, gate)
    for a, b, e, t in zip(got, ref[:3], ref[3:], (x.dtype, x.dtype, torch.float32)):
        within(a, b, e, t)


@pytest.mark.parametrize("gate", ["value", "sigmoid"])
def test_optional_buffers(gate):
    """last and dh0 left out; a state of zeros is no state."""
    x, g, h0, dh, dlast = up(*draw(2, 900, 70, "f32", gate, 5))
    zero = torch.zeros_like(h0)
    h, last = forward(x, g, None, None, gate)
    assert torch.equal(h, forward(x, g, zero, None, gate)[0])
    h2 = poison(*x.shape, dtype=x.dtype)
    la.la_recurrence_forward(x, g, None, h2, None, None, GATE[gate], room(x, 0))
    assert torch.equal(h, h2)
    a, b = backward(x, g, None, h, dh, None, None, gate), backward(x, g, zero, h, dh, zero, None, gate)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    dx, dg = torch.empty_like(x), torch.empty_like(x)
    la.la_recurrence_backward(x, g, None, h, dh, None, dx, dg, None, None, GATE[gate], room(x, 1))
    assert torch.equal(dx, a[0]) and torch.equal(dg, a[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_infinities_and_nan_keep_to_their_channel(dtype):
    """A NaN spoils its channel from its row on and no other; a gate of -infinity starts anew after finite
    rows, +infinity keeps the state."""
    x, g, _, _, _ = draw(1, 600, 66, dtype, "sigmoid", 6)
    g = torch.where(torch.isinf(g), torch.ones_like(g), g)
    g[0, 100, :] = -float("inf")
    g[0, 200:300, :] = float("inf")
    x[0, 250, 3] = 1e30           # rows that the gate keeps out
    clean = forward(*up(x, g), None, None, "sigmoid")[0]
    assert torch.equal(clean[0, 100], x[0, 100].cuda())
    # the kept state, bit for bit inside a segment; at a segment's start it is joined from the segments' own sums,
    # P e + q: another rounding of what is kept, and each of the two is within E and half a step of it
    want, _, E, _ = recurrence64(x, g, None, None, "sigmoid")
    kept = clean[0, 200:300].double().cpu()
    room = 2 * (E[0, 200:300] + half(x.dtype) * want[0, 199].abs() * (1 + 2.0 ** -6))
    assert ((kept - kept[:1]).abs() <= room).all() and ((kept - want[0, 199]).abs() <= room).all()
    x[0, 400, 5] = float("nan")
    h = forward(*up(x, g), None, None, "sigmoid")[0]
    assert torch.isnan(h[0, 400:, 5]).all() and torch.equal(h[0, :400, 5], clean[0, :400, 5])
    keep = [c for c in range(66) if c != 5]
    assert torch.equal(h[0, :, keep], clean[0, :, keep])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gate", ["value", "sigmoid"])
@pytest.mark.parametrize("B,T,C", [(1, 1, 1), (8, 1, 2048), (3, 5, 771), (2, 8, 130)])
def test_steps_go_on_from_a_prompt(B, T, C, gate, dtype):
    """A prompt, then steps of one and of several rows: together the definition over all rows."""
    P = 100
    x, g, h0, _, _ = draw(B, P + 2 * T, C, dtype, gate, 7 + T)
    want, wlast, E, Elast = recurrence64(x, g, h0, None, gate)
    x, g, h0 = up(x, g, h0)
    h, state = forward(x[:, :P].contiguous(), g[:, :P].contiguous(), h0, None, gate)
    parts = [h]
    for cut in [(P + t, P + t + 1) for t in range(T)] + [(P + T, P + 2 * T)]:
        o = poison(B, cut[1] - cut[0], C, dtype=x.dtype)
        la.la_recurrence_step(x[:, cut[0]:cut[1]].contiguous(), g[:, cut[0]:cut[1]].contiguous(), o, state, GATE[gate])
        parts.append(o)
    within(torch.cat(parts, 1), want, E, x.dtype)
    within(state, wlast, Elast, torch.float32)


def test_offsets_beyond_32_bits():
    """More than 2^32 bytes in a tensor and more than 2^31 elements: the last sequence is that of a call of its
    own, bit for bit."""
    B, N, C = 17, 65536, 2048  # 2.28e9 elements
    x = torch.zeros((B, N, C), dtype=torch.bfloat16, device="cuda")
    g = torch.zeros_like(x)
    gen = torch.Generator(device="cuda").manual_seed(8)
    for t in (x, g):
        t[-1] = torch.randn((N, C), device="cuda", generator=gen).to(torch.bfloat16)
    h, last = forward(x, g, None, None, "sigmoid")
    back = backward(x, g, None, h, x, None, None, "sigmoid")
    # cut like the large call: as many sequences of zeros' shape is what decides, so compare by bounds of one rounding
    h1, last1 = forward(x[-1:].contiguous(), g[-1:].contiguous(), None, None, "sigmoid")
    back1 = backward(x[-1:].contiguous(), g[-1:].contiguous(), None, h1, x[-1:].contiguous(), None, None, "sigmoid")
    assert not h[:-1].any() and not last[:-1].any()
    for a, b in zip((h, *back[:2]), (h1, *back1[:2])):
        # rows cut elsewhere are other roundings of the same sums, a bfloat16 step apart at most where they are rounded
        assert ((a[-1:].float() - b.float()).abs() <= 2.0 ** -7 * b.float().abs() + 100 * STEPS * U).all()
    assert (last[-1:] - last1).abs().max() <= 100 * STEPS * U


def test_runs_repeat_bit_for_bit_and_streams_are_taken():
    x, g, h0, dh, dlast = up(*draw(2, 3000, 200, "f32", "sigmoid", 9))
    h, last = forward(x, g, h0, None, "sigmoid")
    back = backward(x, g, h0, h, dh, dlast, None, "sigmoid")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        h2, last2 = forward(x, g, h0, None, "sigmoid")
        back2 = backward(x, g, h0, h2, dh, dlast, None, "sigmoid")
    h3 = torch.empty_like(h)
    la.la_recurrence_forward(x, g, h0, h3, None, None, la.LA_GATE_SIGMOID, room(x, 0), stream=side)
    torch.cuda.synchronize()
    assert torch.equal(h, h2) and torch.equal(last, last2) and torch.equal(h, h3)
    assert all(torch.equal(a, b) for a, b in zip(back, back2))


def test_many_padded_sequences():
    """More sequences than a wave holds lengths of."""
    B, N, C = 70, 200, 66
    x, g, h0, dh, dlast = draw(B, N, C, "f32", "sigmoid", 13)
    n = (torch.arange(B) * 7 % (N + 9) - 4).to(torch.int32)
    h, last = forward(*up(x, g, h0), n.cuda(), "sigmoid")
    want, wlast, E, Elast = recurrence64(x, g, h0, n, "sigmoid")
    within(h, want, E, x.dtype)
    within(last, wlast, Elast, torch.float32)
    got = backward(*up(x, g, h0, want.float(), dh, dlast), n.cuda(), "sigmoid")
    ref = recurrence_backward64(x, g, h0, want.float(), dh, dlast, n, "sigmoid")
    for a, b, e in zip(got, ref[:3], ref[3:]):
        within(a, b, e, torch.float32)


def test_calls_side_by_side():
    """Calls on two streams at once, each with a workspace of its own, give the bits of calls that run alone."""
    sets = [up(*draw(1, 20000, 512, "bf16", "sigmoid", 14 + k)) for k in range(2)]
    alone = []
    for x, g, h0, dh, dlast in sets:
        h, last = forward(x, g, h0, None, "sigmoid")
        alone.append([h, last, *backward(x, g, h0, h, dh, dlast, None, "sigmoid")])
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[], []]
    for turn in range(5):
        for k, (x, g, h0, dh, dlast) in enumerate(sets):
            with torch.cuda.stream(streams[k]):
                h, last = forward(x, g, h0, None, "sigmoid")
                got[k] = [h, last, *backward(x, g, h0, h, dh, dlast, None, "sigmoid")]
    torch.cuda.synchronize()
    for a, b in zip(alone, got):
        assert all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("N", [1, 30, 3000])
def test_captured_calls(N):
    """Two graphs that share a workspace, replayed in turn on new inputs with eager calls in between; every
    replay gives the eager call's bits."""
    sets = [up(*draw(2, N, 130, "bf16", "sigmoid", 20 + k)) for k in range(3)]
    x, g, h0, dh, dlast = [t.clone() for t in sets[0]]
    ws = room(x, 1)
    ws = ws if ws is not None else torch.empty(256, dtype=torch.uint8, device="cuda")
    h, last = forward(x, g, h0, None, "sigmoid", ws)
    state = h0.clone()
    outs = [torch.empty_like(x), torch.empty_like(x), torch.empty_like(h0), torch.empty_like(x)]
    torch.cuda.synchronize()
    graphs = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graphs[0]):
        la.la_recurrence_forward(x, g, h0, h, last, None, la.LA_GATE_SIGMOID, ws)
        la.la_recurrence_step(x, g, outs[3], state, la.LA_GATE_SIGMOID)
    with torch.cuda.graph(graphs[1]):
        la.la_recurrence_backward(x, g, h0, h, dh, dlast, outs[0], outs[1], outs[2], None, la.LA_GATE_SIGMOID, ws)
    for k in (1, 2, 0, 1):
        for a, b in zip((x, g, h0, dh, dlast), sets[k]):
            a.copy_(b)
        state.copy_(h0)
        eh, elast = forward(*sets[k][:3], None, "sigmoid")
        eager = backward(*sets[k][:3], eh, *sets[k][3:], None, "sigmoid")
        s2, o2 = sets[k][2].clone(), torch.empty_like(x)
        la.la_recurrence_step(sets[k][0], sets[k][1], o2, s2, la.LA_GATE_SIGMOID)
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        assert torch.equal(h, eh) and torch.equal(last, elast) and torch.equal(state, s2) and torch.equal(outs[3], o2)
        assert all(torch.equal(a, b) for a, b in zip(outs, eager))


@pytest.mark.parametrize("gate", ["value", "sigmoid"])
def test_wrapper(gate):
    """gated_recurrence: other strides, a head layout, broadcast inputs and gradients, one output used alone."""
    x, g, h0, dh, dlast = draw(6, 200, 48, "f32", gate, 11)
    n = torch.tensor([200, 3, 0, 150, 77, 200], dtype=torch.int32)
    xs, gs, hs = up(x, g, h0)
    xs = xs.reshape(2, 3, 200, 48).transpose(1, 2).contiguous().transpose(1, 2).requires_grad_(True)  # [B, H, N, D] of [B, N, H, D]
    one = gs[:1].reshape(1, 1, 200, 48).clone().requires_grad_(True)                                # one gate for all
    hs = hs.reshape(2, 3, 48).clone().requires_grad_(True)
    h, last = la.gated_recurrence(xs, one.expand(2, 3, 200, 48), hs, n.cuda().reshape(2, 3), gate=gate)
    got = torch.autograd.grad([h, last], [xs, one, hs], [up(dh)[0].reshape(2, 3, 200, 48), up(dlast)[0].reshape(2, 3, 48)])
    ge = g[:1].expand(6, 200, 48)
    want, wlast, E, _ = recurrence64(x, ge, h0, n, gate)
    within(h.reshape(6, 200, 48), want, E, torch.float32)
    dx, dg, dh0, Ex, Eg, E0 = recurrence_backward64(x, ge, h0, want.float(), dh, dlast, n, gate)
    # from the device's h, half a step of float32 and its own error away from `want`
    A = (E + U * want.abs())
    Eg = Eg + torch.cat([torch.zeros(6, 1, 48), A[:, :-1].float()], 1).double() * (dx.abs() + 1) * 4
    within(got[0].reshape(6, 200, 48), dx, Ex, torch.float32)
    within(got[1].reshape(200, 48), dg.sum(0), Eg.sum(0) + 6 * U * dg.abs().sum(0), torch.float32)
    within(got[2].reshape(6, 48), dh0, E0, torch.float32)
    h, last = la.gated_recurrence(xs, one.expand(2, 3, 200, 48), gate=gate)
    ga = torch.autograd.grad(h.sum(), xs, retain_graph=True)[0]  # an expanded gradient of ones
    gb = torch.autograd.grad(h, xs, torch.ones_like(h), retain_graph=True)[0]
    assert torch.equal(ga, gb)
    gl = torch.autograd.grad(last.sum(), xs)[0]
    assert torch.isfinite(gl).all() and gl.abs().sum() > 0
    with pytest.raises(RuntimeError):  # gradients of gradients are not defined
        torch.autograd.grad(torch.autograd.grad(la.gated_recurrence(xs, xs)[0].sum(), xs, create_graph=True)[0].sum(), xs)


def test_wrapper_refuses():
    x = torch.zeros((2, 8, 16), device="cuda")
    for bad in (lambda: la.gated_recurrence(x, x[:, :4]), lambda: la.gated_recurrence(x, x.bfloat16()),
                lambda: la.gated_recurrence(x, x, x[:, 0].bfloat16()), lambda: la.gated_recurrence(x.half(), x.half()),
                lambda: la.gated_recurrence(x, x, None, torch.zeros(2, device="cuda")), lambda: la.gated_recurrence(x, x.cpu()),
                lambda: la.gated_recurrence(x[0, 0], x[0, 0]), lambda: la.gated_recurrence(x, x, gate="relu")):
        with pytest.raises((ValueError, TypeError)):
            bad()
    with pytest.raises(la.LaError):
        la.gated_recurrence(x[:, :0], x[:, :0])
