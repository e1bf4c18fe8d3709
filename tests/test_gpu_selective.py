"""The selective scan against its definition in 64 bits (tests/selective_reference.py), within bounds that count
roundings."""
import math

import pytest
import torch

import paper_2510_21956_amd as la
from layer_reference import within
from selective_reference import Scan64

pytestmark = pytest.mark.gpu
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
STEP = {"softplus": la.LA_STEP_SOFTPLUS, "value": la.LA_STEP_VALUE}
F = torch.float32


def draw(B, N, C, S, G, dtype, step, seed, fast=1.0):
    """x, dt, A, Bm, Cm, D, bias, h0, dy, dlast on the host; decays from nearly 1 to nearly 0."""
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    td = TYPE[dtype]
    dt = r(B, N, C) * 2
    bias = r(C) - 2
    if step == "value":
        dt, bias = torch.exp(dt - 3), None
    A = -torch.exp(r(C, S)) * fast
    return (r(B, N, C).to(td), dt.to(td), A, r(B, N, G, S).to(td), r(B, N, G, S).to(td), r(C), bias, r(B, C, S), r(B, N, C).to(td), r(B, C, S))


def up(*ts):
    return [None if t is None else t.cuda() for t in ts]


def poison(shape, dtype):
    return torch.full(tuple(shape), float("nan"), dtype=dtype, device="cuda")


def room(n):
    return torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") if n else None


def forward(x, dt, A, Bm, Cm, D, bias, h0, lengths, step, keeps=True):
    B, N, C = x.shape
    S, G = A.shape[1], Bm.shape[2]
    y, last = poison(x.shape, x.dtype), poison((B, C, S), F)
    saved = room(la.la_selective_saved_bytes(B, N, C, S)) if keeps else None
    la.la_selective_forward(x, dt, A, Bm, Cm, D, bias, h0, y, last, saved, lengths, STEP[step],
                            room(la.la_selective_workspace_bytes(B, N, C, S, G, 0)))
    return y, last, saved


def backward(x, dt, A, Bm, Cm, D, bias, saved, dy, dlast, lengths, step):
    B, N, C = x.shape
    S, G = A.shape[1], Bm.shape[2]
    out = {"x": poison(x.shape, x.dtype), "dt": poison(x.shape, x.dtype), "A": poison(A.shape, F), "B": poison(Bm.shape, x.dtype),
           "C": poison(Bm.shape, x.dtype), "D": poison((C,), F), "bias": poison((C,), F), "h0": poison((B, C, S), F)}
    la.la_selective_backward(x, dt, A, Bm, Cm, D, bias, saved, dy, dlast, out["x"], out["dt"], out["A"], out["B"], out["C"], out["D"],
                             out["bias"], out["h0"], lengths, STEP[step], room(la.la_selective_workspace_bytes(B, N, C, S, G, 1)))
    return out


def check(x, dt, A, Bm, Cm, D, bias, h0, dy, dlast, lengths, step, place=lambda t: t.cuda()):
    n = None if lengths is None else lengths.cuda()
    ins = [place(t) for t in (x, dt)] + up(A) + [place(t) for t in (Bm, Cm)] + up(D, bias)
    y, last, saved = forward(*ins, *up(h0), n, step)
    x, dt, Bm, Cm, dz = (torch.nan_to_num(t) for t in (x, dt, Bm, Cm, dy))
    ref = Scan64(x, dt, A, Bm, Cm, D, bias, h0, lengths, step)
    within(y, ref.y, ref.Ey, x.dtype)
    within(last, ref.last, ref.Elast, F)
    got = backward(*ins, saved, *up(dy, dlast), n, step)
    want, off = ref.backward(dz, dlast)
    for k in ("x", "dt", "A", "B", "C", "D", "bias", "h0"):
        try:
            within(got[k], want[k], off[k], got[k].dtype)
        except AssertionError as e:
            raise AssertionError((k, *e.args)) from None
    y2, last2, _ = forward(*ins, *up(h0), n, step, keeps=False)
    assert torch.equal(y, y2) and torch.equal(last, last2)


SHAPES = [(1, 1, 1, 1, 1), (2, 1, 64, 16, 1), (3, 2, 65, 4, 1), (1, 33, 2, 16, 2), (2, 257, 130, 16, 1), (1, 100, 771, 20, 3), (1, 700, 16, 8, 1),
          (2, 64, 320, 16, 5), (1, 50, 48, 64, 1), (2, 31, 70, 33, 1), (1, 40, 66, 128, 1), (1, 47, 20, 90, 2), (2, 18, 64, 9, 1), (1, 60, 10, 30, 1), (1, 17, 5, 1, 1)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("step", ["softplus", "value"])
@pytest.mark.parametrize("B,N,C,S,G", SHAPES)
def test_against_the_definition(B, N, C, S, G, step, dtype):
    check(*draw(B, N, C, S, G, dtype, step, B * 1000 + N + C + S), None, step)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,C,S,G", [(40, 65, 16, 1), (300, 12, 5, 3)])
def test_padded_batches(N, C, S, G, dtype):
    """Rows behind a sequence's end hold NaN: none is read, zeros are written there; lengths outside 0 .. N are taken as the
    nearer of the two."""
    lengths = [N, 0, 17, 1, N - 1, -3, N + 99]
    x, dt, A, Bm, Cm, D, bias, h0, dy, dlast = draw(7, N, C, S, G, dtype, "softplus", N)
    for t in (x, dt, Bm, Cm, dy):
        for b, k in enumerate(lengths):
            t[b, max(0, k):] = float("nan")
    n = torch.tensor(lengths, dtype=torch.int32)
    check(x, dt, A, Bm, Cm, D, bias, h0, dy, dlast, n, "softplus")
    check(x, dt, A, Bm, Cm, None, None, None, dy, None, n, "softplus")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_parts_of_wider_rows(dtype):
    def place(t):
        flat = t.reshape(*t.shape[:2], -1)
        rows = poison((*flat.shape[:2], flat.shape[2] + 21), t.dtype)
        rows[..., 5:5 + flat.shape[2]] = flat.cuda()
        return rows[..., 5:5 + flat.shape[2]].unflatten(-1, t.shape[2:])
    check(*draw(2, 70, 66, 12, 2, dtype, "softplus", 5), None, "softplus", place)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,C,S,G", [(1, 1, 1, 1), (3, 70, 16, 1), (2, 48, 5, 3), (2, 130, 64, 1), (1, 9, 128, 1), (8, 2048, 16, 1)])
def test_steps_go_on_from_prompts(B, C, S, G, dtype):
    """A prompt, then steps of one and of several rows, against one call on all rows in 64 bits."""
    x, dt, A, Bm, Cm, D, bias, h0, _, _ = draw(B, 23, C, S, G, dtype, "softplus", C + S)
    ref = Scan64(x, dt, A, Bm, Cm, D, bias, h0, None, "softplus")
    x, dt, A, Bm, Cm, D, bias, h0 = up(x, dt, A, Bm, Cm, D, bias, h0)
    cut = lambda a, b: [t[:, a:b].contiguous() for t in (x, dt)] + [A] + [t[:, a:b].contiguous() for t in (Bm, Cm)] + [D, bias]  # noqa: E731
    y, state, _ = forward(*cut(0, 11), h0, None, "softplus", keeps=False)
    parts = [y]
    for a, b in ((11, 12), (12, 13), (13, 18), (18, 23)):
        y = poison((B, b - a, C), x.dtype)
        la.la_selective_step(*cut(a, b), state, y, STEP["softplus"])
        parts.append(y)
    within(torch.cat(parts, 1), ref.y, ref.Ey, x.dtype)
    within(state, ref.last, ref.Elast, F)


@pytest.mark.parametrize("step", ["softplus", "value"])
def test_extremes(step):
    """Steps from far below to far above what is usual, a decay to exactly nothing, none at all."""
    x, dt, A, Bm, Cm, D, bias, h0, dy, dlast = draw(1, 40, 70, 16, 1, "f32", step, 8)
    dt = dt.clone()
    dt[0, 5], dt[0, 9], dt[0, 12], dt[0, 20] = (-30.0, 25.0, -100.0, 90.0) if step == "softplus" else (1e-12, 25.0, 0.0, 90.0)
    A[:, 3] = 0.0
    A[:, 4] = -1e4
    check(x, dt, A, Bm, Cm, D, bias, h0, dy, dlast, None, step)


@pytest.mark.parametrize("N", [40, 700])
def test_decays_to_nothing_at_once(N):
    """A of minus infinity forgets the state at every row and, like any other, leaves it alone behind a sequence's end:
    the same bits as with a decay that is as good as that."""
    x, dt, A, Bm, Cm, D, bias, h0, dy, dlast = draw(4, N, 70, 16, 1, "f32", "softplus", N)
    n = torch.tensor([N, 17, 0, N - 30], dtype=torch.int32).cuda()
    results = []
    for low in (-float("inf"), -1e30):
        A[:, 5] = low
        A[3, :] = low
        ins = up(x, dt, A, Bm, Cm, D, bias)
        y, last, saved = forward(*ins, *up(h0), n, "softplus")
        got = backward(*ins, saved, *up(dy, dlast), n, "softplus")
        state, z = last.clone(), poison((4, 1, 70), F)
        la.la_selective_step(*[t[:, :1].contiguous() for t in ins[:2]], ins[2], *[t[:, :1].contiguous() for t in ins[3:5]], *ins[5:], state, z,
                             la.LA_STEP_SOFTPLUS)
        results.append([y, last, state, z, *got.values()])
    for a, b in zip(*results):
        assert torch.isfinite(a).all() and torch.equal(a, b)


@pytest.mark.parametrize("S", [2, 4, 13, 24, 30, 40, 60, 90, 128])
def test_segments_of_every_number_of_states(S):
    """Few channels and many rows, which are walked in segments, one sequence ending inside one."""
    check(*draw(2, 333, 20, S, 1, "f32", "softplus", S), torch.tensor([333, 170], dtype=torch.int32), "softplus")
