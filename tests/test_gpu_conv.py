"""The short causal convolution against its definition in 64 bits (tests/selective_reference.py), within bounds that count
roundings."""
import pytest
import torch

import paper_2510_21956_amd as la
from layer_reference import within
from selective_reference import conv64, conv_backward64

pytestmark = pytest.mark.gpu
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
ACT = {"silu": la.LA_ACT_SILU, "none": la.LA_ACT_NONE}


def draw(B, N, C, W, dtype, wtype, seed):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    td, wd = TYPE[dtype], TYPE[wtype]
    return (r(B, N, C).to(td), (r(C, W) / W ** 0.5).to(wd), r(C).to(wd), r(B, W - 1, C).to(td), r(B, N, C).to(td), r(B, W - 1, C).to(td))


def up(*ts):
    return [None if t is None else t.cuda() for t in ts]


def poison(shape, dtype):
    return torch.full(tuple(shape), float("nan"), dtype=dtype, device="cuda")


def forward(x, w, bias, state, lengths, act):
    y, last = poison(x.shape, x.dtype), poison((x.shape[0], w.shape[1] - 1, x.shape[2]), x.dtype)
    la.la_conv_forward(x, w, bias, state, y, last, lengths, ACT[act])
    return y, last


def backward(x, w, bias, state, dy, dlast, lengths, act):
    F = torch.float32
    dx, dw, db = poison(x.shape, x.dtype), poison(w.shape, F), poison(w.shape[:1], F)
    ds = poison((x.shape[0], w.shape[1] - 1, x.shape[2]), x.dtype)
    ws = torch.full((la.la_conv_workspace_bytes(*x.shape, w.shape[1]),), 0xFF, dtype=torch.uint8, device="cuda")
    la.la_conv_backward(x, w, bias, state, dy, dlast, dx, dw, db, ds, lengths, ACT[act], ws)
    return dx, dw, db, ds


def check(x, w, bias, state, dy, dlast, lengths, act, on_device=None):
    n = None if lengths is None else lengths.cuda()
    xd = x.cuda() if on_device is None else on_device
    y, last = forward(xd, *up(w, bias, state), n, act)
    clean = lambda t: torch.nan_to_num(t)  # noqa: E731
    x, dy = clean(x), clean(dy)
    want, wlast, E = conv64(x, w, bias, state, lengths, act)
    within(y, want, E, x.dtype)
    assert torch.equal(last.cpu(), wlast.to(x.dtype))
    got = backward(xd, *up(w, bias, state, dy, dlast), n, act)
    ref, off = conv_backward64(x, w, bias, state, dy, dlast, lengths, act)
    F = torch.float32
    for a, b, e, t in zip(got, ref, off, (x.dtype, F, F, x.dtype)):
        within(a, b, e, t)


SHAPES = [(1, 1, 1, 2), (2, 1, 64, 4), (1, 2, 7, 8), (3, 5, 65, 3), (1, 33, 9, 5), (2, 130, 771, 4), (1, 300, 8, 6), (5, 17, 16, 7), (2, 64, 2048, 4), (1, 1000, 3, 4)]


@pytest.mark.parametrize("dtype,wtype", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("act", ["silu", "none"])
@pytest.mark.parametrize("B,N,C,W", SHAPES)
def test_against_the_definition(B, N, C, W, act, dtype, wtype):
    check(*draw(B, N, C, W, dtype, wtype, B + N + C + W), None, act)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("W", [2, 4, 8])
@pytest.mark.parametrize("N,C,lengths", [(40, 65, [40, 0, 3, 1, 39]), (200, 16, [7, 130, -4, 999, 16])])
def test_padded_batches(N, C, lengths, W, dtype):
    """Rows behind a sequence's end hold NaN: none is read, zeros are written there."""
    x, w, bias, state, dy, dlast = draw(5, N, C, W, dtype, "f32", N + W)
    for t in (x, dy):
        for b, k in enumerate(lengths):
            t[b, max(0, k):] = float("nan")
    check(x, w, bias, state, dy, dlast, torch.tensor(lengths, dtype=torch.int32), "silu")
    check(x, w, None, None, dy, None, torch.tensor(lengths, dtype=torch.int32), "none")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("W", [2, 3, 4, 5])
def test_many_channels_and_rows(W, dtype):
    """Enough of both for runs of 64 rows and more, which take more rows together; ends inside a run, and whole runs behind an end."""
    check(*draw(3, 1400, 4099, W, dtype, "f32", W), torch.tensor([1400, 1000, 37], dtype=torch.int32), "silu")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C,wide,at", [(64, 200, 3), (24, 25, 1), (5, 40, 7)])
def test_parts_of_wider_rows(C, wide, at, dtype):
    """x is read where it stands, at any element; what is beside it is not."""
    x, w, bias, state, dy, dlast = draw(2, 37, C, 4, dtype, "f32", C)
    rows = poison((2, 37, wide), x.dtype)
    rows[..., at:at + C] = x.cuda()
    check(x, w, bias, state, dy, dlast, None, "silu", rows[..., at:at + C])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,C,W", [(1, 1, 2), (3, 70, 4), (8, 2048, 4), (2, 33, 8)])
def test_steps_go_on_from_prompts(B, C, W, dtype):
    """A prompt, then steps of one and of several rows, give what one call on all rows gives, bit for bit."""
    x, w, bias, state, _, _ = draw(B, 23, C, W, dtype, "f32", C + W)
    x, w, bias, state = up(x, w, bias, state)
    want, wlast = forward(x, w, bias, state, None, "silu")
    y, last = forward(x[:, :11].contiguous(), w, bias, state, None, "silu")
    parts = [y]
    for a, b in ((11, 12), (12, 13), (13, 18), (18, 23)):
        y = poison((B, b - a, C), x.dtype)
        la.la_conv_step(x[:, a:b].contiguous(), w, bias, last, y, ACT["silu"])
        parts.append(y)
    assert torch.equal(torch.cat(parts, 1), want) and torch.equal(last, wlast)


def test_step_on_parts_of_wider_rows():
    x = torch.randn(4, 1, 300, device="cuda")
    w, state = torch.randn(100, 4, device="cuda"), torch.randn(4, 3, 100, device="cuda")
    a, b = state.clone(), state.clone()
    y, z = (poison((4, 1, 100), x.dtype) for _ in range(2))
    la.la_conv_step(x[..., 150:250], w, None, a, y, ACT["silu"])
    la.la_conv_step(x[..., 150:250].contiguous(), w, None, b, z, ACT["silu"])
    assert torch.equal(y, z) and torch.equal(a, b)


def test_infinities_stay_in_their_channel():
    """Large arguments of the activation, infinities and NaN: those rows and channels that the taps reach, none else."""
    x = torch.zeros(1, 20, 9)
    x[0, 3, 2], x[0, 5, 4], x[0, 9, 6], x[0, 2, 0], x[0, 2, 1] = float("inf"), float("nan"), -1e30, 200.0, -200.0
    w = torch.full((9, 3), 0.5)
    y, _ = forward(*up(x, w), None, None, None, "silu")
    want = conv64(x, w, None, None, None, "silu")[0]
    spoilt = torch.isnan(want) | torch.isinf(want)
    assert torch.isfinite(y.cpu())[~spoilt].all()
    assert y[0, 3:6, 2].cpu().tolist() == [float("inf")] * 3 and torch.isnan(y[0, 5:8, 4]).all()
    assert y[0, 9:12, 6].abs().max() == 0 and y[0, 2, 0] == 100.0 and abs(y[0, 2, 1]) < 1e-38
