"""The norm with the residual's addition and rows in 8 bits, against their definitions in 64 bits
(tests/layer_reference.py)."""
import pytest
import torch

import paper_2510_21956_amd as la
from layer_reference import U, half, kept64, norm64, norm_backward64, pack64, within

pytestmark = pytest.mark.gpu
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
CODE = {"e4m3": la.LA_E4M3, "int8": la.LA_I8}
EPS = 1e-6


def draw(rows, C, dtype, seed):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen)
    big = torch.exp(r(C))
    return [t.to(TYPE[dtype]) for t in (r(rows, C) * big, r(rows, C) * big * 2, r(rows, C), r(rows, C))] + [1 + 0.1 * r(C)]


def poison(*shape, dtype):
    return torch.full(shape, float("nan"), dtype=dtype, device="cuda")


def bytes_like(x):
    C = x.shape[-1]
    return (torch.full(x.shape, 0x55, dtype=torch.uint8, device="cuda"),
            torch.full((*x.shape[:-1], -(-C // 32)), 0x55, dtype=torch.uint8, device="cuda"))


def values(codes, code):
    return codes.view(torch.float8_e4m3fn).double() if code == "e4m3" else codes.view(torch.int8).double() / 64


def same_bits(codes, scales, x, code):
    """Codes and powers are those of the definition; what does not fit in a finite group is compared as NaN."""
    v, k = pack64(x, code)
    C = x.shape[1]
    assert torch.equal(scales.cpu().long(), k + 127)
    fine = (k < 128).unsqueeze(2).expand_as(v).reshape(x.shape[0], -1)[:, :C]
    v = v.reshape(x.shape[0], -1)[:, :C]
    assert torch.equal(values(codes.cpu(), code)[fine], v[fine])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("code", ["e4m3", "int8"])
@pytest.mark.parametrize("rows,C", [(1, 1), (3, 7), (2, 16), (5, 32), (1, 33), (300, 64), (77, 771), (9, 2048), (3, 16385), (2000, 128)])
def test_pack_and_unpack(rows, C, code, dtype):
    x = draw(rows, C, dtype, rows + C)[0]
    x[0, 0] = 0.0
    x[-1] = 0.0
    codes, scales = bytes_like(x)
    la.la_pack_rows(x.cuda(), codes, scales, CODE[code])
    same_bits(codes, scales, x, code)
    for td in (torch.float32, torch.bfloat16):
        back = poison(rows, C, dtype=td)
        la.la_unpack_rows(codes, scales, back, CODE[code])
        assert torch.equal(back.double().cpu(), kept64(x, code))


@pytest.mark.parametrize("code", ["e4m3", "int8"])
def test_pack_over_the_whole_range(code):
    """Magnitudes from subnormal to the largest float, ties, the borders of a power, infinities and NaN."""
    gen = torch.Generator().manual_seed(1)
    e = torch.arange(-149, 128).double()
    x = (2.0 ** e).unsqueeze(1) * (1 + torch.rand(277, 32, generator=gen).double())
    x[:, 0] = 2.0 ** e * (1.75 if code == "e4m3" else 127 / 64)      # the largest that fits
    x[::2, 1] = torch.nextafter(x[::2, 0].float(), torch.tensor(float("inf"))).double()  # and just above
    x[:, 2] = 2.0 ** e * (17 / 16)                                    # a tie
    x = x.clamp(max=torch.finfo(torch.float32).max).float()
    x[:, ::3] *= -1
    codes, scales = bytes_like(x)
    la.la_pack_rows(x.cuda(), codes, scales, CODE[code])
    same_bits(codes, scales, x, code)
    back = poison(277, 32, dtype=torch.float32)
    la.la_unpack_rows(codes, scales, back, CODE[code])
    want = kept64(x, code)
    normal = (want.abs() >= 2.0 ** -126) | (want == 0)
    # e4m3: from 1.9375 2^127 on, four bits round to 2^128, which is no float: float() makes it an infinity
    assert torch.equal(back.double().cpu()[normal], want[normal].float().double())
    x = torch.ones(4, 100)
    x[0, 40], x[1, 99], x[2, 0] = float("nan"), float("inf"), -float("inf")
    codes, scales = bytes_like(x)
    la.la_pack_rows(x.cuda(), codes, scales, CODE[code])
    la.la_unpack_rows(codes, scales, back := poison(4, 100, dtype=torch.float32), CODE[code])
    bad = torch.zeros(4, 100, dtype=torch.bool)
    bad[0, 32:64], bad[1, 96:], bad[2, :32] = True, True, True
    assert torch.isnan(back.cpu()[bad]).all() and (back.cpu()[~bad] == 1).all()


def norm_bound(s, y, C, dtype):
    """y's roundings: the mean of C squares C U (halved by the root), the root, the quotient and the products 6."""
    return (C / 2 + 6) * U * y.abs()


SHAPES = [(1, 1), (3, 7), (5, 64), (33, 65), (17, 128), (9, 200), (300, 256), (7, 500), (4, 771), (5, 1024), (600, 96), (2, 2048),
          (3, 2500), (2, 4096), (3, 8192), (2, 9000), (1, 16384), (700, 1000)]


@pytest.mark.parametrize("dtype,weight", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("bf16", None)])
@pytest.mark.parametrize("rows,C", SHAPES)
def test_norm_against_the_definition(rows, C, dtype, weight):
    """With and without a residual, forward and backward, the saved sum as it is and in 8 bits."""
    x, r, dy, ds, w = draw(rows, C, dtype, rows * 3 + C)
    td = TYPE[dtype]
    w = None if weight is None else w.to(TYPE[weight])
    wd = None if w is None else w.cuda()
    for res in (None, r):
        s = x if res is None else (x.double() + res.double()).to(td)
        want, rstd = norm64(s, w, EPS)
        y, total = poison(rows, C, dtype=td), None if res is None else poison(rows, C, dtype=td)
        inv = poison(rows, dtype=torch.float32)
        kept, ks = bytes_like(x)
        la.la_rmsnorm_forward(x.cuda(), None if res is None else res.cuda(), wd, y, None, total, kept, ks, inv, EPS, None,
                              la.LA_I8)
        within(y, want, norm_bound(s, want, C, td), td)
        within(inv, rstd[:, 0], (C / 2 + 4) * U * rstd[:, 0], torch.float32)
        if res is not None:
            assert torch.equal(total.cpu(), s)
        same_bits(kept, ks, s, "int8")
        for code in (None, "int8"):
            saved = s.double() if code is None else kept64(s, code)
            args = (s.cuda(), None) if code is None else (kept, ks)
            dx, dw = poison(rows, C, dtype=td), None if w is None else poison(C, dtype=torch.float32)
            ws = torch.full((la.la_rmsnorm_workspace_bytes(rows, C),), 0xFF, dtype=torch.uint8, device="cuda")
            la.la_rmsnorm_backward(*args, wd, inv, dy.cuda(), None if res is None else ds.cuda(), dx, dw, ws,
                                   None if code is None else CODE[code])
            wx, ww, Ex, Ew = norm_backward64(saved, rstd, w, dy, None if res is None else ds)
            within(dx, wx, Ex, td)
            if w is not None:
                within(dw, ww, Ew, torch.float32)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("code", ["e4m3", "int8"])
@pytest.mark.parametrize("rows,C", [(1, 8), (7, 100), (300, 64), (33, 771), (5, 2048), (3, 4096), (2, 12345)])
def test_norm_into_eight_bits(rows, C, code, dtype):
    """The codes stand for y within half a step of the 8 bits (1/16 of a value, or of the smallest normal code;
    1/128 of the power); a power may be the next one where the largest magnitude of a group lies within y's own
    error of a border."""
    x, r, _, _, w = draw(rows, C, dtype, C)
    s = (x.double() + r.double()).to(TYPE[dtype])
    want, _ = norm64(s, w, EPS)
    E = norm_bound(s, want, C, torch.float32)
    codes, scales, total = la.rms_norm_quantised(x.cuda(), w.cuda() if dtype == "f32" else w.cuda(), r.cuda(), eps=EPS, code=code)
    assert torch.equal(total.cpu(), s)
    assert codes.dtype == (torch.float8_e4m3fn if code == "e4m3" else torch.int8) and scales.dtype == torch.float8_e8m0fnu
    power = scales.view(torch.uint8).cpu().double() - 127
    wide = power.repeat_interleave(32, 1)[:, :C]
    got = values(codes.view(torch.uint8).cpu(), code) * 2.0 ** wide
    step = torch.maximum(want.abs() / 16, 2.0 ** (wide - 10)) if code == "e4m3" else 2.0 ** (wide - 7)
    assert ((got - want).abs() <= step * (1 + 1e-6) + E).all()
    lo, hi = pack64(want.abs() - E, code)[1], pack64(want.abs() + E, code)[1]
    assert ((power >= lo) & (power <= hi)).all()
    again = la.rms_norm_quantised(x.cuda(), w.cuda(), r.cuda(), eps=EPS, code=code)
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip((codes, scales), again))


def test_rows_at_odd_addresses_and_in_place():
    """Tensors that start at any element; the residual's own buffer as the sum's."""
    x, r, dy, ds, w = draw(40, 771, "bf16", 3)
    big = [torch.zeros(40 * 771 + 9, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    X, R, Y = (b[k:k + 40 * 771].view(40, 771) for b, k in zip(big, (1, 3, 5)))
    X.copy_(x)
    R.copy_(r)
    y, total = la.rms_norm(x.cuda(), w.cuda(), r.cuda())
    la.la_rmsnorm_forward(X, R, w.cuda(), Y, None, R, None, None, None, EPS)
    assert torch.equal(Y, y) and torch.equal(R, total)
    assert not big[2][:5].any() and not big[2][5 + 40 * 771:].any()  # nothing written around the rows


def test_zero_rows_and_nan():
    x = torch.zeros(3, 100)
    x[1, 7] = float("nan")
    x[2] = 1.0
    y = la.rms_norm(x.cuda(), eps=1e-6).cpu()
    assert not y[0].any() and torch.isnan(y[1]).all() and (y[2] - 1).abs().max() < 1e-6


def test_many_short_rows():
    """More rows than workgroups take in one round, and 2^31 elements."""
    x = torch.randn((1 << 20, 64), device="cuda", dtype=torch.bfloat16, generator=torch.Generator(device="cuda").manual_seed(1))
    y = la.rms_norm(x)
    some = torch.arange(0, 1 << 20, 65537)
    want, _ = norm64(x[some].cpu(), None, EPS)
    within(y[some], want, norm_bound(None, want, 64, torch.bfloat16), torch.bfloat16)
    wide = torch.zeros((140000, 16384), device="cuda", dtype=torch.bfloat16)
    wide[-1] = torch.randn(16384, device="cuda")
    y = la.rms_norm(wide)
    want, _ = norm64(wide[-1:].cpu(), None, EPS)
    within(y[-1:], want, norm_bound(None, want, 16384, torch.bfloat16), torch.bfloat16)
    assert not y[:-1].any()
    codes, scales = la.pack_rows(wide, "int8")
    assert torch.equal(la.unpack_rows(codes[-1:], scales[-1:], "int8", torch.float32).double().cpu(), kept64(wide[-1:].float().cpu(), "int8"))


@pytest.mark.parametrize("checkpoint", [None, "e4m3", "int8"])
def test_norm_wrapper(checkpoint):
    """rms_norm: gradients of a broadcast residual, of other strides, of one output alone; a weight in bfloat16."""
    x, r, dy, ds, w = draw(24, 96, "f32", 5)
    X = x.cuda().reshape(4, 6, 96).transpose(0, 1).contiguous().transpose(0, 1).requires_grad_(True)
    R = r[:6].cuda().reshape(1, 6, 96).clone().requires_grad_(True)
    W = w.cuda().requires_grad_(True)
    y, total = la.rms_norm(X, W, R.expand(4, 6, 96), eps=EPS, checkpoint=checkpoint)
    dx, dr, dw = torch.autograd.grad([y, total], [X, R, W], [dy.cuda().reshape(4, 6, 96), ds.cuda().reshape(4, 6, 96)])
    s = (x.reshape(4, 6, 96).double() + r[:6].reshape(1, 6, 96).double()).float().reshape(24, 96)
    want, rstd = norm64(s, w, EPS)
    within(y.reshape(24, 96), want, norm_bound(s, want, 96, torch.float32), torch.float32)
    wx, ww, Ex, Ew = norm_backward64(s if checkpoint is None else kept64(s, checkpoint), rstd, w, dy, ds)
    within(dx.reshape(24, 96), wx, Ex, torch.float32)
    within(dr.reshape(6, 96), wx.reshape(4, 6, 96).sum(0), Ex.reshape(4, 6, 96).sum(0) + 4 * U * wx.reshape(4, 6, 96).abs().sum(0), torch.float32)
    within(dw, ww, Ew, torch.float32)
    y, total = la.rms_norm(X, W, R.expand(4, 6, 96), eps=EPS, checkpoint=checkpoint)
    only = torch.autograd.grad(total.sum(), [X, R, W], allow_unused=True, retain_graph=True)
    assert (only[0] == 1).all() and (only[1] == 4).all() and only[2] is None
    only = torch.autograd.grad(y.sum(), [X, R, W])
    both = torch.autograd.grad(sum(t.sum() for t in la.rms_norm(X, W, R.expand(4, 6, 96), eps=EPS, checkpoint=checkpoint)), X)[0]
    # the sum's own gradient of 1 is added in the same rounding
    assert (both - only[0] - 1).abs().max() <= 4 * U * (1 + only[0].abs().max())
    h = la.rms_norm(x.cuda().bfloat16().requires_grad_(True), wb := w.cuda().bfloat16().requires_grad_(True))
    assert torch.autograd.grad(h.sum(), wb)[0].dtype == torch.bfloat16


def test_captured_norm():
    """Forward and backward in a graph, replayed on new inputs with eager calls in between."""
    sets = [[t.cuda() for t in draw(300, 1024, "bf16", 30 + k)] for k in range(3)]
    x, r, dy, ds, w = [t.clone() for t in sets[0]]
    y, total, dx = (torch.empty_like(x) for _ in range(3))
    rstd, dw = torch.empty(300, device="cuda"), torch.empty(1024, device="cuda")
    kept, ks = bytes_like(x)
    ws = torch.empty(la.la_rmsnorm_workspace_bytes(300, 1024), dtype=torch.uint8, device="cuda")

    def step(x, r, w, dy, ds, y, total, dx, dw):
        la.la_rmsnorm_forward(x, r, w, y, None, total, kept, ks, rstd, EPS, None, la.LA_E4M3)
        la.la_rmsnorm_backward(kept, ks, w, rstd, dy, ds, dx, dw, ws, la.LA_E4M3)
    step(x, r, w, dy, ds, y, total, dx, dw)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(x, r, w, dy, ds, y, total, dx, dw)
    for k in (1, 2, 0, 1):
        for a, b in zip((x, r, dy, ds, w), sets[k]):
            a.copy_(b)
        outs = [torch.empty_like(t) for t in (y, total, dx, dw)]
        step(sets[k][0], sets[k][1], sets[k][4], sets[k][2], sets[k][3], *outs)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((y, total, dx, dw), outs))


@pytest.mark.parametrize("normalize", [False, True])
@pytest.mark.parametrize("dtype,D", [("f32", 16), ("f32", 64), ("bf16", 128), ("bf16", 256), ("f32", 32)])
@pytest.mark.parametrize("code", ["e4m3", "int8"])
def test_attention_with_checkpoints(dtype, D, code, normalize):
    """linear_attention(checkpoint=...): O is that of the tensors, the gradients are the bits of the plain
    calls at what the 8 bits stand for, and what is kept is a byte and 1/32 an element."""
    if normalize and D == 256:
        pytest.skip("no normalisation at D = 256")
    B, H, N = 2, 3, 333
    gen = torch.Generator(device="cuda").manual_seed(D)
    Q, K, V, dO = (torch.randn((B, H, N, D), device="cuda", generator=gen) for _ in range(4))
    if not normalize:
        Q, K = Q / Q.norm(dim=3, keepdim=True), K / K.norm(dim=3, keepdim=True)
    Q, K, V, dO = (t.to(TYPE[dtype]) for t in (Q, K, V, dO))
    ts = [t.clone().requires_grad_(True) for t in (Q, K, V)]
    kept = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: kept.append(t) or t, lambda t: t):
        O = la.linear_attention(*ts, normalize_qk=normalize, checkpoint=code)
    assert sum(t.numel() * t.element_size() for t in kept) == 3 * B * H * N * (D + -(-D // 32))
    assert torch.equal(O, la.linear_attention(Q, K, V, normalize_qk=normalize))
    got = torch.autograd.grad(O, ts, dO)
    at = [la.unpack_rows(*la.pack_rows(t, code), code, t.dtype).requires_grad_(True) for t in (Q, K, V)]
    for t, a in zip((Q, K, V), at):
        assert torch.equal(a.double().cpu().reshape(-1, D), kept64(t.reshape(-1, D).cpu(), code))
    want = torch.autograd.grad(la.linear_attention(*at, normalize_qk=normalize), at, dO)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_wrappers_refuse():
    x = torch.zeros((4, 64), device="cuda")
    w = torch.ones(64, device="cuda")
    for bad in (lambda: la.rms_norm(x, w[:32]), lambda: la.rms_norm(x, w.bfloat16()), lambda: la.rms_norm(x, w, x[:2]),
                lambda: la.rms_norm(x, w, x.bfloat16()), lambda: la.rms_norm(x.half()), lambda: la.rms_norm(x, w, checkpoint="int4"),
                lambda: la.rms_norm_quantised(x, w, code="int4"), lambda: la.pack_rows(x.half(), "int8"), lambda: la.rms_norm(x, w.cpu()),
                lambda: la.unpack_rows(x, x, "int8", torch.float32)):
        with pytest.raises((ValueError, TypeError)):
            bad()
    for bad in (lambda: la.rms_norm(x[:0]), lambda: la.rms_norm(torch.zeros((1, 16385), device="cuda"))):
        with pytest.raises(la.LaError):
            bad()


def test_a_block_of_them():
    """norm -> projections -> attention with checkpoints -> recurrence -> norm into 8 bits, as a layer uses
    them: every output and gradient against the same layer in 64 bits.  int8 keeps 1/128 of a group's power, at most
    its largest magnitude, a relative error of some 1/100 for Gaussian rows; through one layer 0.05 is allowed, for
    what goes through float32 alone 1e-5."""
    gen = torch.Generator(device="cuda").manual_seed(12)
    B, N, H, D = 2, 150, 3, 32
    C = H * D
    r = lambda *s: torch.randn(s, device="cuda", generator=gen)
    params = [r(B, N, C), r(B, N, C), 1 + 0.1 * r(C), *(r(C, C) / C ** 0.5 for _ in range(4)), 1 + 0.1 * r(C)]

    def layer(x, res, w1, wq, wk, wv, wg, w2, ours, checkpoint):
        n = lambda t, w: t / torch.sqrt((t * t).mean(-1, keepdim=True) + EPS) * w
        if ours:
            y, s = la.rms_norm(x, w1, res, eps=EPS, checkpoint=checkpoint)
        else:
            s = x + res
            y = n(s, w1)
        q, k, v = ((y @ p).reshape(B, N, H, D).transpose(1, 2) for p in (wq, wk, wv))
        if ours:
            o = la.linear_attention(q, k, v, normalize_qk=True, checkpoint=checkpoint)
        else:
            q, k = q / q.norm(dim=3, keepdim=True), k / k.norm(dim=3, keepdim=True)
            W = torch.tril(1 + 0.5 * (q @ k.transpose(2, 3).contiguous()))
            o = (W @ v) / W.sum(3, keepdim=True)
        o = o.transpose(1, 2).reshape(B, N, C)
        g = y @ wg
        if ours:
            h, last = la.gated_recurrence(o, g)
        else:
            h, rows = torch.zeros_like(o[:, 0]), []
            for t in range(N):
                f = torch.sigmoid(g[:, t])
                h = f * h + (1 - f) * o[:, t]
                rows.append(h)
            h, last = torch.stack(rows, 1), h
        if ours:
            return la.rms_norm(h, w2, s, eps=EPS), s, last
        t = h + s
        return (n(t, w2), t), s, last
    p64 = [p.double().cpu().requires_grad_(True) for p in params]
    (y64, t64), _, last64 = layer(*p64, False, None)
    dy, dl = torch.randn(B, N, C, generator=torch.Generator().manual_seed(1)), torch.randn(B, C, generator=torch.Generator().manual_seed(2))
    want = torch.autograd.grad((y64 * dy).sum() + (last64 * dl).sum(), p64)
    for checkpoint, most in ((None, 1e-5), ("int8", 0.05)):
        p = [t.clone().requires_grad_(True) for t in params]
        (y, t), s, last = layer(*p, True, checkpoint)
        for a, b in ((y, y64), (t, t64), (last, last64)):
            assert (a.double().cpu() - b).norm() <= 1e-5 * b.norm()
        got = torch.autograd.grad((y * dy.cuda()).sum() + (last * dl.cuda()).sum(), p)
        for k, (a, b) in enumerate(zip(got, want)):
            assert (a.double().cpu() - b).norm() <= most * b.norm(), (checkpoint, k)
    codes, scales, total = la.rms_norm_quantised(h := t.detach(), p[-1], s.detach(), eps=EPS)
    y8 = la.unpack_rows(codes, scales, "e4m3", torch.float32)
    full = la.rms_norm(h, p[-1].detach(), s.detach(), eps=EPS)[0]
    assert ((y8 - full).abs() <= torch.maximum(full.abs() / 16, full.abs().amax() * 2.0 ** -18)).all()
