"""The norm's backward pass where every workgroup takes several rows one after another, four or five of each group of lanes: what
it requests ahead, the shared sums' reuse of local memory, and dw over many rows.  64-bit references on the device."""
import pytest
import torch

import paper_2510_21956_amd as la
from layer_reference import half, norm64, norm_backward64

pytestmark = pytest.mark.gpu
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
CODE = {"e4m3": la.LA_E4M3, "int8": la.LA_I8}
EPS = 1e-6


def close(got, want, bound, dtype):
    """|got - want| <= bound + half a step of the stored type (at the larger of the two)."""
    assert got.shape == want.shape and torch.isfinite(got).all()
    got = got.double()
    room = bound + half(dtype) * (torch.maximum(got.abs(), want.abs()) + torch.finfo(dtype).tiny)
    off = (got - want).abs() - room
    worst = int(off.argmax())
    assert off.reshape(-1)[worst] <= 0, (worst, got.reshape(-1)[worst].item(), want.reshape(-1)[worst].item())


# Rows to a workgroup: 32, 16, 8, 4, 2 up to 64, 128, 256, 512, 1024 columns, one above; up to 1024 groups of rows are
# shared out to 256 workgroups, a few more than 1024 give some of them a fifth.
SHAPES = [(32 * 1027 - 7, 40), (16 * 1027 - 5, 96), (8 * 1027 - 3, 200), (4 * 1027 - 1, 500), (2 * 1027 - 1, 771), (2053, 1000),
          (1100, 2056), (1100, 2500), (1030, 5001), (1030, 8192), (1030, 9000), (1027, 16384)]


@pytest.mark.parametrize("dtype,weight", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("rows,C", SHAPES)
def test_norm_backward_over_many_rows(rows, C, dtype, weight):
    gen = torch.Generator(device="cuda").manual_seed(rows + C)
    r = lambda *s: torch.randn(*s, device="cuda", generator=gen)
    td = TYPE[dtype]
    channel = torch.exp(r(C))
    x, res, dy, ds = ((r(rows, C) * channel).to(td), (r(rows, C) * channel * 2).to(td), r(rows, C).to(td), r(rows, C).to(td))
    w = (1 + 0.1 * r(C)).to(TYPE[weight])
    ws = torch.full((la.la_rmsnorm_workspace_bytes(rows, C),), 0xFF, dtype=torch.uint8, device="cuda")
    for residual in (False, True):
        s = (x.double() + res.double()).to(td) if residual else x
        for code in (None, "e4m3", "int8"):
            y, total, rstd = torch.empty_like(x), torch.empty_like(x) if residual else None, torch.empty(rows, device="cuda")
            kept = torch.empty(rows, C, dtype=torch.uint8, device="cuda") if code else None
            powers = torch.empty(rows, -(-C // 32), dtype=torch.uint8, device="cuda") if code else None
            la.la_rmsnorm_forward(x, res if residual else None, w, y, None, total, kept, powers, rstd, EPS, None,
                                  CODE[code] if code else None)
            saved = s
            if code:  # what the 8 bits stand for; they are the bits of the packing by itself
                codes, scales = la.pack_rows(s, code)
                assert torch.equal(codes.view(torch.uint8), kept) and torch.equal(scales.view(torch.uint8), powers)
                saved = la.unpack_rows(codes, scales, code, torch.float32)
            _, inv = norm64(s, w, EPS)
            wx, ww, Ex, Ew = norm_backward64(saved, inv, w, dy, ds if residual else None)
            got = []
            for _ in range(2):
                dx, dw = torch.full_like(x, float("nan")), torch.full((C,), float("nan"), device="cuda")
                la.la_rmsnorm_backward(kept if code else s, powers, w, rstd, dy, ds if residual else None, dx, dw, ws,
                                       CODE[code] if code else None)
                got.append((dx, dw))
            close(dx, wx, Ex, td)
            close(dw, ww, Ew, torch.float32)
            assert torch.equal(got[0][0], dx) and torch.equal(got[0][1], dw)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,C", SHAPES)
def test_every_row_counts_once_in_dw(rows, C, dtype):
    """Rows of ones of either sign are their own norms, and with small whole numbers as gradients every sum is a whole
    number that float32 holds: dw is exact, whatever the order, and a row left out or taken twice shows."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    td = TYPE[dtype]
    s = (torch.randint(0, 2, (rows, C), device="cuda", generator=gen) * 2 - 1).to(td)
    dy = torch.randint(-8, 9, (rows, C), device="cuda", generator=gen).to(td)
    w, rstd, dw, dx = torch.ones(C, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(C, device="cuda"), torch.empty_like(s)
    ws = torch.full((la.la_rmsnorm_workspace_bytes(rows, C),), 0xFF, dtype=torch.uint8, device="cuda")
    want = (s.double() * dy.double()).sum(0)
    for code in (None, "e4m3", "int8"):
        y = torch.empty_like(s)
        la.la_rmsnorm_forward(s, None, w, y, None, None, None, None, rstd, 0.0)
        assert torch.equal(y, s) and (rstd == 1).all()
        saved, powers = (s, None) if code is None else la.pack_rows(s, code)
        la.la_rmsnorm_backward(saved, powers, w, rstd, dy, None, dx, dw, ws, CODE[code] if code else None)
        assert torch.equal(dw.double(), want), code


@pytest.mark.parametrize("code", [None, "int8"])
def test_offsets_beyond_32_bits(code):
    """More than 2^31 elements and 2^32 bytes: the last rows' gradients, and dw, which they alone make."""
    rows, C, last = 140000, 16384, 3
    gen = torch.Generator(device="cuda").manual_seed(1)
    s, dy = (torch.zeros((rows, C), device="cuda", dtype=torch.bfloat16) for _ in range(2))
    s[-last:] = torch.randn((last, C), device="cuda", generator=gen).to(torch.bfloat16)
    dy[-last:] = torch.randn((last, C), device="cuda", generator=gen).to(torch.bfloat16)
    w = 1 + 0.1 * torch.randn(C, device="cuda", generator=gen)
    _, inv = norm64(s[-last:], w, EPS)
    rstd = torch.ones(rows, device="cuda")
    rstd[-last:] = inv[:, 0].float()
    saved, powers = (s, None) if code is None else la.pack_rows(s, code)
    if code:
        back = la.unpack_rows(saved, powers, code, torch.bfloat16)
        assert torch.equal(back[-last:], la.unpack_rows(saved[-last:], powers[-last:], code, torch.bfloat16))
        assert not back[:-last].any()
        del back
    dx, dw = torch.full_like(s, float("nan")), torch.empty(C, device="cuda")
    ws = torch.empty(la.la_rmsnorm_workspace_bytes(rows, C), dtype=torch.uint8, device="cuda")
    la.la_rmsnorm_backward(saved, powers, w, rstd, dy, None, dx, dw, ws, CODE[code] if code else None)
    at = s[-last:] if code is None else la.unpack_rows(saved[-last:], powers[-last:], code, torch.float32)
    wx, ww, Ex, Ew = norm_backward64(at, inv, w, dy[-last:], None)
    close(dx[-last:], wx, Ex, torch.bfloat16)
    assert not dx[:-last].any()
    # the rows of zeros add nothing: the bound is that of the three
    close(dw, ww, Ew, torch.float32)
