"""The calls of the operators around the attention on a stream given by name: they run behind the work that is already
there, and other streams that wait for it find their results."""
import pytest
import torch

import paper_2510_21956_amd as la
from paper_2510_21956_amd import binding

pytestmark = pytest.mark.gpu
GATE = la.LA_GATE_SIGMOID


def rand(*shape, seed=0):
    return torch.randn(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))


def outputs(stream, ins, room):
    """Every call with `stream`, each reading what earlier ones wrote."""
    x, g, h0, rows, w, few = ins  # not read here: on their own stream they may still be on their way
    U = torch.uint8
    e = lambda t: torch.empty_like(t)
    h, last, dx, dg, dh0, o = (e(t) for t in (x, h0, x, x, h0, few))
    y, s, dn, dw, rstd = e(rows), e(rows), e(rows), e(w), torch.empty(rows.shape[0], device="cuda")
    kept, ks = torch.empty(rows.shape, dtype=U, device="cuda"), torch.empty(rows.shape[0], 7, dtype=U, device="cuda")
    back, codes, powers = e(rows), e(kept), e(ks)
    torch.cuda.current_stream().synchronize()
    la.la_recurrence_forward(x, g, h0, h, last, None, GATE, room[0], stream=stream)
    la.la_recurrence_backward(x, g, h0, h, h, last, dx, dg, dh0, None, GATE, room[0], stream=stream)
    la.la_recurrence_step(few, few, o, dh0, GATE, stream=stream)
    la.la_rmsnorm_forward(rows, rows.detach(), w, y, None, s, kept, ks, rstd, 1e-6, None, la.LA_I8, stream=stream)
    la.la_rmsnorm_backward(kept, ks, w, rstd, y, s, dn, dw, room[1], la.LA_I8, stream=stream)
    la.la_pack_rows(dn, codes, powers, la.LA_E4M3, stream=stream)
    la.la_unpack_rows(codes, powers, back, la.LA_E4M3, stream=stream)
    la.la_pack_tensors([dn, back], [codes, kept], [powers, ks], la.LA_I8, stream=stream)
    return [h, last, dx, dg, dh0, o, y, s, rstd, dn, dw, codes, powers, back, kept, ks]


@pytest.mark.parametrize("native", [True, False])
def test_calls_on_a_stream_of_their_own(monkeypatch, native):
    la.load_library()
    if not native:
        monkeypatch.setattr(binding, "_native", None)
    ins = [rand(2, 3000, 200), rand(2, 3000, 200, seed=1), rand(2, 200, seed=2), rand(900, 200, seed=3), rand(200, seed=4),
           rand(2, 2, 200, seed=5)]
    room = [torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") for n in
            (la.la_recurrence_workspace_bytes(2, 3000, 200, la.LA_F32, 1), la.la_rmsnorm_workspace_bytes(900, 200))]
    want = outputs(None, ins, room)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    late = [torch.zeros_like(t) for t in ins]
    for turn in range(3):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):  # the inputs arrive on that stream, behind a copy that takes its time
            torch.empty(1 << 28, dtype=torch.uint8, device="cuda").fill_(turn)
            for a, b in zip(late, ins):
                a.copy_(b)
        got = outputs(side, late, room)
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        for t in late:
            t.zero_()
    torch.cuda.synchronize()
