"""What the operators around the attention write through addresses is a change that autograd sees: a backward pass that
saved such a tensor refuses, as after an operation of torch's own in place."""
import pytest
import torch

import paper_2510_21956_amd as la
from paper_2510_21956_amd import binding

pytestmark = pytest.mark.gpu


def rand(*shape, seed=0, dtype=torch.float32):
    return torch.randn(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(dtype)


@pytest.fixture(params=["native", "python"])
def path(request, monkeypatch):
    la.load_library()
    assert binding._native is not None
    if request.param == "python":
        monkeypatch.setattr(binding, "_native", None)


@pytest.mark.parametrize("gate", ["value", "sigmoid"])
def test_a_step_on_a_state_that_a_backward_pass_needs(path, gate):
    x, g = rand(2, 40, 24).requires_grad_(True), torch.sigmoid(rand(2, 40, 24, seed=1)).requires_grad_(True)
    state, one = rand(2, 24, seed=2), rand(2, 1, 24, seed=3)
    h, _ = la.gated_recurrence(x, g, state, gate=gate)
    kept = state.clone()
    want = torch.autograd.grad(la.gated_recurrence(x, g, kept, gate=gate)[0].sum(), [x, g])
    la.la_recurrence_step(one, one, torch.empty_like(one), state, la.LA_GATE_SIGMOID)
    with pytest.raises(RuntimeError, match="inplace operation"):
        torch.autograd.grad(h.sum(), [x, g])
    # a copy of it is left alone
    h, _ = la.gated_recurrence(x, g, kept, gate=gate)
    la.la_recurrence_step(one, one, torch.empty_like(one), kept.clone(), la.LA_GATE_SIGMOID)
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(h.sum(), [x, g]), want))


def test_a_sum_in_the_place_of_a_saved_residual(path):
    """The residual's buffer, which an earlier norm kept for its backward pass, takes the next sum."""
    stream = rand(30, 96, seed=4)
    x, w = rand(30, 96, seed=5), (1 + 0.1 * rand(96, seed=6)).requires_grad_(True)
    y = la.rms_norm(stream, w)
    la.la_rmsnorm_forward(x, stream, w.detach(), torch.empty_like(x), None, stream, None, None, None, 1e-6)
    with pytest.raises(RuntimeError, match="inplace operation"):
        torch.autograd.grad(y.sum(), w)


def test_versions_of_what_is_written_and_read(path):
    """Every written tensor's version grows and no other's; inference tensors, which have none, are taken."""
    F, U = torch.float32, torch.uint8
    x, g, h, dh, dx, dg = (rand(2, 30, 40, seed=k) for k in range(6))
    h0, last, dlast, dh0, state = (rand(2, 40, seed=10 + k) for k in range(5))
    rows = [rand(9, 70, seed=20 + k) for k in range(7)]
    codes, codes2, y8 = (torch.zeros(9, 70, dtype=U, device="cuda") for _ in range(3))
    powers, powers2, ypowers = (torch.zeros(9, 3, dtype=U, device="cuda") for _ in range(3))
    w, dw, rstd = rand(70, seed=30), torch.zeros(70, device="cuda"), torch.zeros(9, device="cuda")
    room = torch.empty(1 << 20, dtype=U, device="cuda")
    gate = la.LA_GATE_SIGMOID
    calls = [
        (lambda: la.la_recurrence_forward(x, g, h0, h, last, None, gate, room), [x, g, h0], [h, last]),
        (lambda: la.la_recurrence_backward(x, g, h0, h, dh, dlast, dx, dg, dh0, None, gate, room), [x, g, h0, h, dh, dlast],
         [dx, dg, dh0]),
        (lambda: la.la_recurrence_step(x, g, h, state, gate), [x, g], [h, state]),
        (lambda: la.la_pack_rows(rows[0], codes, powers, la.LA_I8), [rows[0]], [codes, powers]),
        (lambda: la.la_pack_tensors(rows[:2], [codes, codes2], [powers, powers2], la.LA_I8), rows[:2],
         [codes, codes2, powers, powers2]),
        (lambda: la.la_unpack_rows(codes, powers, rows[0], la.LA_I8), [codes, powers], [rows[0]]),
        (lambda: la.la_rmsnorm_forward(rows[0], rows[1], w, y8, ypowers, rows[2], codes, powers, rstd, 1e-6, la.LA_E4M3, la.LA_I8),
         [rows[0], rows[1], w], [y8, ypowers, rows[2], codes, powers, rstd]),
        (lambda: la.la_rmsnorm_forward(rows[0], rows[1], w, rows[3], None, rows[1], None, None, None, 1e-6), [rows[0], w],
         [rows[1], rows[3]]),
        (lambda: la.la_rmsnorm_backward(rows[2], None, w, rstd, rows[4], rows[5], rows[6], dw, room),
         [rows[2], w, rstd, rows[4], rows[5]], [rows[6], dw]),
    ]
    for k, (call, read, written) in enumerate(calls):
        before = [[t._version for t in ts] for ts in (read, written)]
        call()
        assert [t._version for t in read] == before[0], k
        assert all(t._version > v for t, v in zip(written, before[1])), k
    with torch.inference_mode():
        xi, hi, si = rand(2, 30, 40), torch.empty(2, 30, 40, device="cuda"), torch.zeros(2, 40, device="cuda")
    la.la_recurrence_step(xi, xi, hi, si, gate)
    la.la_recurrence_forward(xi, xi, None, hi, si, None, gate, room)
    torch.cuda.synchronize()
