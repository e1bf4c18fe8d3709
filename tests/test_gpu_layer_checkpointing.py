"""The operators around the attention under torch's activation checkpointing, whose saved tensors can be unpacked one time."""
import pytest
import torch
from torch.utils.checkpoint import checkpoint

import paper_2510_21956_amd as la
from paper_2510_21956_amd import binding

pytestmark = pytest.mark.gpu


def rand(*shape, seed=0):
    return torch.randn(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))


CALLS = {
    "recurrence": lambda x, w: la.gated_recurrence(x, x)[0],
    "norm": lambda x, w: la.rms_norm(x, w),
    "norm with a residual": lambda x, w: la.rms_norm(x, w, x)[0],
    "norm from 8 bits": lambda x, w: la.rms_norm(x, w, x, checkpoint="int8")[0],
    "attention": lambda x, w: la.linear_attention(*[(x * w).view(2, 1, 30, 32)] * 3, normalize_qk=True, checkpoint="e4m3"),
}


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("create_graph", [False, True])
@pytest.mark.parametrize("name", list(CALLS))
def test_recomputed(monkeypatch, name, create_graph, native):
    la.load_library()
    assert binding._native is not None
    if not native:
        monkeypatch.setattr(binding, "_native", None)
    f, x, w = CALLS[name], rand(2, 30, 32).requires_grad_(True), rand(32, seed=1).requires_grad_(True)
    ins = [x] if name == "recurrence" else [x, w]
    y = f(x, w)
    dy = rand(*y.shape, seed=2)
    want = torch.autograd.grad(y, ins, dy)
    again = checkpoint(f, x, w, use_reentrant=False)
    assert torch.equal(again, y)
    got = torch.autograd.grad(again, ins, dy, create_graph=create_graph)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("native", [True, False])
def test_a_sum_used_alone_needs_nothing_that_was_saved(monkeypatch, native):
    """Its gradient passes through, with its history, and a weight that has changed since does not matter."""
    la.load_library()
    if not native:
        monkeypatch.setattr(binding, "_native", None)
    x, r, w = rand(5, 32).requires_grad_(True), rand(5, 32, seed=1).requires_grad_(True), rand(32, seed=2)
    s = la.rms_norm(x, w, r)[1]
    w.zero_()
    ds = rand(5, 32, seed=3).requires_grad_(True)
    gx, gr = torch.autograd.grad(s, [x, r], ds * ds, create_graph=True)
    assert torch.equal(gx, ds * ds) and torch.equal(gr, gx)
    assert torch.allclose(torch.autograd.grad(gx.sum(), ds)[0], 2 * ds)
