"""Gradients of gradients of the operators around the attention are refused also where the native nodes leave a backward
pass to Python: a gradient that is a tensor subclass with a dispatch of its own."""
import pytest
import torch

import paper_2510_21956_amd as la
from paper_2510_21956_amd import binding

pytestmark = pytest.mark.gpu


def rand(*shape, seed=0):
    return torch.randn(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))


class Dispatching(torch.Tensor):
    """Has memory of its own; every operation on it runs as on a plain tensor."""

    @staticmethod
    def __new__(cls, t):
        return torch.Tensor._make_subclass(cls, t, t.requires_grad)

    @classmethod
    def __torch_dispatch__(cls, f, types, args=(), kwargs=None):
        guard = torch._C._DisableTorchDispatch()
        try:
            return f(*args, **(kwargs or {}))
        finally:
            del guard


CALLS = {
    "recurrence": (lambda x: la.gated_recurrence(x, x)[0], (2, 30, 40)),
    "norm": (lambda x: la.rms_norm(x, torch.ones(40, device="cuda")), (6, 40)),
    "norm from 8 bits": (lambda x: la.rms_norm(x, None, x.detach(), checkpoint="int8")[0], (6, 40)),
    "attention": (lambda x: la.linear_attention(x, x, x, normalize_qk=True, checkpoint="e4m3"), (1, 2, 30, 32)),
}


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("gradient", ["without a history", "with a history", "subclass"])
@pytest.mark.parametrize("name", list(CALLS))
def test_second_derivatives_are_refused(monkeypatch, name, gradient, native):
    """Losses that depend on x and on the incoming gradient directly too: without a refusal their derivatives would
    lack a part."""
    la.load_library()
    assert binding._native is not None
    if not native:
        monkeypatch.setattr(binding, "_native", None)
    f, shape = CALLS[name]
    x, dy = rand(*shape).requires_grad_(True), rand(*shape, seed=1)
    plain = torch.autograd.grad(f(x), x, dy)[0]
    assert not plain.requires_grad
    if gradient != "without a history":
        dy = (Dispatching(dy.clone()) if gradient == "subclass" else dy.clone()).requires_grad_(True)

    def loss():
        first = torch.autograd.grad(f(x), x, dy, create_graph=True)[0]
        assert torch.equal(first.detach().as_subclass(torch.Tensor), plain)
        return (first * first).sum() + (x * x).sum() + (dy * dy).sum()
    with pytest.raises(RuntimeError, match="not defined"):
        loss().backward()
    if dy.requires_grad:
        with pytest.raises(RuntimeError, match="not defined"):
            torch.autograd.grad(loss(), dy)
    if native:
        with pytest.raises(RuntimeError, match="not defined"):
            torch.autograd.grad(loss(), x)
