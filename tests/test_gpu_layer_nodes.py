"""The autograd nodes of the operators around the attention in native code and in Python: the same results, bit
for bit, and the same refusals."""
import threading

import pytest
import torch

import paper_2510_21956_amd as la
from paper_2510_21956_amd import binding

pytestmark = pytest.mark.gpu


def rand(*shape, seed=0, dtype=torch.float32):
    return torch.randn(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(dtype)


NAMES = ["recurrence", "recurrence with a state", "state without a gradient", "norm", "norm with a weight",
         "norm with a residual", "norm whose residual has no gradient", "norm from 8 bits", "attention",
         "attention, normalised"]


def calls(dtype):
    x, g, r = (rand(3, 70, 48, seed=k, dtype=dtype) for k in range(3))
    w = 1 + 0.1 * rand(48, seed=4)
    h0, n = rand(3, 48, seed=5), torch.tensor([70, 0, 33], dtype=torch.int32, device="cuda")
    q = [rand(1, 2, 90, 32, seed=6 + k, dtype=dtype) for k in range(3)]
    return {
        "recurrence": (lambda x, g: la.gated_recurrence(x, g), [x, g]),
        "recurrence with a state": (lambda x, g, h0: la.gated_recurrence(x, g.sigmoid(), h0, n, gate="value"), [x, g, h0]),
        "state without a gradient": (lambda x, g: la.gated_recurrence(x, g, h0, n), [x, g]),
        "norm": (lambda x: la.rms_norm(x), [x]),
        "norm with a weight": (lambda x, w: la.rms_norm(x, w, eps=1e-5), [x, w]),
        "norm with a residual": (lambda x, r, w: la.rms_norm(x, w, r), [x, r, w]),
        "norm whose residual has no gradient": (lambda x, w: la.rms_norm(x, w, r), [x, w]),
        "norm from 8 bits": (lambda x, r, w: la.rms_norm(x, w.to(x.dtype), r, checkpoint="int8"), [x, r, w]),
        "attention": (lambda q, k, v: la.linear_attention(q, k, v, 1, 0.5, checkpoint="e4m3"), q),
        "attention, normalised": (lambda q, k, v: la.linear_attention(q, k, v, normalize_qk=True, causal=False, checkpoint="int8"), q),
    }


def run(f, inputs, alone=False):
    ts = [t.clone().requires_grad_(True) for t in inputs]
    shapes = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: shapes.append((tuple(t.shape), t.dtype)) or t.clone(), lambda t: t):
        out = f(*ts)
    out = list(out) if isinstance(out, (list, tuple)) else [out]
    used = out[-1:] if alone else out
    grads = torch.autograd.grad(used, ts, [rand(*o.shape, seed=90 + k, dtype=o.dtype) for k, o in enumerate(used)], allow_unused=True)
    return out, grads, sorted(map(str, shapes))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("name", NAMES)
def test_native_and_python(monkeypatch, name, dtype):
    every = calls(dtype)
    assert list(every) == NAMES
    f, inputs = every[name]
    assert la.load_library() and binding._native is not None
    native = [run(f, inputs, alone) for alone in (False, True)]
    monkeypatch.setattr(binding, "_native", None)
    for (o1, g1, s1), alone in zip(native, (False, True)):
        o2, g2, s2 = run(f, inputs, alone)
        assert len(o1) == len(o2) and all(torch.equal(a, b) for a, b in zip(o1, o2))
        assert all((a is None) == (b is None) and (a is None or torch.equal(a, b)) for a, b in zip(g1, g2)), (name, alone)
        assert s1 == s2, (name, s1, s2)


def test_quantised_native_and_python(monkeypatch):
    x, r, w = rand(9, 200, dtype=torch.bfloat16), rand(9, 200, seed=1, dtype=torch.bfloat16), rand(200, seed=2)
    st = rand(9, 200, seed=3).reshape(9, 200)
    one = [la.rms_norm_quantised(x, w, r, code=c) for c in ("e4m3", "int8")] + [la.rms_norm_quantised(x.requires_grad_(True))]
    assert not any(t.requires_grad for o in one for t in o)
    h, state = torch.empty_like(x).reshape(9, 1, 200), st.clone()
    la.la_recurrence_step(x.detach().reshape(9, 1, 200), r.reshape(9, 1, 200), h, state, la.LA_GATE_SIGMOID)
    monkeypatch.setattr(binding, "_native", None)
    two = [la.rms_norm_quantised(x, w, r, code=c) for c in ("e4m3", "int8")] + [la.rms_norm_quantised(x)]
    bits = lambda t: t.view(torch.uint8) if t.element_size() == 1 else t
    assert all(a.dtype == b.dtype and torch.equal(bits(a), bits(b)) for p, q in zip(one, two) for a, b in zip(p, q))
    h2, state2 = torch.empty_like(h), st.clone()
    la.la_recurrence_step(x.detach().reshape(9, 1, 200), r.reshape(9, 1, 200), h2, state2, la.LA_GATE_SIGMOID)
    assert torch.equal(h, h2) and torch.equal(state, state2)


@pytest.mark.parametrize("native", [True, False])
def test_gradients_of_gradients_are_refused(monkeypatch, native):
    la.load_library()
    if not native:
        monkeypatch.setattr(binding, "_native", None)
    for name, (f, inputs) in calls(torch.float32).items():
        ts = [t.clone().requires_grad_(True) for t in inputs]
        out = f(*ts)
        out = out[0] if isinstance(out, (list, tuple)) else out
        first = torch.autograd.grad((out * out).sum(), ts[0], create_graph=True)[0]
        with pytest.raises(RuntimeError):
            torch.autograd.grad((first * first).sum(), ts[0])


@pytest.mark.parametrize("native", [True, False])
def test_refusals_in_the_same_words(monkeypatch, native):
    la.load_library()
    if not native:
        monkeypatch.setattr(binding, "_native", None)
    x, w = rand(4, 8, 16), rand(16)
    said = []
    for bad in (lambda: la.gated_recurrence(x, x[:2]), lambda: la.gated_recurrence(x, x.bfloat16()), lambda: la.gated_recurrence(x, x, w),
                lambda: la.rms_norm(x, w[:3]), lambda: la.rms_norm(x, w, x[0]), lambda: la.rms_norm(x, w.half()),
                lambda: la.rms_norm_quantised(x, w[:3]), lambda: la.gated_recurrence(x, x, lengths=w), lambda: la.rms_norm(x[:, :0], w),
                lambda: la.linear_attention(x, x, x, checkpoint="int8"), lambda: la.gated_recurrence(x[:0], x[:0])):
        with pytest.raises((ValueError, TypeError, la.LaError)) as e:
            bad()
        said.append("%s: %s" % (type(e.value).__name__, e.value))
    if not hasattr(test_refusals_in_the_same_words, "said"):
        test_refusals_in_the_same_words.said = said
    assert said == test_refusals_in_the_same_words.said


def test_wrapped_inputs_take_the_python_node():
    """A tensor subclass, and a call inside of a dispatch mode."""
    from torch.utils._python_dispatch import TorchDispatchMode

    class Plain(torch.Tensor):
        pass

    class Mode(TorchDispatchMode):
        def __torch_dispatch__(self, f, types, args=(), kwargs=None):
            return f(*args, **(kwargs or {}))
    x, g = rand(2, 30, 40), rand(2, 30, 40, seed=1)
    want = la.gated_recurrence(x, g)
    got = la.gated_recurrence(x.as_subclass(Plain), g)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
    with Mode():
        got = la.gated_recurrence(x, g)
    assert torch.equal(want[0], got[0])
    y = la.rms_norm(x)
    assert torch.equal(y, la.rms_norm(x.as_subclass(Plain)))


def test_captured_training_step():
    """Forward and backward through the wrappers in a graph (torch.autograd.grad, no accumulation into leaves), replayed
    on new inputs with eager steps in between; every replay gives the eager step's bits."""
    def step(x, r, g, w, dy):
        y, s = la.rms_norm(x, w, r, checkpoint="e4m3")
        h, last = la.gated_recurrence(y, g)
        return [h, last, s, *torch.autograd.grad([h, last, s], [x, r, g, w], [dy, last.detach(), dy])]
    draw = lambda k: [rand(2, 400, 96, seed=10 * k + j, dtype=torch.bfloat16) for j in range(3)] + [1 + 0.1 * rand(96, seed=k)] + \
        [rand(2, 400, 96, seed=10 * k + 7, dtype=torch.bfloat16)]
    ins = [t.requires_grad_(j < 4) for j, t in enumerate(draw(0))]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*ins)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step(*ins)
    for k in (1, 2, 0, 1):
        new = draw(k)
        with torch.no_grad():
            for a, b in zip(ins, new):
                a.copy_(b)
        want = step(*[t.requires_grad_(j < 4) for j, t in enumerate(new)])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def block(x, r, g, w, dy):
    """Norm, attention with checkpoints, recurrence, norm into 8 bits, and the gradients."""
    y, s = la.rms_norm(x, w, r, checkpoint="int8")
    q = y.view(2, 300, 4, 32).transpose(1, 2)
    o = la.linear_attention(q, q, q.flip(2), checkpoint="e4m3", normalize_qk=True)
    h, last = la.gated_recurrence(o.transpose(1, 2).reshape(2, 300, 128), g)
    eight = [t.view(torch.uint8) for t in la.rms_norm_quantised(h, w)]
    return [h, last, s, *eight, *torch.autograd.grad([h, last, s], [x, r, g, w], [dy, last.detach(), dy])]


def block_inputs(k):
    return [t.requires_grad_(j < 4) for j, t in enumerate(
        [rand(2, 300, 128, seed=10 * k + j, dtype=torch.bfloat16) for j in range(3)] + [1 + 0.1 * rand(128, seed=k)] +
        [rand(2, 300, 128, seed=10 * k + 7, dtype=torch.bfloat16)])]


def test_captured_block():
    ins = block_inputs(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block(*ins)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = block(*ins)
    for k in (1, 2, 0, 1):
        new = block_inputs(k)
        with torch.no_grad():
            for a, b in zip(ins, new):
                a.copy_(b)
        want = block(*new)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_threads_with_streams_of_their_own():
    """Four threads at once give the bits of calls that run alone."""
    sets = [block_inputs(k) for k in range(4)]
    alone = [[t.detach() for t in block(*s)] for s in sets]
    torch.cuda.synchronize()
    bad = []

    def work(k):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(10):
                    got = block(*sets[k])
                    torch.cuda.current_stream().synchronize()
                    if not all(torch.equal(a, b) for a, b in zip(got, alone[k])):
                        bad.append(k)
        except Exception as e:
            bad.append(e)
    threads = [threading.Thread(target=work, args=(k,)) for k in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad


def test_sizes_beyond_32_bits_are_refused():
    """Sizes that a C int would cut off to ones the library takes: by both paths, before anything runs."""
    big = (1 << 32) + 64
    x = torch.empty(big, dtype=torch.bfloat16, device="cuda")
    for s in ((1, big, 1), (big, 1, 1)):
        v = x.view(*s)
        with pytest.raises(ValueError, match="2\\^31"):
            la.gated_recurrence(v, v)
        with pytest.raises(ValueError, match="2\\^31"):
            la.la_recurrence_step(v, v, v, torch.empty(s[0], 1, device="cuda"), la.LA_GATE_SIGMOID)
    with pytest.raises(ValueError, match="2\\^31"):
        la.rms_norm(x.view(1, big))
    with pytest.raises(ValueError, match="2\\^31"):
        la.rms_norm_quantised(x.view(1, big))
