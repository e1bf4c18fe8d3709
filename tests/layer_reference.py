"""The operators around the attention in 64 bits, row by row from their definitions, and bounds on what
float32 arithmetic may be off by.

Bounds are derived, not measured: U = 2^-24 is half a step of float32 relative to a value, half(dtype)
that of a stored type.  A recurrence's error is a recurrence too: with A_t = f_t A_{t-1} + |u_t|, the sum of
magnitudes, every row adds at most STEPS U A_t and hands the rest on, E_t = f_t E_{t-1} + STEPS U A_t."""
import torch

U = 2.0 ** -24
# Roundings of one row of a recurrence, in units of U relative to its magnitudes: the gate (the
# exponential 2, its argument's none, 1 + E 1, the reciprocal 2, a product 1: 6, twice where 1 - f enters too),
# its product with x 1, the multiply-add 1, and as much again for the product of a segment's gates.
STEPS = 24.0


def half(dtype):
    return torch.finfo(dtype).eps / 2


def gates64(g, x, gate):
    g, x = g.double(), x.double()
    if gate == "value":
        return g, torch.ones_like(g), x
    f, rest = torch.sigmoid(g), torch.sigmoid(-g)
    return f, rest, rest * x


def recurrence64(x, g, h0, lengths, gate):
    """h, last and their bounds for x, g [B, N, C]; h is not rounded."""
    B, N, C = x.shape
    f, _, u = gates64(g, x, gate)
    h = torch.zeros((B, N, C), dtype=torch.float64)
    E = torch.zeros_like(h)
    s = torch.zeros((B, C), dtype=torch.float64) if h0 is None else h0.double().clone()
    A, e = s.abs(), torch.zeros_like(s)
    for t in range(N):
        live = torch.ones((B, 1), dtype=torch.bool) if lengths is None else (t < lengths.clamp(0, N)).unsqueeze(1)
        s = torch.where(live, f[:, t] * s + u[:, t], s)
        A = torch.where(live, f[:, t].abs() * A + u[:, t].abs(), A)
        e = torch.where(live, f[:, t].abs() * e + STEPS * U * A, e)
        h[:, t] = torch.where(live, s, 0.0)
        E[:, t] = torch.where(live, e, 0.0)
    return h, s, E, e


def recurrence_backward64(x, g, h0, h, dh, dlast, lengths, gate):
    """dx, dg, dh0 by the formulas, from the stored h, and their bounds."""
    B, N, C = x.shape
    f, rest, _ = gates64(g, x, gate)
    first = torch.zeros((B, C), dtype=torch.float64) if h0 is None else h0.double()
    e = torch.zeros((B, C), dtype=torch.float64) if dlast is None else dlast.double().clone()
    A, err = e.abs(), torch.zeros_like(e)
    dx, dg, Ex, Eg = (torch.zeros((B, N, C), dtype=torch.float64) for _ in range(4))
    for t in reversed(range(N)):
        live = torch.ones((B, 1), dtype=torch.bool) if lengths is None else (t < lengths.clamp(0, N)).unsqueeze(1)
        d, a = dh[:, t].double() + e, dh[:, t].double().abs() + A
        prev = first if t == 0 else h[:, t - 1].double()
        w = f[:, t] * rest[:, t] if gate == "sigmoid" else torch.ones_like(d)
        diff = prev - x[:, t].double() if gate == "sigmoid" else prev
        off = err + STEPS * U * a
        dx[:, t] = torch.where(live, rest[:, t] * d, 0.0)
        dg[:, t] = torch.where(live, d * diff * w, 0.0)
        Ex[:, t] = torch.where(live, rest[:, t] * off, 0.0)
        Eg[:, t] = torch.where(live, off * diff.abs() * w + STEPS * U * a * diff.abs() * w, 0.0)
        e = torch.where(live, f[:, t] * d, e)
        A = torch.where(live, f[:, t].abs() * a, A)
        err = torch.where(live, f[:, t].abs() * off, err)
    return dx, dg, e, Ex, Eg, err


def within(got, want, bound, dtype):
    """|got - want| <= bound + half a step of the stored type, element by element (the step at the larger of
    the two, and at the type's smallest normal number)."""
    got, want = got.detach().double().cpu(), want.double()
    assert got.shape == want.shape, (got.shape, want.shape)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), "NaN at other places"
    room = bound + half(dtype) * (torch.maximum(got.abs(), want.abs()) + torch.finfo(dtype).tiny)
    off = ((got - want).abs() - room).nan_to_num(nan=0.0)
    worst = int(off.argmax())
    assert off.reshape(-1)[worst] <= 0, (worst, got.reshape(-1)[worst].item(), want.reshape(-1)[worst].item(),
                                         room.reshape(-1)[worst].item())


def pack64(x, code):
    """Codes' values in units of the group's power, and powers k (128: NaN), x [rows, C] by the definition:
    the least power that fits, found by trying."""
    rows, C = x.shape
    x = torch.nn.functional.pad(x.double(), (0, -C % 32)).reshape(rows, -1, 32)
    most = x.abs().amax(2)
    fits = 448.0 if code == "e4m3" else 127.0 / 64.0
    k = torch.full(most.shape, 127, dtype=torch.int64)
    for p in range(126, -128, -1):
        k = torch.where(most <= fits * 2.0 ** p, p, k)
    k = torch.where(most == 0, torch.tensor(-9 if code == "e4m3" else -1), k)  # any would do
    scale = 2.0 ** k.double().unsqueeze(2)
    v = x / scale
    if code == "e4m3":
        step = 2.0 ** (torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3)
        v = torch.round(v / step) * step
    else:
        v = torch.round(v * 64).clamp(-127, 127) / 64
    bad = ~torch.isfinite(x).all(2)
    k = torch.where(bad, torch.tensor(128), k)
    v = torch.where(bad.unsqueeze(2), torch.nan, v)
    return v, k


def kept64(x, code):
    """x [rows, C] as its 8 bits give it back."""
    v, k = pack64(x, code)
    return (v * (2.0 ** k.double().clamp(max=127)).unsqueeze(2)).reshape(x.shape[0], -1)[:, :x.shape[1]]


def norm64(s, w, eps):
    """y, rstd of rows s [rows, C] (the stored sum)."""
    s = s.double()
    rstd = 1.0 / torch.sqrt((s * s).mean(1, keepdim=True) + eps)
    return s * rstd * (1.0 if w is None else w.double()), rstd


def norm_backward64(s, rstd, w, dy, ds):
    """dx, dw by the formulas, and their bounds.  m is a sum of C products, in any order: its error is C U times
    the sum of magnitudes at most; that of dw likewise over the rows."""
    s, dy = s.double(), dy.double()
    n, wd = s * rstd, dy * (1.0 if w is None else w.double())
    C, rows = s.shape[1], s.shape[0]
    m, a = (wd * n).mean(1, keepdim=True), (wd * n).abs().mean(1, keepdim=True)
    dx = rstd * (wd - n * m)
    # rstd: the sum of squares C U relative, halved by the root, and 4 roundings; n, products and the rest 8
    rel = (C / 2 + 12) * U
    Ex = rstd.abs() * (rel * (wd.abs() + 2 * n.abs() * a) + (C + 8) * U * n.abs() * a)
    if ds is not None:
        dx, Ex = dx + ds.double(), Ex + 2 * U * (dx.abs() + ds.double().abs())
    return dx, (dy * n).sum(0), Ex, (rel + (rows + 4) * U) * (dy * n).abs().sum(0)
