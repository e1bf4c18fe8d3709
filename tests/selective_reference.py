"""The short convolution and the selective scan in 64 bits, row by row from their definitions, and bounds on what
float32 arithmetic may be off by.

Bounds are derived, not measured, in units of U = 2^-24, half a step of float32 relative to a value:

  silu       v / (1 + exp(-v)): the exponential 2 (its argument's rounding |v| where it is not made up for, which is in
             bfloat16), 1 + E, the reciprocal 2, products 2: 8 + |v| relative; v itself W + 1 roundings of its magnitudes.
  step       d = softplus(r), r = dt + bias: r's rounding moves d by at most |r| U d; the exponential 2 + |r|, the reciprocal 2,
             products and the polynomial 8: 16 + 2 |r| relative.  Its slope, the sigmoid of r, the same.
  decay      exp(d A): the argument |d A| (STEP + 3), the exponential 2.
  The exponential's instruction gives zero where the result is below the smallest normal number: TINY = 2^-126 more, of
  d and its slope (log(1 + E) and E / (1 + E) are at most E) and of a decay.
  state      a state's error is a recurrence: M_t = a M_{t-1} + |u B|, the sum of magnitudes, and
             E_t = a E_{t-1} + DECAY a M_{t-1} + (STEP + 3) |u B| + 2 U M_t.  Where segments are joined a state goes through
             exp(A sum d): x exp(-x) <= 0.37 times what the sum of a segment's d is off by, 16 + rows / 16 of it; segments have
             at most 2048 rows in the tests: 64 U of the largest M so far.
"""
import torch

from layer_reference import U

TINY = 2.0 ** -126


def _live(lengths, t, B):
    return torch.ones(B, dtype=torch.bool) if lengths is None else t < lengths.clamp(min=0)


def conv64(x, w, bias, state, lengths, act):
    """y, last, and the bounds of y; x [B, N, C], w [C, W], state [B, W - 1, C]."""
    B, N, C = x.shape
    W = w.shape[1]
    x, w = x.double(), w.double()
    state = torch.zeros(B, W - 1, C, dtype=torch.float64) if state is None else state.double()
    y, E, last = torch.zeros(B, N, C, dtype=torch.float64), torch.zeros(B, N, C, dtype=torch.float64), state.clone()
    for b in range(B):
        n = N if lengths is None else min(max(int(lengths[b]), 0), N)
        rows = torch.cat([state[b], x[b, :n]])
        last[b] = rows[n:n + W - 1]
        for t in range(n):
            terms = [w[:, j] * rows[t + j] for j in range(W)] + ([] if bias is None else [bias.double()])
            v, m = sum(terms), sum(z.abs() for z in terms)
            off = (W + 1) * U * m
            if act == "silu":
                y[b, t] = v * torch.sigmoid(v)
                E[b, t] = 1.1 * off + (8 + v.abs()) * U * y[b, t].abs()  # its slope is at most 1.1
            else:
                y[b, t], E[b, t] = v, off
    return y, last, E


def conv_backward64(x, w, bias, state, dy, dlast, lengths, act):
    """dx, dw, dbias, dstate by the formulas, and their bounds."""
    B, N, C = x.shape
    W = w.shape[1]
    x, w, dy = x.double(), w.double(), dy.double()
    state = torch.zeros(B, W - 1, C, dtype=torch.float64) if state is None else state.double()
    dx, Ex = torch.zeros(B, N, C, dtype=torch.float64), torch.zeros(B, N, C, dtype=torch.float64)
    ds, Es = torch.zeros(B, W - 1, C, dtype=torch.float64), torch.zeros(B, W - 1, C, dtype=torch.float64)
    dw, db = torch.zeros(C, W, dtype=torch.float64), torch.zeros(C, dtype=torch.float64)
    Ew, Eb, Mw, Mb = dw.clone(), db.clone(), dw.clone(), db.clone()
    for b in range(B):
        n = N if lengths is None else min(max(int(lengths[b]), 0), N)
        rows = torch.cat([state[b], x[b, :n]])
        d, M, E = (torch.zeros(n + W - 1, C, dtype=torch.float64) for _ in range(3))
        for t in range(n):
            e, off = dy[b, t], torch.zeros(C, dtype=torch.float64)
            if act == "silu":
                terms = [w[:, j] * rows[t + j] for j in range(W)] + ([] if bias is None else [bias.double()])
                v, m = sum(terms), sum(z.abs() for z in terms)
                s = torch.sigmoid(v)
                slope = s * (1 + v * (1 - s))
                # the slope of the slope is at most 1/2; s and 1 - s are (8 + |v|) U off, of terms up to 1 + |v|
                off = e.abs() * (0.5 * (W + 1) * U * m + 2 * (8 + v.abs()) * U * s * (1 + v.abs() * (1 - s)) + 3 * U * slope.abs())
                e = e * slope
            for j in range(W):
                d[t + j] += w[:, j] * e
                M[t + j] += (w[:, j] * e).abs()
                E[t + j] += w[:, j].abs() * off
                dw[:, j] += e * rows[t + j]
                Mw[:, j] += (e * rows[t + j]).abs()
                Ew[:, j] += off * rows[t + j].abs()
            db += e
            Mb += e.abs()
            Eb += off
        if dlast is not None:
            d[n:n + W - 1] += dlast[b].double()
            M[n:n + W - 1] += dlast[b].double().abs()
        E += (W + 2) * U * M
        dx[b, :n], Ex[b, :n], ds[b], Es[b] = d[W - 1:], E[W - 1:], d[:W - 1], E[:W - 1]
    terms = (B * N + 8) * U
    return (dx, dw, db, ds), (Ex, Ew + terms * Mw, Eb + terms * Mb, Es)


def _wide(t, C):
    """[B, N, G, S] of groups to [B, N, C, S] of channels."""
    return t.double().repeat_interleave(C // t.shape[2], 2)


def _steps(dt, bias, step):
    """d, its slope, and how far they may be off, relative."""
    r = dt.double() + (0 if bias is None else bias.double())
    if step == "value":
        return r, torch.ones_like(r), torch.full_like(r, U)
    slope = torch.sigmoid(r)  # less than d
    return torch.nn.functional.softplus(r, threshold=1e9), slope, (16 + 2 * r.abs()) * U + TINY / slope


class Scan64:
    """The selective scan of x, dt [B, N, C], A [C, S], Bm, Cm [B, N, G, S], D, bias [C], h0 [B, C, S] (None: zeros)."""

    def __init__(self, x, dt, A, Bm, Cm, D, bias, h0, lengths, step):
        B, N, C = x.shape
        S = A.shape[1]
        self.d, self.slope, self.rel = _steps(dt, bias, step)
        self.x, self.A, self.D = x.double(), A.double(), torch.zeros(C, dtype=torch.float64) if D is None else D.double()
        self.B, self.C, self.G, self.lengths = _wide(Bm, C), _wide(Cm, C), Bm.shape[2], lengths
        zero = torch.zeros(B, C, S, dtype=torch.float64)
        h = zero if h0 is None else h0.double()
        M, E, most = h.abs(), zero, h.abs()
        self.h, self.M, self.E = [h], [M], [E]  # before every row, and after the last
        self.y, self.Ey = torch.zeros(B, N, C, dtype=torch.float64), torch.zeros(B, N, C, dtype=torch.float64)
        for t in range(N):
            live = _live(lengths, t, B)
            a, off = self.decay(t)
            u = (self.d[:, t] * self.x[:, t]).unsqueeze(2) * self.B[:, t]
            nh, nM = a * h + u, a * M + u.abs()
            nE = a * E + off * a * M + (self.rel[:, t] + 3 * U).unsqueeze(2) * u.abs() + 2 * U * nM
            on = live.reshape(B, 1, 1)
            h, M, E = torch.where(on, nh, h), torch.where(on, nM, M), torch.where(on, nE, E)
            most = torch.maximum(most, M)
            whole = E + 64 * U * most
            Ct = self.C[:, t]
            y = (Ct * h).sum(2) + self.D * self.x[:, t]
            Ey = (Ct.abs() * whole).sum(2) + (S + 4) * U * ((Ct.abs() * M).sum(2) + (self.D * self.x[:, t]).abs())
            self.y[:, t], self.Ey[:, t] = torch.where(on[..., 0], y, 0.0), torch.where(on[..., 0], Ey, 0.0)
            self.h.append(h)
            self.M.append(M)
            self.E.append(whole)
        self.last, self.Elast = h, self.E[-1]

    def decay(self, t):
        z = self.d[:, t].unsqueeze(2) * self.A
        a = torch.exp(z)
        return a, z.abs() * (self.rel[:, t].unsqueeze(2) + 3 * U) + 2 * U + TINY / a.clamp_min(1e-300)

    def backward(self, dy, dlast):
        """Gradients by name, and their bounds."""
        B, N, C = self.x.shape
        S = self.A.shape[1]
        dy = dy.double()
        g = torch.zeros(B, C, S, dtype=torch.float64) if dlast is None else dlast.double()  # what row t hands back
        M, E, most = g.abs(), torch.zeros_like(g), g.abs()
        zero = lambda *s: torch.zeros(*s, dtype=torch.float64)  # noqa: E731
        got = {"x": zero(B, N, C), "dt": zero(B, N, C), "A": zero(C, S), "B": zero(B, N, self.G, S), "C": zero(B, N, self.G, S),
               "D": zero(C), "bias": zero(C)}
        off = {k: v.clone() for k, v in got.items()}
        group = lambda v: v.reshape(B, self.G, C // self.G, S).sum(2)  # noqa: E731
        count = (C // self.G + 8) * U
        rows = (B * N + 8) * U
        for t in reversed(range(N)):
            on = _live(self.lengths, t, B).reshape(B, 1, 1)
            a, da = self.decay(t)
            y, d, x, rel = dy[:, t], self.d[:, t], self.x[:, t], self.rel[:, t]
            c = self.C[:, t] * y.unsqueeze(2)
            w, Mw, Ew = g + c, M + c.abs(), E + 2 * U * (M + c.abs()) + 64 * U * most  # reaches the row's state
            ng, nM, nE = a * w, a * Mw, a * (E + 2 * U * Mw) + (da + U) * a * Mw
            h, Mh, Eh = self.h[t + 1], self.M[t + 1], self.E[t + 1]
            before, Mb, Eb = self.h[t], self.M[t], self.E[t]
            u, ru = (d * x).unsqueeze(2), (rel + U).unsqueeze(2)
            dB, MB = w * u, Mw * u.abs()
            dC, MC = h * y.unsqueeze(2), Mh * y.unsqueeze(2).abs()
            k, Bt = slice(None), self.B[:, t]
            put = lambda name, v, e: (got[name].__setitem__((k, t), torch.where(on if v.dim() == 3 else on[..., 0], v, 0.0)),  # noqa: E731
                                      off[name].__setitem__((k, t), torch.where(on if v.dim() == 3 else on[..., 0], e, 0.0)))
            put("B", group(dB), group(Ew * u.abs() + ru * MB) + count * group(MB))
            put("C", group(dC), group(Eh * y.unsqueeze(2).abs() + U * MC) + count * group(MC))
            gu, Mu, Eu = (w * Bt).sum(2), (Mw * Bt.abs()).sum(2), (Ew * Bt.abs()).sum(2)
            Eu = Eu + (S + 4) * U * Mu
            put("x", d * gu + self.D * y, d.abs() * (Eu + (rel + U) * Mu) + 3 * U * (d.abs() * Mu + (self.D * y).abs()))
            e, Me = ng * before, nM * Mb
            Ee = (a * Ew + (da + U) * a * Mw) * Mb + nM * Eb + U * Me
            gd = (e * self.A).sum(2)
            Ed = ((Ee + 4 * U * Me) * self.A.abs()).sum(2) + (S + 6) * U * (Me * self.A.abs()).sum(2)
            dd, Mdd = x * gu + gd, x.abs() * Mu + (Me * self.A.abs()).sum(2)
            slope = self.slope[:, t]
            edd = slope * (x.abs() * Eu + Ed + 4 * U * Mdd) + (rel + 2 * U) * slope * Mdd
            put("dt", dd * slope, edd)
            l2 = on[..., 0]
            zero_out = lambda v: torch.where(on if v.dim() == 3 else l2, v, 0.0)  # noqa: E731
            got["A"] += zero_out(e * d.unsqueeze(2)).sum(0)
            off["A"] += zero_out(Ee * d.abs().unsqueeze(2) + (rel.unsqueeze(2) + rows + U) * Me * d.abs().unsqueeze(2)).sum(0)
            got["D"] += zero_out(y * x).sum(0)
            off["D"] += zero_out(rows * (y * x).abs()).sum(0)
            got["bias"] += zero_out(dd * slope).sum(0)
            off["bias"] += zero_out(edd + rows * slope * Mdd).sum(0)
            g, M, E = torch.where(on, ng, g), torch.where(on, nM, M), torch.where(on, nE, E)
            most = torch.maximum(most, M)
        got["h0"], off["h0"] = g, E + 64 * U * most
        return got, off
