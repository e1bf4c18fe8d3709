"""The selective state space layer's operators as cases that can be timed and checked: the short causal
convolution and the selective scan, each in training, for prompts and for single tokens.

A case is one call of a user's program through the package's public entry points:

  conv          a training step of causal_conv through the autograd wrapper (causal_conv and
                torch.autograd.grad), with the rows before the first carried in and out or from nothing
  conv_prefill  prompts in a serving program: la_conv_forward on a padded batch
  conv_step     la_conv_step: T new rows of every sequence on its carried rows
  scan          a training step of selective_scan, with a state carried in and out or from nothing
  scan_prefill  prompts: la_selective_forward on a padded batch
  scan_step     la_selective_step: T new rows of every sequence on a carried state

The definitions, for sequences of rows t with channels c:

  convolution  y_t = act(bias + sum_j w_j x_{t-(W-1)+j}), j = 0 .. W-1, act none or v -> v / (1 + exp(-v)).  The W - 1
               rows before the first are the carried ones, or zeros; those carried on are the last W - 1.
  scan         d_t = softplus(dt_t + bias), or dt_t as it is;  h_t[s] = exp(d_t A[s]) h_{t-1}[s] + d_t x_t B_t[s];
               y_t = sum_s C_t[s] h_t[s] + D x_t, for the states s of a channel.  B and C are shared by the channels of a group.

Rows from lengths[b] on are padding: not read, zero in every output.
"""
import math

import torch

own = False


def _case(name, kind, dtype, **more):
    return {"name": name, "kind": kind, "dtype": dtype, **more}


def listed():
    return [
        # one token for every sequence of a serving batch: launches and latency
        _case("conv_step_bf16", "conv_step", "bf16", B=8, N=1, C=2048, W=4, act="silu"),
        # a padded batch of prompts in a serving program, its last rows carried out
        _case("conv_prefill_bf16_ragged", "conv_prefill", "bf16", B=2, N=3001, C=1536, W=4, act="silu"),
        # odd sizes in fp32: three taps, no activation, carried rows
        _case("conv_f32_odd", "conv", "f32", B=3, N=1201, C=771, W=3, act="none", ragged=True, carry=True, wide=False),
        # a training step; x is a part of a wider projection's rows, as it is in such a layer
        _case("conv_bf16", "conv", "bf16", B=8, N=2048, C=2048, W=4, act="silu", ragged=False, carry=False, wide=True),
        # one token for every sequence of a serving batch: the state read and written
        _case("scan_step_bf16", "scan_step", "bf16", B=8, N=1, C=2048, S=16, G=1, step="softplus"),
        # a padded batch of prompts, the state carried out
        _case("scan_prefill_bf16_ragged", "scan_prefill", "bf16", B=2, N=3001, C=2048, S=16, G=1, step="softplus"),
        # a short training step in fp32, a small model's width, steps given as values
        _case("scan_f32", "scan", "f32", B=2, N=512, C=768, S=16, G=1, step="value", ragged=False, carry=True),
        # odd sizes: a padded batch, groups of channels with B and C of their own, states that no power of two divides
        _case("scan_bf16_odd", "scan", "bf16", B=3, N=1003, C=771, S=20, G=3, step="softplus", ragged=True, carry=True),
        # one layer of a training step
        _case("scan_bf16", "scan", "bf16", B=8, N=2048, C=2048, S=16, G=1, step="softplus", ragged=False, carry=False),
        # many states a channel, fp32
        _case("scan_f32_wide", "scan", "f32", B=2, N=2048, C=1024, S=64, G=1, step="softplus", ragged=False, carry=False),
        # a long-context training step: one sequence
        _case("scan_bf16_long", "scan", "bf16", B=1, N=65536, C=1536, S=16, G=1, step="softplus", ragged=False, carry=False),
    ]


def _between(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kind = rng.choice(["conv", "conv", "conv_prefill", "conv_step", "scan", "scan", "scan", "scan_prefill", "scan_step"])
    c = {"kind": kind, "dtype": rng.choice(["f32", "bf16"])}
    scan = kind.startswith("scan")
    c["C"] = rng.choice([_between(rng, 16, 8192), 64 * rng.randint(1, 64), 256 * rng.randint(1, 16)])
    c["B"] = _between(rng, 1, 64)
    c["N"] = rng.choice([1, 1, 2, 3, 5, 8]) if kind.endswith("step") else _between(rng, 2, 65536)
    if scan:
        c["S"] = rng.choice([8, 16, 16, 16, 32, 64, rng.randint(1, 48)])
        c["G"] = rng.choice([g for g in (1, 1, 1, 2, 3, 4, 8) if c["C"] % g == 0])
        c["step"] = rng.choice(["softplus", "softplus", "value"])
    else:
        c["W"] = rng.choice([4, 4, 4, 2, 3, 5, 8])
        c["act"] = rng.choice(["silu", "silu", "none"])
    most = 1.6e9 / c["S"] if scan else 3.3e7
    while c["B"] * c["N"] * c["C"] > most:
        c["B" if c["B"] > 1 else "N"] = max(1, c["B" if c["B"] > 1 else "N"] * 2 // 3)
    if kind in ("conv", "scan"):
        c["ragged"], c["carry"] = rng.random() < 0.4, rng.random() < 0.5
    if kind == "conv":
        c["wide"] = rng.random() < 0.5
    return c


# ---- inputs -------------------------------------------------------------------------------------

def _type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 7919 + 31)
    return gen


def _normal(gen, shape, dtype=torch.float32, scale=1.0, shift=0.0):
    x = torch.randn(shape, device="cuda", dtype=torch.float32, generator=gen)
    return (x * scale + shift).to(dtype)


def _lengths(case):
    """Rows of every sequence: the first fills the batch, the others end ever earlier."""
    B, N = case["B"], case["N"]
    if not (case["kind"].endswith("prefill") or case.get("ragged")):
        return [N] * B
    return [N - b * N // (2 * B) for b in range(B)]


def _conv_inputs(case, seed):
    gen, td = _generator(seed), _type(case)
    B, N, C, W = case["B"], case["N"], case["C"], case["W"]
    # the rows of a projection that makes x and a gate beside it, where the case asks for that
    x = _normal(gen, (B, N, 2 * C if case.get("wide") else C), td)[..., :C]
    w = _normal(gen, (C, W), scale=W ** -0.5)
    bias = _normal(gen, (C,), scale=0.1)
    state = _normal(gen, (B, W - 1, C), td)
    return x, w, bias, state, _normal(gen, (B, N, C), td), _normal(gen, (B, W - 1, C), td)


def _scan_inputs(case, seed):
    """Steps between 0.001 and 0.1 and decays -1 .. -S, spread as a trained layer's are around those that it begins with; B and C
    are parts of the rows of one projection."""
    gen, td = _generator(seed), _type(case)
    B, N, C, S, G = (case[k] for k in "BNCSG")
    x = _normal(gen, (B, N, C), td)
    first = torch.exp(torch.rand((C,), device="cuda", generator=gen) * math.log(100.0) + math.log(0.001))
    bias = first + torch.log(-torch.expm1(-first))  # softplus(bias) = first
    dt = _normal(gen, (B, N, C), scale=0.7)
    if case["step"] == "value":
        dt, bias = (first * torch.exp(dt)), None
    dt = dt.to(td)
    A = -torch.exp(_normal(gen, (C, S), scale=0.2)) * torch.arange(1, S + 1, device="cuda")
    rows = _normal(gen, (B, N, 2 * G * S + 48), td)
    Bm = rows[..., 48:48 + G * S].unflatten(-1, (G, S))
    Cm = rows[..., 48 + G * S:].unflatten(-1, (G, S))
    D = _normal(gen, (C,), scale=0.1, shift=1.0)
    h0 = _normal(gen, (B, C, S), scale=0.1)
    return x, dt, A, Bm, Cm, D, bias, h0, _normal(gen, (B, N, C), td), _normal(gen, (B, C, S))


def prepare(case, seed):
    kind = case["kind"]
    s = {"case": case}
    rows = _lengths(case)
    s["lengths"] = None if min(rows) == case["N"] else torch.tensor(rows, dtype=torch.int32, device="cuda")
    if kind.startswith("conv"):
        s["x"], s["w"], s["bias"], s["state"], s["dy"], s["dlast"] = _conv_inputs(case, seed)
        if kind == "conv":
            if not case["carry"]:
                s["state"] = s["dlast"] = None
            s["wanted"] = [s[n].requires_grad_(True) for n in ("x", "w", "bias", "state") if s[n] is not None]
        else:
            s["y"] = torch.empty((case["B"], case["N"], case["C"]), dtype=_type(case), device="cuda")
            s["last"] = torch.empty_like(s["state"])
        return s
    names = ("x", "dt", "A", "Bm", "Cm", "D", "bias", "h0", "dy", "dlast")
    s.update(zip(names, _scan_inputs(case, seed)))
    if kind == "scan":
        if not case["carry"]:
            s["h0"] = s["dlast"] = None
        s["wanted"] = [s[n].requires_grad_(True) for n in names[:8] if s[n] is not None]
        return s
    s["y"], s["last"] = torch.empty_like(s["x"]), torch.empty_like(s["h0"])
    if own and kind == "scan_prefill":
        import paper_2510_21956_amd as la
        n = la.la_selective_workspace_bytes(case["B"], case["N"], case["C"], case["S"], case["G"], 0)
        s["ws"] = torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")
    return s


# ---- the operators in elementary operations, 32 bits --------------------------------------------

def _counts(s, N):
    """Which rows count, [B, N, 1]; None: all."""
    if s["lengths"] is None:
        return None
    return (torch.arange(N, device="cuda") < s["lengths"].unsqueeze(1)).unsqueeze(2)


def _only(x, counts):
    return x if counts is None else torch.where(counts, x, 0.0)


def _sigmoid(v):
    return 1.0 / (1.0 + torch.exp(-v))


def _conv(case, s):
    """The rows with those before them, what the activation is given, which rows count, the rows carried on."""
    W, N = case["W"], case["N"]
    x = s["x"].detach()
    state = x.new_zeros((case["B"], W - 1, case["C"])) if s["state"] is None else s["state"].detach()
    counts = _counts(s, N)
    rows = torch.cat([state, x], 1)
    n = torch.full((case["B"],), N, device="cuda") if s["lengths"] is None else s["lengths"].long()
    at = n.unsqueeze(1) + torch.arange(W - 1, device="cuda")
    last = torch.gather(rows, 1, at.unsqueeze(2).expand(-1, -1, case["C"]))
    rows = torch.cat([state.float(), _only(x.float(), counts)], 1)
    w = s["w"].detach()
    v = s["bias"].detach() + sum(w[:, j] * rows[:, j:j + N] for j in range(W))
    return rows, v, counts, last, at


def _plain_conv(case, s):
    W, N, td = case["W"], case["N"], _type(case)
    rows, v, counts, last, at = _conv(case, s)
    f = _sigmoid(v) if case["act"] == "silu" else 1.0
    y = _only(v * f, counts).to(td)
    if case["kind"] == "conv_step":
        s["state"].copy_(last)
        return [y, s["state"]]
    if case["kind"] == "conv_prefill":
        return [y, last]
    g = s["dy"].float()
    if case["act"] == "silu":
        g = g * (f * (1.0 + v * (1.0 - f)))
    g = _only(g, counts)
    w, pad = s["w"].detach(), torch.nn.functional.pad
    d = sum(w[:, j] * pad(g, (0, 0, j, W - 1 - j)) for j in range(W))
    if case["carry"]:
        d = d.scatter_add(1, at.unsqueeze(2).expand(-1, -1, case["C"]), s["dlast"].float())
    dw = torch.stack([(g * rows[:, j:j + N]).sum((0, 1)) for j in range(W)], 1)
    out = [y] + ([last] if case["carry"] else []) + [d[:, W - 1:].to(td), dw, g.sum((0, 1))]
    return out + ([d[:, :W - 1].to(td)] if case["carry"] else [])


def _doubled(f, u):
    """h_t = f_t h_{t-1} + u_t along dimension 1, from 0: runs of 1, 2, 4, ... rows are joined."""
    d, n = 1, u.shape[1]
    while d < n:
        u = torch.cat([u[:, :d], torch.addcmul(u[:, d:], f[:, d:], u[:, :-d])], 1)
        f = torch.cat([f[:, :d], f[:, d:] * f[:, :-d]], 1) if 2 * d < n else f
        d *= 2
    return u


def _by_channel(t, C):
    """[B, N, G, S] -> [B, N, C, S] in 32 bits: every channel's share of its group."""
    return t.detach().float().repeat_interleave(C // t.shape[2], 2)


def _by_group(t, G):
    """Sums over the channels of a group: [B, N, C, S] -> [B, N, G, S]."""
    return t.unflatten(2, (G, -1)).sum(3)


def _plain_scan(case, s):
    C, td = case["C"], _type(case)
    counts = _counts(s, case["N"])
    x, dt = _only(s["x"].detach().float(), counts), s["dt"].detach().float()
    if case["step"] == "softplus":
        raw = dt + s["bias"].detach()
        dt = torch.clamp_min(raw, 0.0) + torch.log1p(torch.exp(-raw.abs()))
    dt = _only(dt, counts)
    A, D = s["A"].detach(), s["D"].detach()
    Bc = _by_channel(s["Bm"], C)
    every = None if counts is None else counts.unsqueeze(3)
    f = torch.exp(dt.unsqueeze(3) * A)
    u = _only((dt * x).unsqueeze(3) * Bc, every)
    if s["h0"] is not None:
        h0 = s["h0"].detach()
        u[:, 0] += f[:, 0] * h0
    h = _doubled(f, u)
    del u
    Cc = _only(_by_channel(s["Cm"], C), every)
    y = _only(((Cc * h).sum(3) + D * x), counts).to(td)
    last = h[:, -1].clone()
    if case["kind"] == "scan_step":
        s["h0"].copy_(last)
        return [y, s["h0"]]
    if case["kind"] == "scan_prefill":
        return [y, last]
    dy = _only(s["dy"].float(), counts)
    d = Cc * dy.unsqueeze(3)
    del Cc
    if case["carry"]:
        d[:, -1] += s["dlast"]
    after = torch.cat([f[:, 1:], torch.ones_like(f[:, :1])], 1)  # the decay of the next row
    d = _doubled(after.flip(1), d.flip(1)).flip(1)
    del after
    dC = _by_group(h * dy.unsqueeze(3), case["G"])
    dB = _by_group(d * (dt * x).unsqueeze(3), case["G"])
    first = torch.zeros_like(h[:, :1]) if s["h0"] is None else s["h0"].detach().unsqueeze(1)
    h = torch.cat([first, h[:, :-1]], 1)
    e = d * f * h
    del h
    du = (d * Bc).sum(3)
    dx = dt * du + D * dy
    ddt = x * du + (e * A).sum(3)
    dA = (e * dt.unsqueeze(3)).sum((0, 1))
    dh0 = f[:, 0] * d[:, 0]
    if case["step"] == "softplus":
        ddt = ddt * _sigmoid(raw)
    ddt = _only(ddt, counts)
    out = [y, last] if case["carry"] else [y]
    out += [_only(dx, counts).to(td), ddt.to(td), dA, _only(dB, every).to(td), _only(dC, every).to(td), (dy * x).sum((0, 1))]
    out += [ddt.sum((0, 1))] if case["step"] == "softplus" else []
    return out + ([dh0] if case["carry"] else [])


# ---- a user's calls -----------------------------------------------------------------------------

def _own(case, s):
    import paper_2510_21956_amd as la
    kind = case["kind"]
    if kind == "conv":
        y, last = la.causal_conv(s["x"], s["w"], s["bias"], s["state"], s["lengths"], activation=case["act"])
    elif kind == "scan":
        y, last = la.selective_scan(s["x"], s["dt"], s["A"], s["Bm"], s["Cm"], s["D"], s["bias"], s["h0"], s["lengths"],
                                    step=case["step"])
    if kind in ("conv", "scan"):
        outs, grads = ([y, last], [s["dy"], s["dlast"]]) if case["carry"] else ([y], [s["dy"]])
        return [t.detach() for t in outs] + list(torch.autograd.grad(outs, s["wanted"], grads))
    if kind.startswith("conv"):
        act = la.LA_ACT_SILU if case["act"] == "silu" else la.LA_ACT_NONE
        if kind == "conv_step":
            la.la_conv_step(s["x"], s["w"], s["bias"], s["state"], s["y"], act)
            return [s["y"], s["state"]]
        la.la_conv_forward(s["x"], s["w"], s["bias"], s["state"], s["y"], s["last"], s["lengths"], act)
        return [s["y"], s["last"]]
    step = la.LA_STEP_SOFTPLUS if case["step"] == "softplus" else la.LA_STEP_VALUE
    scan = [s[n] for n in ("x", "dt", "A", "Bm", "Cm", "D", "bias", "h0", "y")]
    if kind == "scan_step":
        la.la_selective_step(*scan, step)
        return [s["y"], s["h0"]]
    la.la_selective_forward(*scan, s["last"], None, s["lengths"], step, s["ws"])
    return [s["y"], s["last"]]


def run(s):
    if own:
        return _own(s["case"], s)
    return (_plain_conv if s["case"]["kind"].startswith("conv") else _plain_scan)(s["case"], s)


def work(case):
    """Every input read once and every output written once; flops of the definitions (an exponential counts as one)."""
    e, kind = 4 if case["dtype"] == "f32" else 2, case["kind"]
    B, N, C = case["B"], case["N"], case["C"]
    T = sum(_lengths(case))  # rows
    pad = (B * N - T) * C * e  # an output's rows behind the sequences' ends
    if kind.startswith("conv"):
        W = case["W"]
        weights, state = C * (W + 1) * 4, B * (W - 1) * C * e
        if kind == "conv":
            carried = 4 * state if case["carry"] else 0
            return {"bytes": 4 * T * C * e + 2 * pad + carried + 2 * weights, "flops": T * C * (6 * W + 12)}
        return {"bytes": 2 * T * C * e + pad + 2 * state + weights, "flops": T * C * (2 * W + 4)}
    S, G = case["S"], case["G"]
    state, weights, row = B * C * S * 4, C * (S + 2) * 4, G * S * e
    if kind == "scan":
        carried = 4 * state if case["carry"] else 0
        return {"bytes": T * (6 * C * e + 4 * row) + 2 * pad + carried + 2 * weights, "flops": T * C * (20 * S + 30)}
    return {"bytes": T * (3 * C * e + 2 * row) + pad + 2 * state + weights, "flops": T * C * (6 * S + 12)}


# ---- the definitions in 64 bits -----------------------------------------------------------------

def _conv64(case, seed):
    """Sequence by sequence through a library convolution and its derivatives, in 64 bits."""
    x, w, bias, state, dy, dlast = (t.double() for t in _conv_inputs(case, seed))
    if case["kind"] == "conv" and not case["carry"]:
        state, dlast = torch.zeros_like(state), torch.zeros_like(dlast)
    x, w, bias, state = (t.clone().requires_grad_(True) for t in (x, w, bias, state))
    ys, lasts, total, W = [], [], 0.0, case["W"]
    for b, n in enumerate(_lengths(case)):
        rows = torch.cat([state[b], x[b, :n]], 0)
        v = torch.nn.functional.conv1d(rows.T.unsqueeze(0), w.unsqueeze(1), bias, groups=case["C"])[0].T
        y = torch.nn.functional.silu(v) if case["act"] == "silu" else v
        total = total + (y * dy[b, :n]).sum() + (rows[n:n + W - 1] * dlast[b]).sum()
        ys.append(torch.nn.functional.pad(y.detach(), (0, 0, 0, case["N"] - n)))
        lasts.append(rows[n:n + W - 1].detach())
    y, last = torch.stack(ys), torch.stack(lasts)
    if case["kind"] != "conv":
        return [y, last]
    dx, dw, dbias, dstate = torch.autograd.grad(total, (x, w, bias, state))
    return [y] + ([last] if case["carry"] else []) + [dx, dw, dbias] + ([dstate] if case["carry"] else [])


def _scan64(case, seed):
    """Row after row, forward and back; what no row before or after enters is taken for many rows at once."""
    x, dt, A, Bm, Cm, D, bias, h0, dy, dlast = (None if t is None else t.double() for t in _scan_inputs(case, seed))
    B, N, C, S, G = (case[k] for k in "BNCSG")
    kind, rows = case["kind"], _lengths(case)
    if kind == "scan" and not case["carry"]:
        h0, dlast = torch.zeros_like(h0), torch.zeros_like(dlast)
    d = torch.nn.functional.softplus(dt + bias, threshold=1e9) if case["step"] == "softplus" else dt.clone()
    slope = torch.sigmoid(dt + bias) if case["step"] == "softplus" else torch.ones_like(dt)
    for b, n in enumerate(rows):  # a row that changes nothing
        d[b, n:] = x[b, n:] = dy[b, n:] = Bm[b, n:] = Cm[b, n:] = 0.0
    run = max(1, int(2.5e8 // (B * C * S)))  # rows at once
    starts = list(range(0, N, run))

    def share(t, r):  # rows first, every channel's own of its group
        return t[:, r].transpose(0, 1).unsqueeze(3).expand(-1, -1, -1, C // G, -1).reshape(-1, B, C, S)

    def states(h, r):
        f = torch.exp(d[:, r].transpose(0, 1).unsqueeze(3) * A)
        u = (d[:, r] * x[:, r]).transpose(0, 1).unsqueeze(3) * share(Bm, r)
        for i in range(f.shape[0]):
            h = torch.addcmul(u[i], f[i], h, out=u[i])
        return f, u
    y, h, begins = torch.zeros_like(x), h0, []
    for a in starts:
        r = slice(a, min(N, a + run))
        begins.append(h)
        _, hs = states(h, r)
        y[:, r] = (hs * share(Cm, r)).sum(3).transpose(0, 1) + D * x[:, r]
        h = hs[-1].clone()
    for b, n in enumerate(rows):
        y[b, n:] = 0.0
    if kind != "scan":
        return [y, h]
    last, g = h, dlast  # g: what reaches the last row's state from behind
    dx, dd, dB, dC = torch.zeros_like(x), torch.zeros_like(x), torch.zeros_like(Bm), torch.zeros_like(Cm)
    dA = torch.zeros_like(A)
    for a, begin in zip(starts[::-1], begins[::-1]):
        r = slice(a, min(N, a + run))
        f, hs = states(begin, r)
        gs = share(Cm, r) * dy[:, r].transpose(0, 1).unsqueeze(3)
        dC[:, r] = (hs * dy[:, r].transpose(0, 1).unsqueeze(3)).reshape(-1, B, G, C // G, S).sum(3).transpose(0, 1)
        for i in range(f.shape[0] - 1, -1, -1):
            gs[i] += g
            g = gs[i] * f[i]
        before = torch.cat([begin.unsqueeze(0), hs[:-1]])
        del hs
        e = gs * f * before
        del before, f
        u = (d[:, r] * x[:, r]).transpose(0, 1).unsqueeze(3)
        dB[:, r] = (gs * u).reshape(-1, B, G, C // G, S).sum(3).transpose(0, 1)
        du = (gs * share(Bm, r)).sum(3).transpose(0, 1)
        dx[:, r] = d[:, r] * du + D * dy[:, r]
        dd[:, r] = (x[:, r] * du + (e * A).sum(3).transpose(0, 1)) * slope[:, r]
        dA += (e * d[:, r].transpose(0, 1).unsqueeze(3)).sum((0, 1))
    for b, n in enumerate(rows):
        dx[b, n:] = dd[b, n:] = dB[b, n:] = dC[b, n:] = 0.0
    out = [y, last] if case["carry"] else [y]
    out += [dx, dd, dA, dB, dC, (dy * x).sum((0, 1))]
    out += [dd.sum((0, 1))] if case["step"] == "softplus" else []
    return out + ([g] if case["carry"] else [])


def exact(case, seed):
    return (_conv64 if case["kind"].startswith("conv") else _scan64)(case, seed)
