"""The operators of the block around a mixer in 64 bits on the CPU, from their definitions, each with the
bounds that its rounding errors stay below.

Errors are propagated like the values: every fp32 operation is off by at most ``E`` = 2^-19 of the magnitude of
its terms (the exponential's 2 units at arguments of up to 8, a reciprocal, a square root, and a handful of
roundings of 2^-24 together stay below it), recurrences carry what they have, and sums carry the sum of it."""
import numpy as np
import torch

D = torch.float64
E = 2.0 ** -19
LINEAR, SIGMOID, SILU = 0, 1, 2


def live(lengths, B, n):
    """[B, n, 1]: tokens before their sequence's length."""
    if lengths is None:
        return torch.ones(B, n, 1, dtype=torch.bool)
    return (torch.arange(n)[None] < lengths.view(B, 1))[..., None]


def glr(x, r, g, decay, state=None, lengths=None):
    """(y, last, bound of y, bound of last) of the gated linear recurrence."""
    B, n, C = x.shape
    on = live(lengths, B, n)
    x, r, g = (torch.where(on, t, torch.zeros((), dtype=t.dtype)).to(D) for t in (x, r, g))
    log_a = decay.to(D) * torch.sigmoid(r)
    a, b = log_a.exp(), (-torch.expm1(2 * log_a)).sqrt() * torch.sigmoid(g) * x
    a = torch.where(on, a, torch.ones((), dtype=D))
    h = torch.zeros(B, C, dtype=D) if state is None else state.to(D)
    H, err, ys, es = h.abs(), torch.zeros(B, C, dtype=D), [], []
    for t in range(n):
        err = a[:, t] * err + E * (a[:, t] * H + b[:, t].abs())
        h, H = a[:, t] * h + b[:, t], a[:, t] * H + b[:, t].abs()
        ys.append(h), es.append(err)
    if n == 0:
        return torch.zeros(B, 0, C, dtype=D), h, torch.zeros(B, 0, C, dtype=D), err
    zero = torch.zeros((), dtype=D)
    return torch.where(on, torch.stack(ys, 1), zero), h, torch.stack(es, 1), err


def glr_grad(x, r, g, decay, dy, state=None, dlast=None, lengths=None):
    """{name: (gradient, bound)} of sum(dy y) + sum(dlast last), by the formula."""
    B, n, C = x.shape
    on = live(lengths, B, n)
    x, r, g, dy = (torch.where(on, t, torch.zeros((), dtype=t.dtype)).to(D) for t in (x, r, g, dy))
    decay = decay.to(D)
    s, i = torch.sigmoid(r), torch.sigmoid(g)
    a, m = (decay * s).exp(), (-torch.expm1(2 * decay * s)).sqrt()
    a = torch.where(on, a, torch.ones((), dtype=D))
    b = torch.where(on, m * i * x, torch.zeros((), dtype=D))
    h = torch.zeros(B, C, dtype=D) if state is None else state.to(D)
    H, err = h.abs(), torch.zeros(B, C, dtype=D)
    before = []
    for t in range(n):
        before.append((h, H, err))
        err = a[:, t] * err + E * (a[:, t] * H + b[:, t].abs())
        h, H = a[:, t] * h + b[:, t], a[:, t] * H + b[:, t].abs()
    d = torch.zeros(B, C, dtype=D) if dlast is None else dlast.to(D)  # the gradient of the state behind a token
    dm, de = d.abs(), torch.zeros(B, C, dtype=D)
    out = {k: [torch.zeros(B, n, C, dtype=D), torch.zeros(B, n, C, dtype=D)] for k in ("dx", "dr", "dg", "es")}
    for t in reversed(range(n)):
        G, Gm, Ge = d + dy[:, t], dm + dy[:, t].abs(), de + E * (dm + dy[:, t].abs())
        hb, Hb, He = before[t]
        X, I, S, M, A = x[:, t], i[:, t], s[:, t], m[:, t], a[:, t]
        e, em = G * (A * hb - I * X * (1 / M - M)), Gm * (A * Hb + (I * X).abs() / M)
        ee = Ge * (A * Hb + (I * X).abs() / M) + Gm * (A * He + E * (A * Hb + (I * X).abs() / M))
        for k, v, bound in (("dx", G * M * I, (Ge + 2 * E * Gm) * M * I),
                            ("dg", G * M * X * I * (1 - I), (Ge + 3 * E * Gm) * M * (X * I).abs() * (1 - I)
                             + E * Gm * M * (X * I).abs()),
                            ("dr", e * decay * S * (1 - S), decay.abs() * S * ((ee + 3 * E * em) * (1 - S) + E * em)),
                            ("es", e * S, (ee + 2 * E * em) * S)):
            out[k][0][:, t], out[k][1][:, t] = v, bound
        d, dm, de = A * G, A * Gm, A * Ge + E * A * Gm
    zero = torch.zeros((), dtype=D)
    res = {k: (torch.where(on, out[k][0], zero), out[k][1]) for k in ("dx", "dr", "dg")}
    es, bound = torch.where(on, out["es"][0], zero), torch.where(on, out["es"][1], zero)
    # (sums of up to B n values one after another)
    res["ddecay"] = (es.sum((0, 1)), bound.sum((0, 1)) + (B * n + 8) * 2.0 ** -24 * es.abs().sum((0, 1)))
    res["dstate"] = (d, de)
    return res


def words(rows, C, seed, offset):
    """[rows, C] of 32 random bits: Philox4x32-10 of (column / 4, row, offset) under the seed, word column % 4."""
    u, low, half = np.uint64, np.uint64(0xFFFFFFFF), np.uint64(32)
    groups = (C + 3) // 4
    c = np.empty((4, rows, groups), dtype=u)
    c[0], c[1] = np.arange(groups, dtype=u), np.arange(rows, dtype=u)[:, None]
    c[2], c[3] = u(offset & 0xFFFFFFFF), u(offset >> 32)
    key = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        p, q = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        c[0], c[1], c[2], c[3] = (q >> half) ^ c[1] ^ u(key[0]), q & low, (p >> half) ^ c[3] ^ u(key[1]), p & low
        key = [(key[0] + 0x9E3779B9) & 0xFFFFFFFF, (key[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.moveaxis(c, 0, -1).reshape(rows, groups * 4)[:, :C]


def act_of(act, v):
    """(value, slope)."""
    s = torch.sigmoid(v)
    return {LINEAR: (v, torch.ones_like(v)), SIGMOID: (s, s * (1 - s)), SILU: (v * s, s * (1 + v * (1 - s)))}[act]


def norm(x, y, gate=None, w_post=None, scale=None, w_pre=None, dx_out=None, dh=None, post=True, pre=True, act=SILU,
         alpha=1.0, eps=1e-6, dropout=0.0, seed=0, offset=0):
    """{name: (value, bound)} of the forward's outputs on rows [R, C] and, with dx_out, of the gradients."""
    x, y = x.to(D), y.to(D)
    R, C = x.shape
    one = torch.ones((), dtype=D)
    wp, sc, wr = (one if w is None else w.to(D) for w in (w_post if post else None, scale, w_pre if pre else None))
    k = torch.ones(R, C, dtype=D)
    if dropout:
        k = torch.from_numpy(words(R, C, seed, offset) >= np.uint64(int(dropout * 2.0 ** 32))).to(D) / (1 - dropout)
    a, slope = (one, one) if gate is None else act_of(act, gate.to(D))
    # |slope| of a gate takes up to 1 + |v| of rounding
    room = one if gate is None else slope.abs() + E * 8 * (1 + gate.to(D).abs())
    r1 = (y.square().mean(-1, keepdim=True) + eps).rsqrt() if post else one
    u = y * r1
    f = k * sc * a * u * wp
    xo = alpha * x + f
    mag = alpha * x.abs() if alpha > 0 else -alpha * x.abs()
    mag = mag + f.abs()
    e = 4 * E  # a norm, an activation and the products
    out = {"x_out": (xo, e * mag)}
    r2 = (xo.square().mean(-1, keepdim=True) + eps).rsqrt() if pre else one
    if pre:
        # r2's own error: the mean's terms carry 2 |x'| e mag
        off = e * ((xo.abs() * mag).mean(-1, keepdim=True) * r2 * r2 + 1)
        out["h"] = (xo * r2 * wr, (e * mag + off * xo.abs()) * r2 * wr.abs())
    if dx_out is None:
        return out
    t, tm = dx_out.to(D), dx_out.to(D).abs()
    if pre:
        hat, gw, hm = xo * r2, dh.to(D) * wr, mag * r2
        t = t + r2 * (gw - hat * (gw * hat).mean(-1, keepdim=True))
        tm = tm + r2 * (gw.abs() + hm * (gw.abs() * hm).mean(-1, keepdim=True)) * (1 + hm.square().mean(-1, keepdim=True))
    e = 16 * E
    q, qm = t * k * a, tm * k * a.abs()
    dn, dnm = q * sc * wp, qm * sc.abs() * wp.abs()
    dy, dym = (r1 * (dn - u * (dn * u).mean(-1, keepdim=True)),
               r1 * (dnm + u.abs() * (dnm * u.abs()).mean(-1, keepdim=True))) if post else (dn, dnm)
    out["dx"], out["dy"] = (alpha * t, e * abs(alpha) * tm), (dy, e * dym)
    if gate is not None:
        out["dgate"] = (t * k * sc * u * wp * slope, e * tm * k * (sc * u * wp).abs() * (room + a.abs() + 1))
    out["dscale"] = ((q * u * wp).sum(0), e * (qm * (u * wp).abs()).sum(0))
    if post:
        out["dw_post"] = ((q * sc * u).sum(0), e * (qm * (sc * u).abs()).sum(0))
    if pre:
        out["dw_pre"] = ((dh.to(D) * hat).sum(0), e * (dh.to(D).abs() * hm * (1 + hm.square().mean(-1, keepdim=True))).sum(0))
    return out


def ffn(x, w, dout=None, act=SILU, between=0.0):
    """{name: (value, bound)}: out and, with dout, dx and dw.  between: the rounding of the projections' gradients."""
    x, w = x.to(D), w.to(D)
    K, F = x.shape[1], w.shape[1]
    # a sum of K products one after another, each step off by a unit of fp32 (twice: matrix units cut off)
    step = lambda n: (n + 16) * 2.0 ** -23  # noqa: E731
    zg, zu = x @ w[0].t(), x @ w[1].t()
    eg, eu = step(K) * (x.abs() @ w[0].abs().t()), step(K) * (x.abs() @ w[1].abs().t())
    a, slope = act_of(act, zg)
    ea = 1.1 * eg + E * (1 + zg.abs()) * (a.abs() + 1e-30)  # (|act'| stays below 1.1)
    out = {"out": (a * zu, ea * zu.abs() + (a.abs() + ea) * eu + E * (a * zu).abs())}
    if dout is None:
        return out
    d = dout.to(D)
    es = eg + E * 8 * (1 + zg.abs())  # (|act''| stays below 1; the slope's terms go up to 1 + |z|)
    dz = torch.cat([d * zu * slope, d * a], 1)
    bz = torch.cat([d.abs() * (zu.abs() * es + (slope.abs() + es) * eu), d.abs() * ea], 1)
    bz = bz + (E + between) * (dz.abs() + bz)
    dzm, wf = dz.abs() + bz, w.reshape(2 * F, K)
    out["dx"] = (dz @ wf, bz @ wf.abs() + step(2 * F) * (dzm @ wf.abs()))
    out["dw"] = ((dz.t() @ x).view(2, F, K),
                 (bz.t() @ x.abs() + step(x.shape[0]) * (dzm.t() @ x.abs())).view(2, F, K))
    return out
