"""The operators around the mixers in 64 bits on the CPU, from their definitions, each with the
magnitude its rounding errors scale with (the same sums over absolute values)."""
import torch

D = torch.float64


def lengths_of(lengths, B, n):
    return [n] * B if lengths is None else [min(max(int(v), 0), n) for v in lengths]


def conv(x, w, bias=None, silu=True, lengths=None, state=None):
    """(out, state, |pre|): x [B, n, C], w [C, W], state [B, W - 1, C]; |pre| is the sum of absolute terms."""
    x, w = x.to(D), w.to(D)
    B, n, C = x.shape
    W = w.shape[1]
    bias = torch.zeros(C, dtype=D) if bias is None else bias.to(D)
    first = torch.zeros(B, W - 1, C, dtype=D) if state is None else state.to(D)
    rows = torch.cat([first, x], 1)
    lens = lengths_of(lengths, B, n)
    last = torch.stack([rows[i, m:m + W - 1] for i, m in enumerate(lens)])
    keep = torch.arange(n)[None, :, None] < torch.tensor(lens).view(B, 1, 1)
    # what lies at and after a length is not read
    rows = torch.cat([first, torch.where(keep, x, torch.zeros((), dtype=D))], 1)
    pre, mag = bias.expand(B, n, C), bias.abs().expand(B, n, C)
    for j in range(W):
        pre = pre + rows[:, j:j + n] * w[:, j]
        mag = mag + (rows[:, j:j + n] * w[:, j]).abs()
    out = pre * torch.sigmoid(pre) if silu else pre
    return torch.where(keep, out, torch.zeros((), dtype=D)), last, mag


def conv_grad(x, w, bias, dout, silu=True, lengths=None):
    """(dx, dw, dbias) by the formula."""
    x, w, dout = x.to(D), w.to(D), dout.to(D)
    B, n, C = x.shape
    W = w.shape[1]
    keep = torch.arange(n)[None, :, None] < torch.tensor(lengths_of(lengths, B, n)).view(B, 1, 1)
    zero = torch.zeros((), dtype=D)
    x, g = torch.where(keep, x, zero), torch.where(keep, dout, zero)
    rows = torch.cat([torch.zeros(B, W - 1, C, dtype=D), x], 1)
    if silu:
        pre = sum(rows[:, j:j + n] * w[:, j] for j in range(W)) + (0 if bias is None else bias.to(D))
        s = torch.sigmoid(pre)
        g = g * s * (1 + pre * (1 - s))
    after = torch.cat([g, torch.zeros(B, W - 1, C, dtype=D)], 1)
    dx = sum(after[:, W - 1 - j:W - 1 - j + n] * w[:, j] for j in range(W))
    dw = torch.stack([(g * rows[:, j:j + n]).sum((0, 1)) for j in range(W)], 1)
    return torch.where(keep, dx, zero), dw, g.sum((0, 1))


def ssm(x, delta, a, b, c, skip=None, bias=None, softplus=True, lengths=None, state=None):
    """(y, state, |y|, |state|): the serial recurrence, and the same over absolute values."""
    x, delta, a, b, c = (t.to(D) for t in (x, delta, a, b, c))
    B, n, H, P = x.shape
    G, N = b.shape[2:]
    d = delta + (0 if bias is None else bias.to(D))
    if softplus:
        d = torch.nn.functional.softplus(d, threshold=1e9)
    skip = torch.zeros(H, dtype=D) if skip is None else skip.to(D)
    lens = torch.tensor(lengths_of(lengths, B, n))
    b, c = b.repeat_interleave(H // G, 2), c.repeat_interleave(H // G, 2)
    h = torch.zeros(B, H, N, P, dtype=D) if state is None else state.to(D).clone()
    m = h.abs()
    y, ym = torch.zeros(B, n, H, P, dtype=D), torch.zeros(B, n, H, P, dtype=D)
    for t in range(n):
        live = t < lens
        if not bool(live.any()):
            break
        e = torch.exp(d[:, t] * a)[..., None, None]
        add = (d[:, t, :, None] * b[:, t])[..., None] * x[:, t, :, None]
        h2 = e * h + add
        m2 = e * m + add.abs()
        pick = live.view(B, 1, 1, 1)
        h, m = torch.where(pick, h2, h), torch.where(pick, m2, m)
        yt = (c[:, t, :, :, None] * h2).sum(2) + skip[:, None] * x[:, t]
        yn = (c[:, t, :, :, None].abs() * m2).sum(2) + (skip[:, None] * x[:, t]).abs()
        y[:, t], ym[:, t] = torch.where(live.view(B, 1, 1), yt, 0 * y[:, t]), yn
    return y, h, ym, m


def _turn(v, cos, sin, at, interleaved, back=False):
    rot = 0 if cos is None else 2 * cos.shape[1]
    if rot == 0:
        return v, v.abs()
    cs, sn = cos.to(D)[at][:, :, None], sin.to(D)[at][:, :, None]
    if back:
        sn = -sn
    out, mag = v.clone(), v.abs()
    i = torch.arange(rot // 2)
    first, second = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    p, q = v[..., first], v[..., second]
    out[..., first], out[..., second] = p * cs - q * sn, q * cs + p * sn
    mag[..., first], mag[..., second] = (p * cs).abs() + (q * sn).abs(), (q * cs).abs() + (p * sn).abs()
    return out, mag


def qk_norm(x, w, cos, sin, at, heads, eps, interleaved=False):
    """(out, |out|), [B, heads, n, d]: x [B, n, Hx, d], at [B, n] table rows."""
    x = x.to(D)
    w = torch.ones(x.shape[-1], dtype=D) if w is None else w.to(D)
    y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w
    out, mag = _turn(y, cos, sin, at, interleaved)
    per = heads // x.shape[2]
    return tuple(t.transpose(1, 2).repeat_interleave(per, 1) for t in (out, mag))


def qk_norm_grad(x, w, cos, sin, at, dout, eps, interleaved=False):
    """(dx, dw, |dx|, |dw|) by the formula; dout [B, heads, n, d]."""
    x, dout = x.to(D), dout.to(D)
    B, n, Hx, d = x.shape
    w = torch.ones(d, dtype=D) if w is None else w.to(D)
    g = dout.transpose(1, 2).unflatten(2, (Hx, dout.shape[1] // Hx))
    dy, _ = _turn(g.sum(3), cos, sin, at, interleaved, back=True)
    _, mag = _turn(g.abs().sum(3), cos, sin, at, interleaved, back=True)
    if cos is not None and cos.shape[1]:  # |p cos| + |q sin| whatever the signs
        mag = _turn(g.abs().sum(3), cos.abs(), sin.abs(), at, interleaved, back=True)[1]
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    u = x * r
    m = (dy * w * u).mean(-1, keepdim=True)
    dx = r * (dy * w - u * m)
    dxm = r * ((mag * w).abs() + u.abs() * (mag * (w * u).abs()).mean(-1, keepdim=True))
    return dx, (dy * u).sum((0, 1, 2)), dxm, (mag * u.abs()).sum((0, 1, 2))
