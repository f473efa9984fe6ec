"""The operators of the block around a mixer, as cases that can be timed and checked:

  glr     the gated linear recurrence: prompts, its gradient, single tokens
  norm    the norms after and before a block with its gate, residual scale and dropout: forward, gradient
  ffn     the gated feed-forward projections with their activation and product: forward, gradient

``run`` computes a case with elementary torch operations in 32 bits, or, where ``own`` is true, with
the library's entry points.  ``exact`` computes it from the definition in 64 bits.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
LINEAR, SIGMOID, SILU = 0, 1, 2
EPS = 1e-6


def listed():
    return [
        # glr: a training batch, the batch and length of the framework's head-size-64 workload, 2048 channels
        glr("glr_prompts_bf16", "prompt", "bf16", 8, 2048, 2048),
        # one long prompt with few channels: the work has to be split along the sequence
        glr("glr_long_bf16", "prompt", "bf16", 1, 32768, 1024),
        # a ragged batch that continues from kept states, odd channel count, 32 bits
        glr("glr_ragged_f32", "prompt", "f32", 5, 333, 203, ragged=True, carried=True),
        # the gradient in a training step
        glr("glr_gradient_bf16", "gradient", "bf16", 8, 2048, 2048),
        # one token for each of 64 sequences
        glr("glr_token_bf16", "token", "bf16", 64, 1, 2048),
        # norm: between two blocks of a training step, with everything on
        norm("norm_train_bf16", "forward", "bf16", 8, 2048, 2048, drop=0.1),
        # its gradient
        norm("norm_gradient_bf16", "gradient", "bf16", 8, 2048, 2048, drop=0.1),
        # one token for each of 64 sequences
        norm("norm_token_bf16", "forward", "bf16", 64, 1, 2048),
        # ffn: a training batch of 8192 tokens, 2048 channels, 5632 inner ones
        ffn("ffn_train_bf16", "forward", "bf16", 8192, 2048, 5632),
        # its gradient
        ffn("ffn_gradient_bf16", "gradient", "bf16", 8192, 2048, 5632),
        # one token for each of 16 sequences: the weights' bytes count
        ffn("ffn_token_bf16", "forward", "bf16", 16, 2048, 5632),
        # a short prompt, odd sizes, 32 bits
        ffn("ffn_odd_f32", "gradient", "f32", 333, 260, 1031),
    ]


def glr(name, kind, dtype, B, n, C, ragged=False, carried=False):
    return {"name": name, "op": "glr", "kind": kind, "dtype": dtype, "B": B, "n": n, "C": C, "ragged": ragged,
            "carried": carried}


def norm(name, kind, dtype, B, n, C, drop=0.0, act=SILU, gated=True, post=True, pre=True):
    return {"name": name, "op": "norm", "kind": kind, "dtype": dtype, "B": B, "n": n, "C": C, "drop": drop, "act": act,
            "gated": gated, "post": post, "pre": pre}


def ffn(name, kind, dtype, rows, K, F, act=SILU):
    return {"name": name, "op": "ffn", "kind": kind, "dtype": dtype, "rows": rows, "K": K, "F": F, "act": act}


def draw(rng):
    """One more case: an operator, a direction, a type, and sizes spread over the listed range."""
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))

    def width(lo, hi):  # three in four are multiples of 8, as projections are
        v = log(lo, hi)
        return max(8, v // 8 * 8) if rng.random() < 0.75 else v

    flag = lambda p=0.5: rng.random() < p  # noqa: E731
    op = rng.choice(["glr", "glr", "norm", "norm", "ffn"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    top = 32e6 if dtype == "bf16" else 16e6  # values of a token tensor
    if op == "glr":
        kind = rng.choice(["prompt", "prompt", "gradient", "token"])
        B, C = log(1, 64), width(24, 4096)
        n = 1 if kind == "token" else log(1, max(2, min(32768 if kind == "prompt" else 8192, top / (B * C))))
        c = glr("", kind, dtype, B, n, C, kind != "token" and flag(), kind != "token" and flag())
    elif op == "norm":
        kind = rng.choice(["forward", "gradient"])
        C, B = width(24, 8192), log(1, 64)
        n = 1 if flag(0.25) else log(1, max(2, min(16384, top / (B * C))))
        c = norm("", kind, dtype, B, n, C, rng.choice([0.0, 0.1, 0.25]), rng.choice([LINEAR, SIGMOID, SILU, SILU]),
                 flag(0.75), flag(0.75), flag(0.75))
    else:
        kind = rng.choice(["forward", "gradient"])
        K, F = width(32, 4096), width(32, 8192)
        most = 8192 * 2048 * 5632 / (1 if dtype == "bf16" else 16)
        c = ffn("", kind, dtype, log(1, max(2, min(16384, most / (K * F)))), K, F, rng.choice([SIGMOID, SILU, SILU]))
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------

def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 29)
    T = TYPES[case["dtype"]]

    def normal(*shape, scale=1.0, dtype=T):
        return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)

    def uniform(lo, hi, *shape):
        return torch.rand(shape, generator=g, device=DEV) * (hi - lo) + lo

    def empty(*shape, dtype=T):
        return torch.empty(shape, dtype=dtype, device=DEV)

    s = {"case": case}
    if own:
        from paper_2510_27258_gb300 import hla
        s["hla"] = hla
    if case["op"] == "glr":
        B, n, C = case["B"], case["n"], case["C"]
        pad = -(-C // 8) * 8  # x, r and g are parts of one projection
        rows = normal(B, n, 3 * pad)
        s["x"], s["r"], s["g"] = rows[..., :C], rows[..., pad:pad + C], rows[..., 2 * pad:2 * pad + C]
        s["decay"] = 8 * torch.log(uniform(0.9, 0.999, C))
        s["lengths"] = None
        if case["ragged"]:  # any length, none and all among them
            s["lengths"] = torch.randint(0, n + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
            s["lengths"][B - 1] = n
        s["state"] = normal(B, C, scale=0.5, dtype=torch.float32)
        s["out"], s["state_out"] = empty(B, n, C), empty(B, C, dtype=torch.float32)
        if case["kind"] == "token":
            for name in ("x", "r", "g", "out"):
                s[name] = s[name][:, 0]
            return s
        if case["kind"] == "gradient":
            s["dout"], s["dstate_out"] = normal(B, n, C), normal(B, C, dtype=torch.float32)
            grads = empty(B, n, 3 * pad)  # written side by side, as the projection's gradient reads them
            s["dx"], s["dr"], s["dg"] = grads[..., :C], grads[..., pad:pad + C], grads[..., 2 * pad:2 * pad + C]
            s["dstate_in"] = empty(B, C, dtype=torch.float32)
        if own and case["kind"] == "gradient":  # the states that a training step's forward leaves for its gradient
            s["marks"] = empty(B, hla.hla_glr_marks(n), C, dtype=torch.float32)
            hla.hla_glr_forward(s["x"], s["r"], s["g"], s["decay"], lengths=s["lengths"],
                                state_in=s["state"] if case["carried"] else None, marks=s["marks"])
            s["ws"] = hla.alloc_workspace(hla.hla_glr_backward_workspace_bytes(B, n, C, T), DEV)
    elif case["op"] == "norm":
        B, n, C = case["B"], case["n"], case["C"]
        s["x"] = normal(B, n, C)
        s["y"] = normal(B, n, C, scale=0.5)
        s["gate"] = normal(B, n, C) if case["gated"] else None
        for name in ("w_post", "w_pre"):
            s[name] = (1 + normal(C, scale=0.2, dtype=torch.float32)).to(T)
        s["scale"] = uniform(0.1, 1.0, C).to(T)
        s["alpha"] = 1.0 if case["post"] else 0.875
        s["seed"], s["offset"] = int(seed) * 1000003 + 12345678901, int(seed) * 7 + 4
        if case["kind"] == "gradient":
            s["dx_out"], s["dh"] = normal(B, n, C), normal(B, n, C) if case["pre"] else None
            if own:
                s["ws"] = hla.alloc_workspace(hla.hla_block_norm_backward_workspace_bytes(B * n, C, T), DEV)
    else:
        M, K, F = case["rows"], case["K"], case["F"]
        s["x"] = normal(M, K)
        s["w"] = normal(2, F, K, scale=K ** -0.5)  # gate rows, then up rows
        if case["kind"] == "gradient":
            s["dout"] = normal(M, F)
        if own:
            size = hla.hla_ffn_workspace_bytes if case["kind"] == "forward" else hla.hla_ffn_backward_workspace_bytes
            s["ws"] = hla.alloc_workspace(size(M, K, F, T), DEV)
    return s


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------

def run(s):
    case = s["case"]
    if own:
        return {"glr": _own_glr, "norm": _own_norm, "ffn": _own_ffn}[case["op"]](s["hla"], s, case)
    return {"glr": _plain_glr, "norm": _plain_norm, "ffn": _plain_ffn}[case["op"]](s, case)


def _own_glr(hla, s, case):
    if case["kind"] == "token":
        hla.hla_glr_step(s["x"], s["r"], s["g"], s["decay"], s["state"], s["out"])
        return s["out"], s["state"]
    if case["kind"] == "gradient":
        grads = hla.hla_glr_backward(s["x"], s["r"], s["g"], s["decay"], s["dout"], s["marks"], s["dx"], s["dr"], s["dg"],
                                     dstate_out=s["dstate_out"], dstate_in=s["dstate_in"], lengths=s["lengths"],
                                     workspace=s["ws"])
        return grads + (s["dstate_in"],)
    hla.hla_glr_forward(s["x"], s["r"], s["g"], s["decay"], s["out"], lengths=s["lengths"],
                        state_in=s["state"] if case["carried"] else None, state_out=s["state_out"])
    return s["out"], s["state_out"]


def _own_norm(hla, s, case):
    kw = dict(w_post=s["w_post"] if case["post"] else None, scale=s["scale"], w_pre=s["w_pre"] if case["pre"] else None,
              post_norm=case["post"], pre_norm=case["pre"], act=case["act"], alpha=s["alpha"], eps=EPS,
              dropout=case["drop"], seed=s["seed"], offset=s["offset"])
    if case["kind"] == "gradient":
        got = hla.hla_block_norm_backward(s["x"], s["y"], s["gate"], s["dx_out"], s["dh"], workspace=s["ws"], **kw)
    else:
        got = hla.hla_block_norm_forward(s["x"], s["y"], s["gate"], **kw)
    return [t for t in got if t is not None]


def _own_ffn(hla, s, case):
    if case["kind"] == "gradient":
        return hla.hla_ffn_backward(s["x"], s["w"], s["dout"], act=case["act"], workspace=s["ws"])
    return hla.hla_ffn_forward(s["x"], s["w"], act=case["act"], workspace=s["ws"])


def _sigmoid(v):
    return 1 / (1 + torch.exp(-v))


def _plain_glr(s, case):
    T = s["x"].dtype
    x, r, g, decay = s["x"].float(), s["r"].float(), s["g"].float(), s["decay"]
    sig, inp = _sigmoid(r), _sigmoid(g)
    log_a = decay * sig
    a, m = torch.exp(log_a), torch.sqrt(-torch.expm1(2 * log_a))
    if case["kind"] == "token":
        s["state"].mul_(a).add_(m * inp * x)
        s["out"].copy_(s["state"])
        return s["out"], s["state"]
    B, n, C = x.shape
    live = None
    b = m * inp * x
    if s["lengths"] is not None:
        live = (torch.arange(n, device=DEV) < s["lengths"][:, None])[..., None]
        a, b = torch.where(live, a, 1.0), torch.where(live, b, 0.0)
    first = s["state"] if case["carried"] else x.new_zeros(B, C)
    h = _scan(a, b.clone(), first)
    last = h[:, n - 1]
    if case["kind"] == "prompt":
        return (h if live is None else torch.where(live, h, 0.0)).to(T), last.clone()
    dout = s["dout"].float()
    if live is not None:
        dout = torch.where(live, dout, 0.0)
    # reversed in time: G_t = dout_t + a_{t+1} G_{t+1}, from the gradient of the state after the last token
    later = torch.cat([a[:, 1:], a.new_ones(B, 1, C)], 1)
    grad = _scan(later.flip(1), dout.flip(1), s["dstate_out"]).flip(1)
    before = torch.cat([first[:, None], h[:, :-1]], 1)
    per_log = grad * (a * before - inp * x * a * a / m)
    out = [grad * m * inp, per_log * decay * sig * (1 - sig), grad * m * x * inp * (1 - inp), per_log * sig]
    if live is not None:
        out = [torch.where(live, v, 0.0) for v in out]
    s["dx"].copy_(out[0]), s["dr"].copy_(out[1]), s["dg"].copy_(out[2])
    s["dstate_in"].copy_(a[:, 0] * grad[:, 0])
    return s["dx"], s["dr"], s["dg"], out[3].sum((0, 1)), s["dstate_in"]


def _scan(a, b, first):
    """h_t = a_t h_{t-1} + b_t along dimension 1 by doubling (b is overwritten)."""
    n, k = a.shape[1], 1
    a, b[:, 0] = a.clone(), b[:, 0] + a[:, 0] * first
    while k < n:
        b[:, k:] += a[:, k:] * b[:, :-k].clone()
        a[:, k:] *= a[:, :-k].clone()
        k *= 2
    return b


def _words(rows, C, seed, offset):
    """32 random bits for each value: word c % 4 of Philox4x32-10 at (c / 4, row, offset) under the seed."""
    low = 0xFFFFFFFF
    c = [torch.arange(-(-C // 4), device=DEV)[None], torch.arange(rows, device=DEV)[:, None]]
    c = list(torch.broadcast_tensors(*c)) + [offset & low, offset >> 32]
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        p0, p1 = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(p1 >> 32) & low ^ c[1] ^ k0, p1 & low, (p0 >> 32) & low ^ c[3] ^ k1, p0 & low]
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack(c, -1).flatten(1)[:, :C]


def _kept(s, case, shape):
    """What dropout multiplies by: 0 or 1 / (1 - p)."""
    p = case["drop"]
    if not p:
        return None
    keep = _words(shape[0] * shape[1], shape[2], s["seed"], s["offset"]) >= int(p * 4294967296.0)
    return torch.where(keep, 1 / (1 - p), 0.0).view(shape)


def _activation(act, v):
    """(value, slope)."""
    if act == LINEAR:
        return v, torch.ones_like(v)
    sig = _sigmoid(v)
    if act == SIGMOID:
        return sig, sig * (1 - sig)
    return v * sig, sig * (1 + v * (1 - sig))


def _plain_norm(s, case):
    T = s["x"].dtype
    x, y, scale = s["x"].float(), s["y"].float(), s["scale"].float()
    w_post = s["w_post"].float() if case["post"] else 1.0
    r1 = torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) if case["post"] else 1.0
    unit = y * r1
    a, slope = _activation(case["act"], s["gate"].float()) if case["gated"] else (1.0, None)
    kept = _kept(s, case, x.shape)
    kept = 1.0 if kept is None else kept
    x_out = s["alpha"] * x + kept * scale * a * unit * w_post
    r2 = torch.rsqrt((x_out * x_out).mean(-1, keepdim=True) + EPS) if case["pre"] else None
    if case["kind"] == "forward":
        return [x_out.to(T)] + ([(x_out * r2 * s["w_pre"].float()).to(T)] if case["pre"] else [])
    t = s["dx_out"].float()
    if case["pre"]:
        dh, hat = s["dh"].float(), x_out * r2
        gw = dh * s["w_pre"].float()
        t = t + r2 * (gw - hat * (gw * hat).mean(-1, keepdim=True))
        dw_pre = (dh * hat).sum((0, 1))
    through = t * kept * a
    dn = through * scale
    got = [(s["alpha"] * t).to(T)]
    if case["post"]:
        gw = dn * w_post
        got.append((r1 * (gw - unit * (gw * unit).mean(-1, keepdim=True))).to(T))
    else:
        got.append(dn.to(T))
    if case["gated"]:
        got.append((t * kept * scale * unit * w_post * slope).to(T))
    if case["post"]:
        got.append((dn * unit).sum((0, 1)))
    got.append((through * unit * w_post).sum((0, 1)))
    if case["pre"]:
        got.append(dw_pre)
    return got


def _plain_ffn(s, case):
    T = s["x"].dtype
    x, w = s["x"].float(), s["w"].float()
    gate, up = x @ w[0].t(), x @ w[1].t()
    a, slope = _activation(case["act"], gate)
    if case["kind"] == "forward":
        return (a * up).to(T)
    dout = s["dout"].float()
    dgate, dup = dout * up * slope, dout * a
    dx = dgate @ w[0] + dup @ w[1]
    return dx.to(T), torch.stack([dgate.t() @ x, dup.t() @ x]).to(T)


# ------------------------------------------------------------------------------------------------
# the least work of one pass
# ------------------------------------------------------------------------------------------------

def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "ffn":
        M, K, F = case["rows"], case["K"], case["F"]
        if case["kind"] == "gradient":
            return {"bytes": (2 * M * K + M * F + 4 * F * K) * e, "flops": 12 * M * K * F}
        return {"bytes": (M * K + M * F + 2 * F * K) * e, "flops": 4 * M * K * F}
    B, n, C = case["B"], case["n"], case["C"]
    v = B * n * C
    if case["op"] == "glr":
        states = B * C * 4 * (1 + (case["carried"] or case["kind"] == "token"))
        if case["kind"] == "gradient":
            # (with the state before every 32nd token, without which the tokens are read a second time)
            return {"bytes": 7 * v * e + B * -(-n // 32) * C * 4 + 2 * B * C * 4 + 2 * C * 4, "flops": 45 * v}
        return {"bytes": 4 * v * e + states + C * 4, "flops": 20 * v}
    tensors = 2 + case["gated"]
    if case["kind"] == "gradient":
        sums = C * 4 * (1 + case["post"] + case["pre"])
        return {"bytes": (2 * tensors + 1 + case["pre"]) * v * e + 3 * C * e + sums, "flops": 50 * v}
    return {"bytes": (tensors + 1 + case["pre"]) * v * e + 3 * C * e, "flops": 20 * v}


# ------------------------------------------------------------------------------------------------
# the definition in 64 bits
# ------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"glr": _exact_glr, "norm": _exact_norm, "ffn": _exact_ffn}[case["op"]](s, case)


def _exact_glr(s, case):
    token, back = case["kind"] == "token", case["kind"] == "gradient"
    x, r, g = ((s[k][:, None] if token else s[k]).double().detach().clone().requires_grad_(back) for k in ("x", "r", "g"))
    B, n, C = x.shape
    if n > 16384 and back:
        return None
    decay = s["decay"].double().detach().clone().requires_grad_(back)
    first = s["state"].double() if token or case["carried"] else x.new_zeros(B, C)
    first = first.detach().clone().requires_grad_(back)
    log_a = decay * torch.sigmoid(r)
    keep = log_a.exp()
    add = (-torch.expm1(2 * log_a)).sqrt() * torch.sigmoid(g) * x
    length = [n] * B if s["lengths"] is None else s["lengths"].tolist()
    end = torch.tensor(length, device=DEV)[:, None]
    whole = min(length)
    rows, h = [], first
    for t, (k, b) in enumerate(zip(keep.unbind(1), add.unbind(1))):
        new = torch.addcmul(b, k, h)
        h = new if t < whole else torch.where(t < end, new, h)
        rows.append(h)
    out = torch.stack(rows, 1)
    out = out.masked_fill(torch.arange(n, device=DEV)[None, :, None] >= end[..., None], 0.0)
    if back:
        grads = torch.autograd.grad((out, h), (x, r, g, decay, first), (s["dout"].double(), s["dstate_out"].double()))
        return grads
    return (out[:, 0] if token else out), h


def _exact_words(rows, C, seed, offset):
    """Philox4x32-10 by its rounds, in numpy's unsigned integers."""
    u, low, half = np.uint64, np.uint64(0xFFFFFFFF), np.uint64(32)
    groups = (C + 3) // 4
    ctr = np.empty((4, rows, groups), dtype=u)
    ctr[0], ctr[1] = np.arange(groups, dtype=u), np.arange(rows, dtype=u)[:, None]
    ctr[2], ctr[3] = u(offset % 2 ** 32), u(offset // 2 ** 32)
    key = [seed % 2 ** 32, seed // 2 ** 32]
    for rnd in range(10):
        a, b = ctr[0] * u(0xD2511F53), ctr[2] * u(0xCD9E8D57)
        k = [u((key[i] + rnd * w) % 2 ** 32) for i, w in enumerate((0x9E3779B9, 0xBB67AE85))]
        ctr[0], ctr[2] = (b >> half) ^ ctr[1] ^ k[0], (a >> half) ^ ctr[3] ^ k[1]
        ctr[1], ctr[3] = b & low, a & low
    return np.moveaxis(ctr, 0, -1).reshape(rows, groups * 4)[:, :C]


def _exact_norm(s, case):
    names = ["x", "y"] + ["gate"] * case["gated"] + ["w_post"] * case["post"] + ["scale"] + ["w_pre"] * case["pre"]
    v = {k: s[k].double().detach().clone().requires_grad_() for k in names}
    B, n, C = v["x"].shape
    f = v["y"]
    if case["post"]:
        f = f / (f.square().mean(-1, keepdim=True) + EPS).sqrt() * v["w_post"]
    if case["gated"]:
        f = f * {LINEAR: lambda t: t, SIGMOID: torch.sigmoid, SILU: torch.nn.functional.silu}[case["act"]](v["gate"])
    f = f * v["scale"]
    if case["drop"]:
        kept = _exact_words(B * n, C, s["seed"], s["offset"]) >= np.uint64(int(case["drop"] * 2.0 ** 32))
        f = f * torch.from_numpy(kept).to(DEV).view(B, n, C) / (1 - case["drop"])
    out = [s["alpha"] * v["x"] + f]
    if case["pre"]:
        out.append(out[0] / (out[0].square().mean(-1, keepdim=True) + EPS).sqrt() * v["w_pre"])
    if case["kind"] == "forward":
        return [t.detach() for t in out]
    return list(torch.autograd.grad(out, [v[k] for k in names], [s[k].double() for k in ("dx_out", "dh")[:len(out)]]))


def _exact_ffn(s, case):
    if case["rows"] * case["K"] * case["F"] > 2e11:
        return None
    back = case["kind"] == "gradient"
    x, w = (s[k].double().detach().clone().requires_grad_(back) for k in ("x", "w"))
    z = torch.nn.functional.linear(x, w.flatten(0, 1))
    gate, up = z.chunk(2, -1)
    out = (torch.nn.functional.silu(gate) if case["act"] == SILU else torch.sigmoid(gate)) * up
    return torch.autograd.grad(out, (x, w), s["dout"].double()) if back else out
