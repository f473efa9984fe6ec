"""The operators around and beside the HLA mixers, as cases that can be timed and checked:

  conv    the short causal depthwise convolution: prompts, its gradient, single tokens
  scan    the selective state space scan: prompts, single tokens
  heads   the norm of queries and keys for each head with the position rotation: forward, gradient

``run`` computes a case with elementary torch operations in 32 bits, or, where ``own`` is true, with
the library's entry points.  ``exact`` computes it from the definition in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
CHUNK = 64  # of the plain scan


def listed():
    return [
        # conv: the x, B and C channels of a layer of 32 heads of 64 (2048 + 2 * 128) over two long prompts
        conv("conv_prompt_bf16", "prompt", "bf16", 2, 8192, 2304),
        # a ragged batch that continues from kept states: odd channel count, three taps, 32 bits
        conv("conv_ragged_f32", "prompt", "f32", 5, 333, 203, width=3, ragged=True, carried=True),
        # the gradient in a training step, 16 heads of 64 (1024 + 2 * 128)
        conv("conv_gradient_bf16", "gradient", "bf16", 8, 2048, 1280),
        # one token for each of 64 sequences
        conv("conv_token_bf16", "token", "bf16", 64, 1, 2304),
        # scan: a batch of prompts; the batch and length of the framework's head-size-64 workload
        scan("scan_prompts_bf16", "prompt", "bf16", 8, 2048, 32, 64, 1, 128),
        # one long prompt with few heads: the work has to be split along the sequence
        scan("scan_long_bf16", "prompt", "bf16", 1, 32768, 16, 64, 2, 64),
        # ragged prompts that continue from kept states, small heads, 32 bits
        scan("scan_ragged_f32", "prompt", "f32", 3, 517, 6, 32, 2, 16, ragged=True, carried=True),
        # one token for each of 64 sequences, as the decode workload has it
        scan("scan_token_bf16", "token", "bf16", 64, 1, 32, 64, 1, 128),
        # one token of one sequence: latency
        scan("scan_token_one_bf16", "token", "bf16", 1, 1, 16, 64, 1, 128),
        # heads: before the framework's head-size-64 training workload
        heads("heads_train_bf16", "prompt", "bf16", 8, 2048, 16, 16, 64, 64),
        # its gradient with four query heads to a key head
        heads("heads_gradient_bf16", "gradient", "bf16", 8, 2048, 16, 4, 64, 64),
        # one token for each of 64 sequences, part of each head rotated
        heads("heads_token_bf16", "token", "bf16", 64, 1, 32, 8, 128, 64),
    ]


def conv(name, kind, dtype, B, n, C, width=4, ragged=False, carried=False, silu=True):
    return {"name": name, "op": "conv", "kind": kind, "dtype": dtype, "B": B, "n": n, "C": C, "width": width,
            "ragged": ragged, "carried": carried, "silu": silu}


def scan(name, kind, dtype, B, n, H, P, G, N, ragged=False, carried=False):
    return {"name": name, "op": "scan", "kind": kind, "dtype": dtype, "B": B, "n": n, "H": H, "P": P, "G": G,
            "N": N, "ragged": ragged, "carried": carried}


def heads(name, kind, dtype, B, n, H, Hk, d, rot, interleaved=False):
    return {"name": name, "op": "heads", "kind": kind, "dtype": dtype, "B": B, "n": n, "H": H, "Hk": Hk, "d": d,
            "rot": rot, "interleaved": interleaved}


def draw(rng):
    """One more case: an operator, a direction, a type, and sizes spread over the listed range."""
    def log(lo, hi):
        v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return v + 1 if v == 3072 else v

    op = rng.choice(["conv", "conv", "scan", "scan", "heads"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    top = 64e6 if dtype == "bf16" else 16e6  # values of a token tensor
    flag = lambda: rng.random() < 0.5  # noqa: E731
    if op == "conv":
        kind = rng.choice(["prompt", "prompt", "gradient", "token"])
        C = log(24, 4096)
        B = log(1, 64)
        n = 1 if kind == "token" else log(1, max(2, min(16384, top / (B * C) / (3 if kind == "gradient" else 2))))
        c = conv("", kind, dtype, B, n, C, rng.choice([2, 3, 4, 4]), kind != "token" and flag(),
                 kind == "prompt" and flag(), flag())
    elif op == "scan":
        kind = rng.choice(["prompt", "prompt", "token"])
        G = rng.choice([1, 1, 2, 4])
        H, P, N = G * log(1, 16), rng.choice([16, 32, 64, 64, 128]), rng.choice([16, 32, 64, 128, 128])
        if H * P == 3072:
            H += G
        B = log(1, max(1, min(64, 16e6 / (H * N * P))) if kind == "token" else 16)
        n = 1 if kind == "token" else log(1, max(2, min(32768, top / (8 if dtype == "f32" else 2) / (B * H * P), 8e6 / (B * G * N))))
        c = scan("", kind, dtype, B, n, H, P, G, N, kind != "token" and flag(), kind == "prompt" and flag())
    else:
        kind = rng.choice(["prompt", "gradient", "token"])
        Hk = log(1, 16)
        H, d = Hk * rng.choice([1, 2, 4]), rng.choice([16, 32, 64, 64, 128])
        if H * d == 3072 or Hk * d == 3072:
            Hk, H = Hk + 1, H // Hk * (Hk + 1)
        B = log(1, 64 if kind == "token" else 16)
        n = 1 if kind == "token" else log(1, max(2, min(16384, top / 4 / (B * H * d))))
        c = heads("", kind, dtype, B, n, H, Hk, d, rng.choice([d, d // 2, 0]), flag())
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------

def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 17)
    T = TYPES[case["dtype"]]

    def normal(*shape, scale=1.0, dtype=T):
        return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)

    def uniform(lo, hi, *shape):
        return torch.rand(shape, generator=g, device=DEV) * (hi - lo) + lo

    def some_lengths(B, n):  # any length, none and all among them
        v = torch.randint(0, n + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
        v[B - 1] = n
        return v

    B, n = case["B"], case["n"]
    s = {"case": case}
    if own:
        from paper_2510_27258_gb300 import hla
        s["hla"] = hla
    if case["op"] == "conv":
        C, W = case["C"], case["width"]
        pad = -(-C // 8) * 8 + 64  # the channels are a slice of a wider projection
        s["x"] = normal(B, n, pad)[..., :C]
        s["w"] = normal(C, W, scale=W ** -0.5)
        s["bias"] = normal(C, scale=0.1)
        s["lengths"] = some_lengths(B, n) if case["ragged"] else None
        if case["kind"] == "gradient":
            s["dout"] = normal(B, n, C)
            s["dx"] = torch.empty(B, n, C, dtype=T, device=DEV)
            if own:
                s["ws"] = hla.alloc_workspace(hla.hla_conv_backward_workspace_bytes(B, n, C, W, T), DEV)
        else:
            s["state"] = normal(B, W - 1, C)
            s["out"] = torch.empty(B, n, C, dtype=T, device=DEV)
            s["state_out"] = torch.empty(B, W - 1, C, dtype=T, device=DEV)
        if case["kind"] == "token":
            s["x"], s["out"] = s["x"][:, 0], s["out"][:, 0]
    elif case["op"] == "scan":
        H, P, G, N = case["H"], case["P"], case["G"], case["N"]
        rows = normal(B, n, H * P + 2 * G * N)  # the convolution's output: x, B, C side by side
        rows = (rows.float() * torch.sigmoid(rows.float())).to(T)
        s["x"] = rows[..., :H * P].unflatten(-1, (H, P))
        s["b"] = rows[..., H * P:H * P + G * N].unflatten(-1, (G, N))
        s["c"] = rows[..., H * P + G * N:].unflatten(-1, (G, N))
        s["delta"] = normal(B, n, -(-H // 8) * 8, scale=0.5)[..., :H]
        s["a"] = -uniform(1.0, 16.0, H)
        step = torch.exp(uniform(math.log(1e-3), math.log(1e-1), H))
        s["bias"] = step + torch.log(-torch.expm1(-step))  # softplus(bias) = step
        s["skip"] = uniform(0.5, 1.5, H)
        s["lengths"] = some_lengths(B, n) if case["ragged"] else None
        s["state"] = normal(B, H, N, P, scale=0.1, dtype=torch.float32)
        s["out"] = torch.empty(B, n, H, P, dtype=T, device=DEV)
        s["state_out"] = torch.empty(B, H, N, P, dtype=torch.float32, device=DEV)
        if case["kind"] == "token":
            for name in ("x", "b", "c", "delta", "out"):
                s[name] = s[name][:, 0]
        elif own:
            s["ws"] = hla.alloc_workspace(hla.hla_ssm_workspace_bytes(B, n, H, P, G, N, T), DEV)
    else:
        H, Hk, d, rot = case["H"], case["Hk"], case["d"], case["rot"]
        rows = normal(B, n, (H + 2 * Hk) * d)  # the projection's output: q, k, v side by side
        s["q"] = rows[..., :H * d].unflatten(-1, (H, d))
        s["k"] = rows[..., H * d:(H + Hk) * d].unflatten(-1, (Hk, d))
        s["wq"], s["wk"] = (1 + normal(d, scale=0.2, dtype=torch.float32)).to(T), (1 + normal(d, scale=0.2, dtype=torch.float32)).to(T)
        top = 8192 if case["kind"] == "token" else n
        angle = torch.arange(top, device=DEV, dtype=torch.float64)[:, None] * \
            10000.0 ** (-torch.arange(rot // 2, device=DEV, dtype=torch.float64) * 2 / max(rot, 1))
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        s["positions"] = None
        if case["kind"] == "token":
            s["positions"] = torch.randint(0, top, (B, n), generator=g, device=DEV, dtype=torch.int32)
        if case["kind"] == "gradient":
            s["dq_out"], s["dk_out"] = normal(B, H, n, d), normal(B, H, n, d)
            if own:
                s["ws"] = hla.alloc_workspace(hla.hla_qk_norm_backward_workspace_bytes(B, n, H, Hk, d, T), DEV)
        else:
            s["q_out"] = torch.empty(B, H, n, d, dtype=T, device=DEV)
            s["k_out"] = torch.empty(B, H, n, d, dtype=T, device=DEV)
    return s


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------

EPS = 1e-6


def run(s):
    case = s["case"]
    if own:
        return _own(s["hla"], s, case)
    return {"conv": _plain_conv, "scan": _plain_scan, "heads": _plain_heads}[case["op"]](s, case)


def _own(hla, s, case):
    kind = case["kind"]
    if case["op"] == "conv":
        if kind == "token":
            hla.hla_conv_step(s["x"], s["w"], s["state"], s["bias"], s["out"], silu=case["silu"])
            return s["out"], s["state"]
        if kind == "gradient":
            return hla.hla_conv_backward(s["x"], s["w"], s["dout"], s["bias"], s["dx"], silu=case["silu"],
                                         lengths=s["lengths"], workspace=s["ws"])
        hla.hla_conv_forward(s["x"], s["w"], s["bias"], s["out"], silu=case["silu"], lengths=s["lengths"],
                             state_in=s["state"] if case["carried"] else None, state_out=s["state_out"])
        return s["out"], s["state_out"]
    if case["op"] == "scan":
        if kind == "token":
            hla.hla_ssm_step(s["x"], s["delta"], s["a"], s["b"], s["c"], s["state"], s["out"], skip=s["skip"],
                             delta_bias=s["bias"])
            return s["out"], s["state"]
        hla.hla_ssm_forward(s["x"], s["delta"], s["a"], s["b"], s["c"], s["out"], skip=s["skip"],
                            delta_bias=s["bias"], lengths=s["lengths"],
                            state_in=s["state"] if case["carried"] else None, state_out=s["state_out"],
                            workspace=s["ws"])
        return s["out"], s["state_out"]
    if kind == "gradient":
        return hla.hla_qk_norm_backward(s["q"], s["k"], s["wq"], s["wk"], s["cos"], s["sin"], s["dq_out"],
                                        s["dk_out"], positions=s["positions"], eps=EPS,
                                        interleaved=case["interleaved"], workspace=s["ws"])
    return hla.hla_qk_norm_forward(s["q"], s["k"], s["wq"], s["wk"], s["cos"], s["sin"], s["q_out"], s["k_out"],
                                   positions=s["positions"], eps=EPS, interleaved=case["interleaved"])


def _plain_conv(s, case):
    T, W, n = s["x"].dtype, case["width"], case["n"]
    x, w, bias = s["x"].float(), s["w"].float(), s["bias"].float()
    if case["kind"] == "token":
        win = torch.cat([s["state"].float(), x[:, None]], 1)
        pre = (win * w.t()).sum(1) + bias
        s["state"].copy_(win[:, 1:])
        s["out"].copy_(pre / (1 + torch.exp(-pre)) if case["silu"] else pre)
        return s["out"], s["state"]
    live = None
    if s["lengths"] is not None:
        live = (torch.arange(n, device=DEV) < s["lengths"][:, None])[..., None]
    first = s["state"].float() if case["carried"] else x.new_zeros(x.shape[0], W - 1, x.shape[2])
    xp = torch.cat([first, x], 1)
    pre = bias + sum(w[:, j] * xp[:, j:j + n] for j in range(W))
    if case["kind"] == "gradient":
        g = s["dout"].float()
        if case["silu"]:
            sig = 1 / (1 + torch.exp(-pre))
            g = g * sig * (1 + pre * (1 - sig))
        if live is not None:
            g = torch.where(live, g, 0.0)
        gp = torch.cat([g, g.new_zeros(g.shape[0], W - 1, g.shape[2])], 1)
        dx = sum(w[:, j] * gp[:, W - 1 - j:W - 1 - j + n] for j in range(W))
        dw = torch.stack([(g * xp[:, j:j + n]).sum((0, 1)) for j in range(W)], 1)
        return dx.to(T), dw, g.sum((0, 1))
    out = pre / (1 + torch.exp(-pre)) if case["silu"] else pre
    if live is not None:
        out = torch.where(live, out, 0.0)
        at = s["lengths"].long()[:, None] + torch.arange(W - 1, device=DEV)
        last = xp[torch.arange(x.shape[0], device=DEV)[:, None], at]
    else:
        last = xp[:, n:]
    return out.to(T), last.to(T)


def _softplus(v):
    return torch.where(v > 0, v, 0.0) + torch.log1p(torch.exp(-v.abs()))


def _plain_scan(s, case):
    T, per = s["x"].dtype, case["H"] // case["G"]
    H, P, N, B, n = case["H"], case["P"], case["N"], case["B"], case["n"]
    dl = _softplus(s["delta"].float() + s["bias"])
    if case["kind"] == "token":
        b, c = (s[k].float().repeat_interleave(per, 1) for k in ("b", "c"))
        x = s["x"].float()
        s["state"].mul_(torch.exp(dl * s["a"])[..., None, None]).add_((dl[..., None] * b)[..., None] * x[:, :, None])
        s["out"].copy_((c[..., None] * s["state"]).sum(2) + s["skip"][:, None] * x)
        return s["out"], s["state"]
    x, b, c = s["x"].float(), s["b"].float(), s["c"].float()
    if s["lengths"] is not None:
        live = torch.arange(n, device=DEV) < s["lengths"][:, None]
        dl = torch.where(live[..., None], dl, 0.0)
    Z = -(-n // CHUNK)

    def chunks(v):  # [B, n, ...] -> [B, Z, CHUNK, ...]
        v = torch.cat([v, v.new_zeros((B, Z * CHUNK - n) + v.shape[2:])], 1)
        return v.unflatten(1, (Z, CHUNK))

    xc, bc, cc, dc = chunks(x), chunks(b), chunks(c), chunks(dl).transpose(2, 3)  # dc: [B, Z, H, Q]
    la = dc * s["a"][:, None]
    cum = la.cumsum(-1)
    after = la.flip(-1).cumsum(-1).flip(-1) - la  # decay that follows a token in its chunk
    low = torch.ones(CHUNK, CHUNK, dtype=torch.bool, device=DEV).tril()
    dec = torch.exp(torch.where(low, cum[..., :, None] - cum[..., None, :], -math.inf))
    w = torch.einsum("bzqgn,bzkgn->bzgqk", cc, bc).repeat_interleave(per, 2) * dec * dc[..., None, :]
    del dec
    y = torch.einsum("bzhqk,bzkhp->bzqhp", w, xc)
    del w
    wx = (torch.exp(after) * dc).transpose(2, 3)[..., None] * xc
    loc = torch.einsum("bzkgn,bzkgjp->bzgjnp", bc, wx.unflatten(3, (case["G"], per))).flatten(2, 3)
    del wx
    tot = cum[..., -1].transpose(1, 2)  # [B, H, Z]
    # carry[z, c]: decay of what chunk c leaves until chunk z begins (z = Z: until the end)
    ones = torch.ones(Z + 1, Z, dtype=torch.bool, device=DEV)
    step = torch.where(ones.tril(-2), torch.cat([tot.new_zeros(B, H, 1), tot], -1)[..., None], 0.0)
    carry = torch.exp(torch.where(ones.tril(-1), step.cumsum(2), -math.inf))
    hs = torch.einsum("bhzc,bchnp->bzhnp", carry, loc)
    if case["carried"]:
        hs = hs + torch.exp(torch.cat([tot.new_zeros(B, H, 1), tot.cumsum(-1)], -1)).transpose(1, 2)[..., None, None] * s["state"][:, None]
    y = y + torch.einsum("bzqgn,bzgjnp->bzqgjp", cc, hs[:, :Z].unflatten(2, (case["G"], per))).flatten(3, 4) * \
        torch.exp(cum).transpose(2, 3)[..., None]
    y = y.flatten(1, 2)[:, :n] + s["skip"][:, None] * x
    if s["lengths"] is not None:
        y = torch.where(live[..., None, None], y, 0.0)
    return y.to(T), hs[:, Z].contiguous()


def _turn(s, case, v, back):
    """The rotation of [B, n, heads, d] by the positions' angles, or its inverse."""
    rot = case["rot"]
    if not rot:
        return v
    if s["positions"] is not None:
        cs, sn = s["cos"][s["positions"].long()], s["sin"][s["positions"].long()]
    else:
        cs, sn = s["cos"][None, :case["n"]], s["sin"][None, :case["n"]]
    cs, sn = cs[:, :, None], -sn[:, :, None] if back else sn[:, :, None]
    if case["interleaved"]:
        a, b = v[..., 0:rot:2], v[..., 1:rot:2]
        r = torch.stack([a * cs - b * sn, b * cs + a * sn], -1).flatten(-2)
    else:
        a, b = v[..., :rot // 2], v[..., rot // 2:rot]
        r = torch.cat([a * cs - b * sn, b * cs + a * sn], -1)
    return torch.cat([r, v[..., rot:]], -1)


def _plain_heads(s, case):
    per, got = case["H"] // case["Hk"], []
    for name in ("q", "k"):
        v, w = s[name].float(), s["w" + name].float()
        r = torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS)
        if case["kind"] == "gradient":
            g = s["d" + name + "_out"].float().transpose(1, 2)
            if name == "k":
                g = g.unflatten(2, (case["Hk"], per)).sum(3)
            g = _turn(s, case, g, True)
            unit = v * r
            gw = g * w
            got.append((r * (gw - unit * (gw * unit).mean(-1, keepdim=True))).to(s[name].dtype))
            got.append((g * unit).sum((0, 1, 2)))
        else:
            y = _turn(s, case, v * r * w, False).transpose(1, 2)
            if name == "k":
                y = y.repeat_interleave(per, 1)
            got.append(s[name + "_out"].copy_(y))
    return (got[0], got[2], got[1], got[3]) if case["kind"] == "gradient" else tuple(got)


# ------------------------------------------------------------------------------------------------
# the least work of one pass
# ------------------------------------------------------------------------------------------------

def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    B, n = case["B"], case["n"]
    if case["op"] == "conv":
        C, W = case["C"], case["width"]
        v = B * n * C
        w = C * (W + 1) * e
        if case["kind"] == "gradient":
            return {"bytes": 3 * v * e + w + C * (W + 1) * 4, "flops": v * (6 * W + 10)}
        states = B * (W - 1) * C * e * (1 + (case["carried"] or case["kind"] == "token"))
        return {"bytes": 2 * v * e + w + states, "flops": v * (2 * W + 5)}
    if case["op"] == "scan":
        H, P, G, N = case["H"], case["P"], case["G"], case["N"]
        states = B * H * N * P * 4 * (1 + (case["carried"] or case["kind"] == "token"))
        return {"bytes": B * n * (2 * H * P + 2 * G * N + H) * e + states + H * 12, "flops": B * n * H * N * P * 4}
    H, Hk, d, rot = case["H"], case["Hk"], case["d"], case["rot"]
    rows = B * n
    table = (n if case["kind"] != "token" else rows) * rot * 4
    if case["kind"] == "gradient":
        return {"bytes": rows * (2 * (H + Hk) + 2 * H) * d * e + table + 2 * d * (e + 4),
                "flops": rows * d * (14 * (H + Hk) + H)}
    return {"bytes": rows * ((H + Hk) + 2 * H) * d * e + table + 2 * d * e, "flops": rows * d * 7 * (H + Hk)}


# ------------------------------------------------------------------------------------------------
# the definition in 64 bits
# ------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"conv": _exact_conv, "scan": _exact_scan, "heads": _exact_heads}[case["op"]](s, case)


def _exact_conv(s, case):
    W, B, C = case["width"], case["B"], case["C"]
    token = case["kind"] == "token"
    x = s["x"].double()
    x = x[:, None] if token else x
    n = x.shape[1]
    if B * n * C * W > 1.2e9:
        return None
    first = s["state"].double() if token or case["carried"] else x.new_zeros(B, W - 1, C)
    length = [n] * B if s["lengths"] is None else s["lengths"].tolist()
    w, bias = s["w"].double(), s["bias"].double()
    if case["kind"] == "gradient":
        x, w, bias = x.clone().requires_grad_(), w.requires_grad_(), bias.requires_grad_()
    rows = torch.cat([first, x], 1)
    out = torch.einsum("bncw,cw->bnc", rows.unfold(1, W, 1), w) + bias
    if case["silu"]:
        out = torch.nn.functional.silu(out)
    keep = torch.zeros(B, n, 1, dtype=torch.bool, device=DEV)
    for i, m in enumerate(length):
        keep[i, :m] = True
    out = out.masked_fill(~keep, 0.0)
    if case["kind"] == "gradient":
        return torch.autograd.grad(out, (x, w, bias), s["dout"].double().masked_fill(~keep, 0.0))
    last = torch.stack([rows[i, m:m + W - 1] for i, m in enumerate(length)])
    return (out[:, 0], last) if token else (out, last)


def _exact_scan(s, case):
    B, n, H, G, N, P = (case[k] for k in ("B", "n", "H", "G", "N", "P"))
    token = case["kind"] == "token"
    up = lambda v: (v[:, None] if token else v).double()  # noqa: E731
    x, b, c = up(s["x"]), up(s["b"]), up(s["c"])
    delta = torch.nn.functional.softplus(up(s["delta"]) + s["bias"].double(), threshold=1e9)
    # a pass over the tokens costs about the state's size a token, or the launches
    if n * max(B * H * N * P / 2e11, 4e-5) > 12:
        return None
    h = s["state"].double().clone() if token or case["carried"] else x.new_zeros(B, H, N, P)
    h = h.view(B, G, H // G, N, P)
    length = torch.full((B,), n, device=DEV) if s["lengths"] is None else s["lengths"].long()
    y = x.new_zeros(B, n, H, P)
    decay = torch.exp(delta * s["a"].double())
    for t in range(n):
        live = (t < length)[:, None, None, None, None]
        if s["lengths"] is None:
            live = None
        a = decay[:, t].view(B, G, H // G, 1, 1)
        dx = (delta[:, t, :, None] * x[:, t]).view(B, G, H // G, 1, P)
        new = a * h + b[:, t].view(B, G, 1, N, 1) * dx
        h = new if live is None else torch.where(live, new, h)
        y[:, t] = torch.matmul(c[:, t].view(B, G, 1, 1, N), h).view(B, H, P)
    y = y + s["skip"].double()[:, None] * x
    y = y * (torch.arange(n, device=DEV) < length[:, None])[..., None, None]
    return (y[:, 0] if token else y), h.reshape(B, H, N, P)


def _exact_heads(s, case):
    B, n, H, Hk, d, rot = (case[k] for k in ("B", "n", "H", "Hk", "d", "rot"))
    at = torch.arange(n, device=DEV).expand(B, n) if s["positions"] is None else s["positions"].long()
    turn = torch.complex(s["cos"].double(), s["sin"].double())[at][:, None]  # [B, 1, n, rot / 2]
    got = []
    for name in ("q", "k"):
        v, w = s[name].double().detach().clone().requires_grad_(), s["w" + name].double().requires_grad_()
        y = (v / (v.square().mean(-1, keepdim=True) + EPS).sqrt() * w).permute(0, 2, 1, 3)
        if rot:
            inter = case["interleaved"]
            pairs = y[..., :rot].unflatten(-1, (rot // 2, 2) if inter else (2, rot // 2))
            pairs = pairs if inter else pairs.transpose(-1, -2)
            z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
            z = z if inter else z.transpose(-1, -2)
            y = torch.cat([z.flatten(-2), y[..., rot:]], -1)
        if name == "k":
            y = y[:, :, None].expand(B, Hk, H // Hk, n, d).reshape(B, H, n, d)
        got.append(torch.autograd.grad(y, (v, w), s["d" + name + "_out"].double()) if case["kind"] == "gradient" else y.detach())
    return (got[0][0], got[1][0], got[0][1], got[1][1]) if case["kind"] == "gradient" else tuple(got)
