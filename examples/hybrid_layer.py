"""A layer of two recurrent mixers side by side, as a serving or training program would run it:

    rows of one projection -> short convolution -> q/k norm with rotation -> second-order HLA heads
                                               `-> selective state space heads
    both outputs -> output projection

``prompt`` runs any number of prompts at once and leaves a constant-size state, ``token`` continues
each by one token, ``gradients`` is a training step through the HLA half.  Run it on a GB300:

    python examples/hybrid_layer.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2510_27258_gb300 import hla  # noqa: E402

WIDTH = 4  # taps of the convolution


class Layer:
    """Sizes and weights: H HLA heads of size d (Hk key heads), S scan heads of size P in G groups, N states."""

    def __init__(self, model, H=4, Hk=2, d=64, S=4, P=64, G=1, N=128, dtype=torch.bfloat16, device="cuda", seed=0,
                 positions=4096):
        g = torch.Generator().manual_seed(seed)
        self.H, self.Hk, self.d, self.S, self.P, self.G, self.N = H, Hk, d, S, P, G, N
        # channels of a projection row: q | k | v | x | b | c | raw steps
        self.parts = [H * d, Hk * d, H * d, S * P, G * N, G * N]
        self.C = sum(self.parts)

        def make(*shape, scale=1.0, kind=dtype):
            return (torch.randn(*shape, generator=g) * scale).to(device=device, dtype=kind)

        self.w_in = make(model, self.C + S, scale=model ** -0.5)
        self.w_out = make(H * d + S * P, model, scale=(H * d + S * P) ** -0.5)
        self.conv_w, self.conv_b = make(self.C, WIDTH, scale=WIDTH ** -0.5), make(self.C, scale=0.1)
        # unit norm after the weights: |q|^2 = |k|^2 = 1, as the HLA operators like their keys
        self.wq, self.wk = make(d, scale=0.0) + d ** -0.5, make(d, scale=0.0) + d ** -0.5
        angle = torch.arange(positions)[:, None] * 10000.0 ** (-torch.arange(d // 2) * 2.0 / d)
        self.cos, self.sin = angle.cos().to(device), angle.sin().to(device)
        self.a = -(torch.rand(S, generator=g) * 15 + 1).to(device)
        self.step_bias = torch.full((S,), -3.0, device=device)
        self.skip = torch.ones(S, device=device)

    def split(self, rows):
        """q, k, v, x, b, c of convolved rows, as views."""
        q, k, v, x, b, c = rows.split(self.parts, -1)
        return (q.unflatten(-1, (self.H, self.d)), k.unflatten(-1, (self.Hk, self.d)), v.unflatten(-1, (self.H, self.d)),
                x.unflatten(-1, (self.S, self.P)), b.unflatten(-1, (self.G, self.N)), c.unflatten(-1, (self.G, self.N)))

    def new_state(self, B):
        """Convolution rows, HLA tuples and scan states before the first token."""
        dev, T = self.w_in.device, self.w_in.dtype
        return {"conv": torch.zeros(B, WIDTH - 1, self.C, dtype=T, device=dev),
                "hla": torch.zeros(B, self.H, hla.hla2_state_floats(self.d, self.d), device=dev),
                "ssm": torch.zeros(B, self.S, self.N, self.P, device=dev), "at": 0}


def prompt(layer, tokens, state):
    """[B, n, model] -> [B, n, model]; ``state`` is updated to after the last token."""
    B, n, _ = tokens.shape
    rows = tokens @ layer.w_in
    conv = hla.hla_conv_forward(rows[..., :layer.C], layer.conv_w, layer.conv_b, state_in=state["conv"],
                                state_out=state["conv"])
    q, k, v, x, b, c = layer.split(conv)
    q, k = hla.hla_qk_norm_forward(q, k, layer.wq, layer.wk, layer.cos, layer.sin, pos0=state["at"])
    mixed = hla.hla2_forward(q, k, v.transpose(1, 2).contiguous(), state_in=state["hla"], state_out=state["hla"])
    scanned = hla.hla_ssm_forward(x, rows[..., layer.C:], layer.a, b, c, skip=layer.skip, delta_bias=layer.step_bias,
                                  state_in=state["ssm"], state_out=state["ssm"])
    state["at"] += n
    return torch.cat([mixed.transpose(1, 2).flatten(2), scanned.flatten(2)], -1) @ layer.w_out


def token(layer, tokens, state):
    """One token a sequence: [B, model] -> [B, model], the state updated in place."""
    rows = tokens @ layer.w_in
    conv = hla.hla_conv_step(rows[:, :layer.C], layer.conv_w, state["conv"], layer.conv_b)
    q, k, v, x, b, c = layer.split(conv)
    q, k = hla.hla_qk_norm_forward(q[:, None], k[:, None], layer.wq, layer.wk, layer.cos, layer.sin, pos0=state["at"])
    mixed = hla.hla2_step(q[:, :, 0], k[:, :, 0], v.contiguous(), state["hla"])
    scanned = hla.hla_ssm_step(x, rows[:, layer.C:], layer.a, b, c, state["ssm"], skip=layer.skip,
                               delta_bias=layer.step_bias)
    state["at"] += 1
    return torch.cat([mixed.flatten(1), scanned.flatten(1)], -1) @ layer.w_out


def hla_half(layer, tokens):
    """The HLA heads' output [B, H, n, d] from an empty state, and what its gradients need."""
    used = sum(layer.parts[:3])
    rows = (tokens @ layer.w_in[:, :used])
    conv = hla.hla_conv_forward(rows, layer.conv_w[:used], layer.conv_b[:used])
    q, k, v = conv.split(layer.parts[:3], -1)
    q, k = q.unflatten(-1, (layer.H, layer.d)), k.unflatten(-1, (layer.Hk, layer.d))
    v = v.unflatten(-1, (layer.H, layer.d)).transpose(1, 2).contiguous()
    qn, kn = hla.hla_qk_norm_forward(q, k, layer.wq, layer.wk, layer.cos, layer.sin)
    return hla.hla2_forward(qn, kn, v), (rows, q, k, qn, kn, v)


def gradients(layer, tokens, dout):
    """Gradients of sum(dout * output of the HLA half): of the tokens and of every weight before it."""
    _, (rows, q, k, qn, kn, v) = hla_half(layer, tokens)
    used = rows.shape[-1]
    dqn, dkn, dv = hla.hla2_backward(qn, kn, v, dout)
    dconv = torch.empty_like(rows)  # the gradients of q, k and v are written side by side
    dq, dk, dvr = dconv.split(layer.parts[:3], -1)
    _, _, dwq, dwk = hla.hla_qk_norm_backward(q, k, layer.wq, layer.wk, layer.cos, layer.sin, dqn, dkn,
                                              dq.unflatten(-1, (layer.H, layer.d)),
                                              dk.unflatten(-1, (layer.Hk, layer.d)))
    dvr.unflatten(-1, (layer.H, layer.d)).copy_(dv.transpose(1, 2))
    drows, dconv_w, dconv_b = hla.hla_conv_backward(rows, layer.conv_w[:used], dconv, layer.conv_b[:used])
    return {"tokens": drows @ layer.w_in[:, :used].t(), "w_in": tokens.flatten(0, 1).t() @ drows.flatten(0, 1),
            "conv_w": dconv_w, "conv_b": dconv_b, "wq": dwq, "wk": dwk}


def main():
    torch.manual_seed(0)
    layer = Layer(256)
    B, n, more = 2, 300, 5
    tokens = torch.randn(B, n + more, 256, device="cuda").to(torch.bfloat16)
    whole, state = layer.new_state(B), layer.new_state(B)
    want = prompt(layer, tokens, whole)
    got = [prompt(layer, tokens[:, :n], state)] + [token(layer, tokens[:, n + i], state)[:, None] for i in range(more)]
    err = (torch.cat(got, 1).float() - want.float()).norm() / want.float().norm()
    print("a prompt of %d tokens and %d single tokens against %d at once: relative difference %.1e" % (n, more, n + more, err))
    grads = gradients(layer, tokens, torch.randn(B, layer.H, n + more, layer.d, device="cuda").to(torch.bfloat16))
    print("gradient norms: " + ", ".join("%s %.3g" % (k, float(v.float().norm())) for k, v in grads.items()))
    assert err < 2e-2 and all(torch.isfinite(v).all() for v in grads.values())


if __name__ == "__main__":
    main()
