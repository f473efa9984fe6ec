"""A block of a recurrent model, as a serving or training program would run it:

    norm -> one projection -> short convolution -> gated linear recurrence -> projection
         -> norm with gate, residual scale and dropout, residual sum, norm
         -> gated feed-forward -> projection -> norm with residual scale, residual sum

``prompt`` runs any number of prompts at once and leaves a constant-size state, ``token`` continues each by
one token, ``gradients`` is a training step.  Run it on a GB300:

    python examples/recurrent_block.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2510_27258_gb300 import hla  # noqa: E402

WIDTH = 4  # taps of the convolution


class Block:
    """Sizes and weights: D model channels, C recurrent ones, F inner ones of the feed-forward part."""

    def __init__(self, D, C, F, dtype=torch.bfloat16, device="cuda", seed=0, dropout=0.0):
        g = torch.Generator().manual_seed(seed)
        self.D, self.C, self.F, self.dropout = D, C, F, dropout
        self.parts = [C, C, C, D]  # of a projection row: x | r | g | gate

        def make(*shape, scale=1.0, kind=dtype):
            return (torch.randn(*shape, generator=g) * scale).to(device=device, dtype=kind)

        self.w_in, self.w_out = make(D, sum(self.parts), scale=D ** -0.5), make(C, D, scale=C ** -0.5)
        self.conv_w, self.conv_b = make(C, WIDTH, scale=WIDTH ** -0.5), make(C, scale=0.1)
        self.decay = 8 * torch.log(0.9 + 0.099 * torch.rand(C, generator=g)).to(device)
        self.w_ff, self.w_down = make(2, F, D, scale=D ** -0.5), make(F, D, scale=F ** -0.5)
        for name in ("w_first", "w_post", "w_pre", "w_last"):
            setattr(self, name, 1 + make(D, scale=0.1))
        self.scale, self.scale_last = 0.5 + make(D, scale=0.1), 0.5 + make(D, scale=0.1)

    def new_state(self, B):
        """Convolution rows and recurrent states before the first token."""
        dev, T = self.w_in.device, self.w_in.dtype
        return {"conv": torch.zeros(B, WIDTH - 1, self.C, dtype=T, device=dev), "glr": torch.zeros(B, self.C, device=dev)}


def first_norm(block, x):
    """The norm before the block (nothing is added to x)."""
    return hla.hla_block_norm_forward(x, torch.zeros_like(x), w_pre=block.w_first, post_norm=False)[1]


def after_mixer(block, x, y, gate, seed):
    return hla.hla_block_norm_forward(x, y, gate, w_post=block.w_post, scale=block.scale, w_pre=block.w_pre,
                                      dropout=block.dropout, seed=seed)


def after_ffn(block, x, y):
    return hla.hla_block_norm_forward(x, y, w_post=block.w_last, scale=block.scale_last, pre_norm=False)[0]


def prompt(block, x, state, seed=0):
    """[B, n, D] -> [B, n, D]; ``state`` is updated to after the last token."""
    conv, r, g, gate = (first_norm(block, x) @ block.w_in).split(block.parts, -1)
    conv = hla.hla_conv_forward(conv, block.conv_w, block.conv_b, state_in=state["conv"], state_out=state["conv"])
    mixed = hla.hla_glr_forward(conv, r, g, block.decay, state_in=state["glr"], state_out=state["glr"])
    x, h = after_mixer(block, x, mixed @ block.w_out, gate, seed)
    return after_ffn(block, x, hla.hla_ffn_forward(h, block.w_ff) @ block.w_down)


def token(block, x, state):
    """One token a sequence: [B, D] -> [B, D], the state updated in place (no dropout)."""
    conv, r, g, gate = (first_norm(block, x) @ block.w_in).split(block.parts, -1)
    conv = hla.hla_conv_step(conv, block.conv_w, state["conv"], block.conv_b)
    mixed = hla.hla_glr_step(conv, r, g, block.decay, state["glr"])
    x, h = after_mixer(block, x, mixed @ block.w_out, gate, 0)
    return after_ffn(block, x, hla.hla_ffn_forward(h, block.w_ff) @ block.w_down)


def gradients(block, x0, dout, seed=0):
    """Gradients of sum(dout * prompt(x0)) from an empty state: of the tokens and of every weight."""
    B, n, D = x0.shape
    flat = lambda t: t.flatten(0, 1)  # noqa: E731
    h0 = first_norm(block, x0)
    rows = h0 @ block.w_in
    cx, r, g, gate = rows.split(block.parts, -1)
    conv = hla.hla_conv_forward(cx, block.conv_w, block.conv_b)
    marks = torch.empty(B, hla.hla_glr_marks(n), block.C, device=x0.device)
    mixed = hla.hla_glr_forward(conv, r, g, block.decay, marks=marks)
    y1 = mixed @ block.w_out
    x1, h1 = after_mixer(block, x0, y1, gate, seed)
    inner = hla.hla_ffn_forward(h1, block.w_ff)
    y2 = inner @ block.w_down
    grads = {}
    dx1, dy2, _, grads["w_last"], grads["scale_last"], _ = hla.hla_block_norm_backward(
        x1, y2, None, dout, w_post=block.w_last, scale=block.scale_last, pre_norm=False)
    grads["w_down"] = flat(inner).t() @ flat(dy2)
    dh1, grads["w_ff"] = hla.hla_ffn_backward(h1, block.w_ff, dy2 @ block.w_down.t())
    drows = torch.empty_like(rows)  # the gradients of the row's parts are written side by side
    dcx, dr, dg, dgate = drows.split(block.parts, -1)
    dx0, dy1, _, grads["w_post"], grads["scale"], grads["w_pre"] = hla.hla_block_norm_backward(
        x0, y1, gate, dx1, dh1, dgate=dgate, w_post=block.w_post, scale=block.scale, w_pre=block.w_pre,
        dropout=block.dropout, seed=seed)
    grads["w_out"] = flat(mixed).t() @ flat(dy1)
    dconv, _, _, grads["decay"] = hla.hla_glr_backward(conv, r, g, block.decay, dy1 @ block.w_out.t(), marks, dr=dr, dg=dg)
    _, grads["conv_w"], grads["conv_b"] = hla.hla_conv_backward(cx, block.conv_w, dconv, block.conv_b, dcx)
    grads["w_in"] = flat(h0).t() @ flat(drows)
    dx, _, _, _, _, grads["w_first"] = hla.hla_block_norm_backward(
        x0, torch.zeros_like(x0), None, dx0, drows @ block.w_in.t(), w_pre=block.w_first, post_norm=False)
    grads["tokens"] = dx
    return grads


def main():
    torch.manual_seed(0)
    block = Block(256, 320, 704)
    B, n, more = 2, 300, 5
    x = torch.randn(B, n + more, 256, device="cuda").to(torch.bfloat16)
    want = prompt(block, x, block.new_state(B))
    state = block.new_state(B)
    got = [prompt(block, x[:, :n].contiguous(), state)] + [token(block, x[:, n + i], state)[:, None] for i in range(more)]
    err = (torch.cat(got, 1).float() - want.float()).norm() / want.float().norm()
    print("a prompt of %d tokens and %d single tokens against %d at once: relative difference %.1e" % (n, more, n + more, err))
    grads = gradients(block, x, torch.randn(B, n + more, 256, device="cuda").to(torch.bfloat16))
    print("gradient norms: " + ", ".join("%s %.3g" % (k, float(v.float().norm())) for k, v in sorted(grads.items())))
    assert err < 2e-2 and all(torch.isfinite(v).all() for v in grads.values())


if __name__ == "__main__":
    main()
