"""The 64-bit references of the block's operators against differences, and their random bits against the
published vectors of Philox4x32-10."""
import pytest
import torch

import block_ref as R

D = torch.float64


def gen(seed):
    return torch.Generator().manual_seed(seed)


def rand(g, *shape):
    return torch.randn(*shape, generator=g, dtype=D)


def along(f, v, d):
    """The difference of f along d."""
    e = 1e-6
    return (f(v + e * d) - f(v - e * d)) / (2 * e)


@pytest.mark.parametrize("key,ctr,want", [
    ((0, 0), (0, 0, 0), 0x6627e8d5), ((0xffffffff, 0xffffffff), (0xffffffff, 0xffffffff, 0xffffffff), 0x408f276d)])
def test_philox_vectors(key, ctr, want):
    """Known answers: all zeros, and (rows and columns would be too many here) all ones through the rounds themselves."""
    if ctr[0] == 0:
        got = R.words(1, 4, 0, 0)[0]
        assert [int(v) for v in got] == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
        return
    c, k = [0xffffffff] * 4, list(key)
    for _ in range(10):
        p, q = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(q >> 32) ^ c[1] ^ k[0], q & 0xffffffff, (p >> 32) ^ c[3] ^ k[1], p & 0xffffffff]
        k = [(k[0] + 0x9E3779B9) & 0xffffffff, (k[1] + 0xBB67AE85) & 0xffffffff]
    assert c[0] == want and c[1:] == [0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]


@pytest.mark.parametrize("name", ["x", "r", "g", "decay", "state"])
def test_glr_gradients(name):
    g = gen(3)
    B, n, C = 3, 7, 2
    v = {"x": rand(g, B, n, C), "r": rand(g, B, n, C), "g": rand(g, B, n, C), "decay": -0.1 - rand(g, C).abs(),
         "state": rand(g, B, C)}
    dy, dl, lens = rand(g, B, n, C), rand(g, B, C), torch.tensor([7, 0, 4])

    def loss(t):
        y, last, _, _ = R.glr(**{**v, name: t}, lengths=lens)
        return (y * dy).sum() + (last * dl).sum()
    got = R.glr_grad(v["x"], v["r"], v["g"], v["decay"], dy, v["state"], dl, lens)["d" + name][0]
    d = rand(g, *v[name].shape)
    assert abs(float((got * d).sum() - along(loss, v[name], d))) < 1e-7


@pytest.mark.parametrize("act", [R.LINEAR, R.SIGMOID, R.SILU])
@pytest.mark.parametrize("post,pre", [(True, True), (False, True), (True, False)])
@pytest.mark.parametrize("name", ["x", "y", "gate", "w_post", "scale", "w_pre"])
def test_norm_gradients(name, post, pre, act):
    g = gen(5)
    v = {"x": rand(g, 4, 6), "y": rand(g, 4, 6), "gate": rand(g, 4, 6), "w_post": rand(g, 6), "scale": rand(g, 6),
         "w_pre": rand(g, 6)}
    if name == "w_post" and not post or name == "w_pre" and not pre:
        return
    kw = dict(post=post, pre=pre, act=act, alpha=0.7, eps=1e-3, dropout=0.3, seed=11, offset=2 ** 33 + 1)
    dx, dh = rand(g, 4, 6), rand(g, 4, 6)

    def loss(t):
        out = R.norm(**{**v, name: t}, **kw)
        return (out["x_out"][0] * dx).sum() + ((out["h"][0] * dh).sum() if pre else 0)
    got = R.norm(**v, dx_out=dx, dh=dh, **kw)["d" + name][0]
    d = rand(g, *v[name].shape)
    assert abs(float((got * d).sum() - along(loss, v[name], d))) < 1e-7


@pytest.mark.parametrize("act", [R.LINEAR, R.SIGMOID, R.SILU])
@pytest.mark.parametrize("name", ["x", "w"])
def test_ffn_gradients(name, act):
    g = gen(7)
    v = {"x": rand(g, 4, 5), "w": rand(g, 2, 3, 5)}
    dout = rand(g, 4, 3)
    got = R.ffn(**v, dout=dout, act=act)["d" + name][0]
    d = rand(g, *v[name].shape)
    want = along(lambda t: (R.ffn(**{**v, name: t}, act=act)["out"][0] * dout).sum(), v[name], d)
    assert abs(float((got * d).sum() - want)) < 1e-7
