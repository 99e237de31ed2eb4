"""The layer of a few tokens against the oracle: routing bit for bit, outputs within bounds from the arithmetic.

Bounds, per output.  bf16: the hidden activations are rounded once (2^-8 of each, carried through |W2| and the gate weights), the output once (2^-8); fp32 sums, here and for
fp32 layers, 2^-20 of the sum of all magnitudes that enter (fewer than 16 roundings of 2^-24 of it: a lane's and a wave's partial sums are of random signs, and the
deepest chain of additions has 64 of them, of which half the worst case is taken).
"""
import math

import numpy as np
import pytest
import torch

from oracle import block8_oracle as B
from oracle import moe_oracle as O
from paper_2206_03382_amd import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def moe():
    assert torch.cuda.is_available(), "these tests need a GPU"
    from paper_2206_03382_amd import moe as m
    m.lib()
    return m


def stored_values(m):
    raw = m.q.view(torch.uint8).cpu().numpy()
    e = m.s.cpu().numpy().astype(np.int64) - 127
    e = np.repeat(np.repeat(e, 128, axis=-1)[..., :raw.shape[-1]], 128, axis=-2)[..., :raw.shape[-2], :]
    return np.ascontiguousarray((B.e4m3_table()[raw] * 2.0 ** e)[..., :m.width].transpose(0, 2, 1))


def magnitudes(x, r, W1, b1, W2, b2, act, C):
    """(sum of what the hidden roundings can move, sum of all magnitudes) of every output, in float64."""
    T, k = r["idx"].shape
    moved, total = np.zeros_like(x), np.zeros_like(x)
    for t in range(T):
        for j in range(k):
            e = r["idx"][t, j]
            if r["loc"][t, j] >= C:
                continue
            h = O.activation(x[t] @ W1[e] + (0 if b1 is None else b1[e]), act)
            up = np.abs(x[t]) @ np.abs(W1[e]) + (0 if b1 is None else np.abs(b1[e]))
            w = r["gate_w"][t, j]
            moved[t] += w * (np.abs(h) @ np.abs(W2[e]))
            total[t] += w * (1.2 * up @ np.abs(W2[e]) + (0 if b2 is None else np.abs(b2[e])))
    return moved, total


# T, M, H, E, k, f, act, normalize, bias
CASES = [(1, 8, 8, 1, 1, 1.0, 0, 0, False), (1, 256, 512, 4, 1, 1.0, 0, 0, True), (1, 264, 136, 9, 3, 2.0, 2, 1, False), (2, 512, 256, 8, 8, 8.0, 1, 1, True),
         (5, 256, 512, 4, 1, 0.5, 1, 0, True), (16, 520, 776, 8, 2, 2.0, 1, 1, False), (17, 256, 264, 40, 4, 10.0, 2, 1, True), (33, 128, 384, 2, 2, 1.0, 2, 1, False),
         (64, 384, 640, 3, 1, 3.0, 1, 0, True), (64, 136, 256, 64, 8, 1.0, 0, 1, False), (48, 1024, 512, 8, 2, 0.3, 1, 1, True), (9, 2048, 1024, 16, 2, 2.0, 1, 1, False),
         (64, 264, 128, 130, 2, 1.0, 1, 1, True), (3, 4096, 256, 5, 2, 2.0, 2, 0, False), (64, 256, 2056, 1, 1, 1.0, 2, 1, False),
         # many blocks: with as many units as experts and with fewer, of up to 16 tokens and of more; many experts
         (16, 264, 1096, 40, 4, 2.0, 1, 1, True), (64, 128, 520, 64, 2, 0.5, 2, 0, False), (12, 64, 1160, 70, 3, 4.0, 1, 1, False), (20, 64, 1160, 70, 3, 1.0, 0, 1, True),
         (2, 520, 128, 512, 3, 100.0, 1, 1, False), (1, 1032, 136, 512, 1, 1.0, 2, 0, True),
         # little enough for every block to work out the logits: odd tokens and experts, more pieces than waves
         (7, 136, 264, 7, 3, 1.0, 1, 1, True), (8, 16, 72, 64, 2, 2.0, 2, 0, False), (3, 256, 128, 9, 9, 9.0, 1, 1, False), (8, 128, 136, 8, 2, 0.4, 0, 1, True),
         # few blocks and long sums: parts of them to a block; the second with dropped choices, the third with one choice, the last ones in more parts
         (1, 1544, 1032, 4, 2, 2.0, 1, 1, True), (9, 1032, 520, 2, 2, 0.5, 2, 1, True), (3, 1096, 2056, 3, 1, 0.4, 1, 0, True), (1, 8200, 264, 8, 1, 1.0, 2, 0, False), (2, 4104, 4160, 1, 1, 1.0, 0, 0, True)]


@pytest.mark.parametrize("kind", ["bf16", "fp32", "8bit", "8bit_fp32"])
@pytest.mark.parametrize("T,M,H,E,k,f,act,normalize,bias", CASES)
def test_few_tokens(moe, T, M, H, E, k, f, act, normalize, bias, kind):
    dt = torch.float32 if "fp32" in kind else torch.bfloat16
    g = np.random.default_rng(T * M + H)

    def draw(*shape, std=1.0):
        t = torch.from_numpy((g.standard_normal(shape) * std).astype(np.float32)).to(dt)
        return t.cuda(), t.float().numpy()
    (x, xn), (Wg, Wgn) = draw(T, M), draw(M, E, std=1 / math.sqrt(M))
    (W1, W1n), (W2, W2n) = draw(E, M, H, std=1 / math.sqrt(M)), draw(E, H, M, std=1 / math.sqrt(H))
    (b1, b1n), (b2, b2n) = (draw(E, H, std=0.2), draw(E, M, std=0.2)) if bias else ((None, None), (None, None))
    if kind.startswith("8bit"):
        W1, W2 = (moe.quantize8(w, blocks=True, rows=False, transposed=True)[1] for w in (W1, W2))
        W1n, W2n = stored_values(W1), stored_values(W2)
    layer = moe.FewTokenLayer(Wg, None, W1, b1, W2, b2, T, k, f, normalize, act, keep_routing=True)
    layer.out.fill_(float("nan"))
    out = layer.forward(x)
    r = O.moe_layer(xn, Wgn, None, W1n, b1n, W2n, b2n, k, f, normalize, act)
    for key in ("idx", "loc", "counts"):
        assert np.array_equal(layer.routing[key].cpu().numpy(), r[key]), key
    f64 = [None if a is None else a.astype(np.float64) for a in (xn, W1n, b1n, W2n, b2n)]
    moved, total = magnitudes(f64[0], r, f64[1], f64[2], f64[3], f64[4], act, r["C"])
    bound = 2.0 ** -20 * total + (2.0 ** -8 * (1.01 * moved + np.abs(r["out"])) if dt == torch.bfloat16 else 2.0 ** -23 * np.abs(r["out"])) + 1e-6 * moved
    off = np.abs(out.double().cpu().numpy() - r["out"])
    assert (off <= bound).all(), (off - bound).max()
    assert torch.equal(layer.forward(x).clone(), out)              # the same in every run


def test_same_routing_and_dropped_tokens(moe):
    """A gate that sends every token to one expert with a small capacity: the dropped ones are exactly zero."""
    T, M, H, E = 40, 128, 256, 4
    x = torch.randn((T, M), device="cuda").bfloat16()
    x[:, 0] = 5.0
    Wg = torch.zeros((M, E), device="cuda").bfloat16()
    Wg[0, 2] = 4.0
    W1, W2 = torch.randn((E, M, H), device="cuda").bfloat16(), torch.randn((E, H, M), device="cuda").bfloat16()
    layer = moe.FewTokenLayer(Wg, None, W1, None, W2, None, T, 1, 1.0, 0, 0, keep_routing=True)
    out = layer.forward(x)
    full = moe.MoELayer(Wg, None, W1, None, W2, None, T=T, k=1, f=1.0, normalize=0, act=0, keep_routing=True)
    want = full.forward(x)
    assert (layer.routing["idx"] == 2).all() and torch.equal(layer.routing["loc"], full.routing["loc"])
    assert (out[10:] == 0).all() and (out[:10].abs().amax(1) > 0).all()
    off = (out.float() - want.float()).norm() / want.float().norm()
    assert off <= 2.0 ** -7


def test_gate_bias_and_nan_tokens(moe):
    """A token of NaNs costs itself, not the tokens that share its experts."""
    T, M, H, E = 12, 256, 512, 4
    g = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()     # noqa: E731
    x, Wg, W1, W2 = rnd(T, M), rnd(M, E) / 16, rnd(E, M, H) / 16, rnd(E, H, M) / 16
    bias = torch.tensor([0.0, 3.0, 0.0, -2.0], device="cuda")
    layer = moe.FewTokenLayer(Wg, bias, W1, None, W2, None, T, 2, 4.0, 1, 1, keep_routing=True)
    clean = layer.forward(x).clone()
    assert (layer.routing["idx"] == 1).any(1).float().mean() > 0.5
    y = x.clone()
    y[5] = float("nan")
    got = layer.forward(y)
    keep = torch.arange(T, device="cuda") != 5
    assert torch.equal(got[keep], clean[keep])


def test_refusals(moe):
    bf = dict(dtype=torch.bfloat16, device="cuda")
    Wg, W1, W2 = torch.zeros((64, 4), **bf), torch.zeros((4, 64, 128), **bf), torch.zeros((4, 128, 64), **bf)
    with pytest.raises(moe.MoEError):
        moe.FewTokenLayer(Wg, None, W1, None, W2, None, moe.FEW_MAX_TOKENS + 1, 1, 1.0, 0, 0)
    with pytest.raises(ValueError):
        moe.FewTokenLayer(Wg, None, W1, None, W2.float(), None, 4, 1, 1.0, 0, 0)
    with pytest.raises(ValueError):
        moe.FewTokenLayer(Wg, None, W1, None, W1, None, 4, 1, 1.0, 0, 0)
    with pytest.raises(ValueError):
        moe.FewTokenLayer(Wg, None, W1, None, W2, None, 4, 1, 1.0, 0, 0).forward(torch.zeros((5, 64), **bf))
    with pytest.raises(moe.MoEError):
        moe.FewTokenLayer(Wg, None, W1, None, W2, None, 4, 5, 1.0, 0, 0)       # k > E
