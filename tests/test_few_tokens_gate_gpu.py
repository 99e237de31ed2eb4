"""The gate of the few-token layer: logits with a bias, gate weights and routing against 64 bits, masked experts, gate weights at any address; and the layer at blocks of 32
columns that have a plan of their own.

Bounds.  Logits: exact products and fp64 sums, rounded once: 2^-24 of the logit, and 1e-13 of the sum of magnitudes for the fp64 roundings.  Gate weights, against the softmax in
64 bits of the library's own logits: two exponentials of two units in the last place, a sum of up to 14 roundings, a division and the subtraction from the largest logit:
32 * 2^-24, and 2 * 2^-24 of that difference.  Outputs: as test_few_tokens_gpu.py."""
import math

import numpy as np
import pytest
import torch

from oracle import moe_oracle as O
from test_few_tokens_gpu import magnitudes, stored_values

pytestmark = pytest.mark.gpu

INF = float("inf")


@pytest.fixture(scope="module")
def moe():
    assert torch.cuda.is_available(), "these tests need a GPU"
    from paper_2206_03382_amd import moe as m
    m.lib()
    return m


def layer_inputs(moe, T, M, H, E, kind, seed):
    dt = torch.float32 if "fp32" in kind else torch.bfloat16
    g = np.random.default_rng(seed)

    def draw(*shape, std=1.0):
        t = torch.from_numpy((g.standard_normal(shape) * std).astype(np.float32)).to(dt)
        return t.cuda(), t.float().numpy()
    x, Wg = draw(T, M), draw(M, E, std=1 / math.sqrt(M))
    W1, W2 = draw(E, M, H, std=1 / math.sqrt(M)), draw(E, H, M, std=1 / math.sqrt(H))
    if kind.startswith("8bit"):
        q = [moe.quantize8(w[0], blocks=True, rows=False, transposed=True)[1] for w in (W1, W2)]
        W1, W2 = ((m, stored_values(m)) for m in q)
    return x, Wg, W1, W2, g


def assert_gate(routing, x, Wg, bias, k, normalize):
    """Logits by themselves, then choices, arrivals and weights from the library's logits."""
    logits = routing["logits"].cpu().numpy()
    ref = x.astype(np.float64) @ Wg.astype(np.float64) + bias.astype(np.float64)
    mags = np.abs(x.astype(np.float64)) @ np.abs(Wg.astype(np.float64)) + np.abs(bias)
    live = np.isfinite(ref)
    assert np.array_equal(np.isfinite(logits), live) and (logits[~live] == ref[~live]).all()
    assert (np.abs(logits - ref)[live] <= (2.0 ** -24 * np.abs(ref) + 1e-13 * mags)[live]).all()
    r = O.route(np.maximum(logits, np.finfo(np.float32).min), k, 1 << 20, normalize)        # the oracle's are finite; of either kind the order and the weight, 0, are the same
    for key in ("idx", "loc", "counts"):
        assert np.array_equal(routing[key].cpu().numpy(), r[key]), key
    chosen = np.take_along_axis(logits.astype(np.float64), r["idx"].astype(np.int64), 1)
    apart = np.where(chosen > -1e30, logits.max(1, keepdims=True) - chosen, 0.0)
    got = routing["gate_w"].double().cpu().numpy()
    assert (np.abs(got - r["gate_w"]) <= (32 + 2 * apart) * 2.0 ** -24 * r["gate_w"] + 1e-38).all()
    return r


# in the first product; one slice; two; four; more than 16 tokens; planned; more experts than lanes; as many choices as experts
GATES = [(5, 256, 512, 4, 1, 0), (3, 136, 264, 9, 3, 1), (8, 16, 72, 64, 2, 0), (12, 1024, 136, 8, 2, 1), (1, 2056, 136, 16, 4, 1), (9, 3080, 64, 24, 2, 0), (16, 4104, 72, 8, 2, 1),
         (2, 8200, 64, 130, 8, 1), (33, 264, 136, 12, 2, 1), (64, 1032, 72, 200, 4, 0), (40, 264, 2056, 9, 2, 1), (1, 520, 128, 512, 3, 1), (7, 264, 128, 5, 5, 1)]


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("T,M,H,E,k,normalize", GATES)
def test_gate_with_bias(moe, T, M, H, E, k, normalize, kind):
    (x, xn), (Wg, Wgn), (W1, W1n), (W2, W2n), g = layer_inputs(moe, T, M, H, E, kind, T + M)
    bias = (g.standard_normal(E) * 2).astype(np.float32)
    layer = moe.FewTokenLayer(Wg, torch.from_numpy(bias).cuda(), W1, None, W2, None, T, k, float(E), normalize, 1, keep_routing=True)
    for t in layer.routing.values():
        t.fill_(77)
    layer.forward(x)
    assert_gate(layer.routing, xn, Wgn, bias, k, normalize)
    bare = moe.FewTokenLayer(Wg, None, W1, None, W2, None, T, k, float(E), normalize, 1, keep_routing=True)
    bare.forward(x)
    assert_gate(bare.routing, xn, Wgn, np.zeros(E, dtype=np.float32), k, normalize)


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("T,M,H,E,k,normalize", [g for g in GATES if g[3] > 2 * g[4]])
def test_masked_experts(moe, T, M, H, E, k, normalize, kind):
    """Biases of minus infinity and of fp32's lowest value keep experts out, whichever way the logits are worked out; equal ones go to the lowest index."""
    (x, xn), (Wg, Wgn), (W1, _), (W2, _), g = layer_inputs(moe, T, M, H, E, kind, T + M + 1)
    for low in (-INF, float(np.finfo(np.float32).min)):
        for open_ in (k + 1, 1):                                   # the second: fewer live experts than choices where k > 1
            bias = np.full(E, low, dtype=np.float32)
            bias[g.permutation(E)[:open_]] = 0.5
            layer = moe.FewTokenLayer(Wg, torch.from_numpy(bias).cuda(), W1, None, W2, None, T, k, float(E), normalize, 1, keep_routing=True)
            out = layer.forward(x)
            assert_gate(layer.routing, xn, Wgn, bias, k, normalize)
            assert torch.isfinite(out).all()


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("T,M,H,E,k,normalize", [(5, 256, 512, 4, 1, 0), (8, 16, 72, 64, 2, 0), (12, 1024, 136, 8, 2, 1), (16, 4104, 72, 10, 2, 1), (40, 264, 136, 9, 2, 1)])
def test_gate_weights_at_any_address(moe, T, M, H, E, k, normalize, kind):
    """Wg one element behind an aligned address: the same numbers."""
    (x, _), (Wg, _), (W1, _), (W2, _), _ = layer_inputs(moe, T, M, H, E, kind, 5)
    behind = torch.empty(M * E + 1, dtype=Wg.dtype, device="cuda")[1:].view(M, E).copy_(Wg)
    assert behind.data_ptr() % 16 == Wg.element_size()
    a, b = (moe.FewTokenLayer(w, None, W1, None, W2, None, T, k, 2.0, normalize, 1, keep_routing=True) for w in (Wg, behind))
    assert torch.equal(a.forward(x), b.forward(x))
    for key in a.routing:
        assert torch.equal(a.routing[key], b.routing[key])


@pytest.mark.parametrize("kind", ["fp32", "8bit", "8bit_fp32"])
@pytest.mark.parametrize("T,M,H,E,k", [(1, 264, 2560, 16, 8), (4, 136, 648, 64, 8), (16, 520, 640, 32, 2), (24, 264, 384, 32, 2), (64, 136, 648, 16, 2)])
def test_narrow_blocks_with_a_plan(moe, T, M, H, E, k, kind):
    (x, xn), (Wg, Wgn), (W1, W1n), (W2, W2n), g = layer_inputs(moe, T, M, H, E, kind, H)
    bias = g.standard_normal(E).astype(np.float32)
    layer = moe.FewTokenLayer(Wg, torch.from_numpy(bias).cuda(), W1, None, W2, None, T, k, 0.8, 1, 2, keep_routing=True)
    layer.out.fill_(float("nan"))
    out = layer.forward(x).double().cpu().numpy()
    r = O.moe_layer(xn, Wgn, bias, W1n, None, W2n, None, k, 0.8, 1, 2)
    for key in ("idx", "loc", "counts"):
        assert np.array_equal(layer.routing[key].cpu().numpy(), r[key]), key
    f64 = [a.astype(np.float64) for a in (xn, W1n, W2n)]
    moved, total = magnitudes(f64[0], r, f64[1], None, f64[2], None, 2, r["C"])
    bound = 2.0 ** -20 * total + (2.0 ** -8 * (1.01 * moved + np.abs(r["out"])) if x.dtype == torch.bfloat16 else 2.0 ** -23 * np.abs(r["out"])) + 1e-6 * moved
    assert (np.abs(out - r["out"]) <= bound).all()
