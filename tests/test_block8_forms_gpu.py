"""The forms of the 8-bit products that sizes and arguments choose: the large tile with results that are streamed past the caches, with each activation to 8 bits; 8-bit results without
an activation and with an exponent for each row of B; the whole layer against its pieces.

Bounds as test_block8_gpu.py: bf16 results half a unit in the last place and 2^-14 of the sum of the magnitudes; 8-bit results a rounding to the format (2^-4 of a value, 2^-10 of the
block's power of two, which is at most a 224th of its largest) of what is off by 1.3 * 2^-14 of that sum (slopes of the activations: at most 1.13), fp32's by (K / 32 + 40) * 2^-24 of it."""
import math

import numpy as np
import pytest
import torch

from oracle import block8_oracle as B
from oracle import moe_oracle as O
from test_block8_gpu import UNIT, operand, values

pytestmark = pytest.mark.gpu

ACTS = {-1: lambda v: v, 0: torch.relu, 1: lambda v: v * torch.special.ndtr(v), 2: lambda v: v * torch.sigmoid(v)}
# experts, rows of a slab, K, N: large tiles; operands and results of more than 96 MB
STREAMED = (10, 1200, 2184, 2104)
TO_8BITS = [(24, 453, 1040, 776), (2, 300, 520, 392)]                # the large tile; the small one


@pytest.fixture(scope="module")
def moe():
    assert torch.cuda.is_available(), "these tests need a GPU"
    from paper_2206_03382_amd import moe as m
    m.lib()
    return m


def to_8bits(moe, A, B, bias, act, dtype, counts=None, gather=None):
    E, N = B.q.shape[:2]
    C = gather.shape[1] if gather is not None else A.q.shape[1]
    out = moe._alloc8((E,), C, N, False, "cuda")
    out.q.view(torch.uint8).fill_(0x11)
    out.s.fill_(99)
    p = lambda t: None if t is None else t.data_ptr()              # noqa: E731
    st = moe.lib().moe_matmul8(p(A.q), p(A.s), p(B.q), p(B.s), moe.SCALE_BLOCKS if B.blocks else moe.SCALE_ROWS, p(bias), act, moe.F32 if dtype == torch.float32 else moe.BF16, p(counts),
                               None, p(gather), A.q.shape[0] if gather is not None else 0, E, C, A.width, N, None, p(out.q), p(out.s), moe._stream())
    assert st == moe.OK
    return out


def assert_rows_in_8bits(m, e, n, ref, mags, lost):
    """Rows 0 .. n - 1 of expert e hold ref (float64, on the GPU), zeros past the width and 1 as the exponents past the blocks; the others are as they were."""
    N = m.width
    raw = m.q[e].view(torch.uint8)
    exps = m.s[e].to(torch.int64) - 127
    nb = -(-N // 128)
    assert (raw[n:] == 0x11).all() and (m.s[e, n:] == 99).all() and (raw[:n, N:] == 0).all() and (exps[:n, nb:] == 0).all()
    top = torch.zeros((n, nb * 128), dtype=torch.float64, device="cuda")
    top[:, :N] = ref.abs() + lost * mags
    amax = top.view(n, nb, 128).amax(-1)
    low = torch.zeros_like(top)
    low[:, :N] = (ref.abs() - lost * mags).clamp(min=0)
    low = low.view(n, nb, 128).amax(-1)
    two = torch.exp2(exps[:n, :nb].double())
    assert (low <= 448 * two).all() and ((exps[:n, :nb] == -126) | (amax > 224 * two)).all()
    table = torch.from_numpy(B.e4m3_table()).cuda()
    got = (table[raw[:n, :N].long()].view(n, N) * two.repeat_interleave(128, 1)[:, :N])
    bound = 2.0 ** -4 * ref.abs() + 1.07 * lost * mags + two.repeat_interleave(128, 1)[:, :N] * 2.0 ** -10
    assert ((got - ref).abs() <= bound).all()


def problem(moe, E, C, K, N, dtype, blocks, seed):
    rng = np.random.default_rng(seed)
    A, a = operand(moe, rng, E, C, K, False, spread=1)
    W, w = operand(moe, rng, E, N, K, blocks, spread=1)
    W = moe.Block8(W.q, (W.s.int() - 5).to(torch.uint8), K, blocks)          # near 1 / sqrt(K): activations where they curve
    W.s[..., -(-K // 128):] = 127
    w = w * 2.0 ** -5
    bias = torch.from_numpy((rng.standard_normal((E, N)) * 0.3).astype(np.float32)).to(dtype).cuda()
    fills = [int(n) for n in rng.integers(0, C + C // 4, E)]
    fills[0], fills[1] = C, 1
    return A, torch.from_numpy(a).cuda(), W, torch.from_numpy(w).cuda(), bias, fills


def reference(a, w, bias, act, e, n):
    up = a[e, :n] @ w[e].T + bias[e].double()
    return ACTS[act](up), a[e, :n].abs() @ w[e].abs().T + bias[e].double().abs()


@pytest.mark.parametrize("blocks", [True, False])
def test_streamed_results(moe, blocks):
    E, C, K, N = STREAMED
    A, a, W, w, bias, fills = problem(moe, E, C, K, N, torch.bfloat16, blocks, 1)
    counts = torch.tensor(fills, dtype=torch.int32, device="cuda")
    out = torch.full((E, C, N), 7.0, dtype=torch.bfloat16, device="cuda")
    moe.matmul8(A, W, bias=bias, counts=counts, out=out)
    for e, n in enumerate(fills):
        n = min(n, C)
        ref, mags = reference(a, w, bias, -1, e, n)
        assert (out[e, n:] == 7).all() and ((out[e, :n].double() - ref).abs() <= UNIT[torch.bfloat16] * ref.abs() + 2.0 ** -14 * mags).all()


@pytest.mark.parametrize("act", [0, 1, 2])
def test_streamed_results_in_8bits(moe, act):
    E, C, K, N = STREAMED
    A, a, W, w, bias, fills = problem(moe, E, C, K, N, torch.bfloat16, True, 2)
    out = to_8bits(moe, A, W, bias, act, torch.bfloat16, counts=torch.tensor(fills, dtype=torch.int32, device="cuda"))
    for e, n in enumerate(fills):
        n = min(n, C)
        assert_rows_in_8bits(out, e, n, *reference(a, w, bias, act, e, n), 1.2 * 2.0 ** -14)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("act", [-1, 0, 1, 2])
@pytest.mark.parametrize("blocks", [True, False])
@pytest.mark.parametrize("E,C,K,N", TO_8BITS)
def test_results_in_8bits(moe, E, C, K, N, blocks, act, dtype):
    A, a, W, w, bias, fills = problem(moe, E, C, K, N, dtype, blocks, 3 + act)
    out = to_8bits(moe, A, W, bias, act, dtype, counts=torch.tensor(fills, dtype=torch.int32, device="cuda"))
    lost = 1.2 * 2.0 ** -14 if dtype == torch.bfloat16 else 1.2 * (K / 32 + 40) * 2.0 ** -24 + (2.0 ** -18 if act > 0 else 0)       # the full activations' own roundings
    for e, n in enumerate(fills):
        n = min(n, C)
        assert_rows_in_8bits(out, e, n, *reference(a, w, bias, act, e, n), lost)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,M,H,E,k,f,act,normalize,bias", [(300, 256, 520, 8, 2, 1.25, 1, 1, True), (1000, 264, 384, 5, 1, 0.6, 2, 0, False), (777, 520, 776, 24, 4, 0.5, 0, 1, True),
                                                            (2600, 1032, 1544, 16, 2, 1.0, 2, 1, True), (65, 128, 136, 3, 3, 3.0, 0, 0, False)])
def test_layer_is_its_pieces(moe, T, M, H, E, k, f, act, normalize, bias, dtype):
    """moe_layer_forward8: routing as the oracle's on the normed tokens, a gate bias and dropped choices among them; the output bit for bit that of the experts' layer on the norm's
    8-bit tokens and the combine, both of which are checked by themselves."""
    g = torch.Generator(device="cuda").manual_seed(T)
    rnd = lambda *s, std=1.0: (torch.randn(s, generator=g, device="cuda") * std).to(dtype)      # noqa: E731
    W1, W2 = (moe.quantize8(rnd(E, a, b, std=1 / math.sqrt(a)), blocks=True, rows=False, transposed=True)[1] for a, b in ((M, H), (H, M)))
    Wg, w = rnd(M, E, std=1 / math.sqrt(M)), rnd(M)
    b1, b2 = (rnd(E, H, std=0.2), rnd(E, M, std=0.2)) if bias else (None, None)
    gate_bias = torch.randn(E, generator=g, device="cuda") if bias else None
    layer = moe.NormMoELayer8(w, 1e-6, Wg, gate_bias, W1, b1, W2, b2, T, k, f, normalize, act, keep_routing=True)
    layer.out.fill_(float("nan"))
    x, res = rnd(T, M), rnd(T, M)
    out, h = layer.forward(x, res)
    n = moe.rms_norm(x, w, 1e-6, residual=res, want_8=True)
    assert torch.equal(h, n["h"]) and torch.equal(layer.normed["y"], n["y"])
    r = layer.routing
    logits = O.gate_logits(n["y"].double().cpu().numpy(), Wg.double().cpu().numpy(), None if gate_bias is None else gate_bias.cpu().numpy())
    C = moe.capacity(T, E, k, f)
    want = O.route(logits, k, C, normalize)
    for key in ("idx", "loc", "counts"):
        assert np.array_equal(r[key].cpu().numpy(), want[key]), key
    if f < 1:
        assert (want["counts"] > C).any()
    slots = torch.from_numpy(O.slot_source(want["idx"], want["loc"], E, C).astype(np.int32)).cuda()
    Y = moe.expert_ffn8(n["y8"], W1, b1, W2, b2, act, dtype, counts=r["counts"], slot_src=slots)
    assert torch.equal(out, moe.decode(Y, r["idx"], r["loc"], r["gate_w"]))
    assert torch.isfinite(out).all()
