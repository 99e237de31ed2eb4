"""NaNs go through the activations: a NaN among an expert's inputs, weights or biases is in every output that its value enters, whatever the activation, and in no other."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

NAN = float("nan")


@pytest.fixture(scope="module")
def moe():
    assert torch.cuda.is_available(), "these tests need a GPU"
    from paper_2206_03382_amd import moe as m
    m.lib()
    return m


def drawn(g, *shape, std=1.0):
    return torch.randn(shape, generator=g, device="cuda") * std


def matmul8_to_8bits(moe, A, B, bias, act, code):
    E, C, N = A.q.shape[0], A.q.shape[1], B.q.shape[1]
    out = moe._alloc8((E,), C, N, False, "cuda")
    p = lambda t: None if t is None else t.data_ptr()              # noqa: E731
    st = moe.lib().moe_matmul8(p(A.q), p(A.s), p(B.q), p(B.s), moe.SCALE_BLOCKS if B.blocks else moe.SCALE_ROWS, p(bias), act, code, None, None, None, 0, E, C, A.width, N,
                               None, p(out.q), p(out.s), moe._stream())
    assert st == moe.OK
    return out


@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("E,C,K,N", [(2, 40, 264, 136), (24, 453, 1040, 776)])      # both tiles
def test_matmul8(moe, E, C, K, N, dtype, act):
    """A row of A with a NaN block: that row of the result, all of it.  A NaN in the bias: its column, and in 8 bits its blocks."""
    g = torch.Generator(device="cuda").manual_seed(C)
    a = drawn(g, E, C, K)
    a[1, 3, K - 1] = NAN
    A, _ = moe.quantize8(a)
    B, _ = moe.quantize8(drawn(g, E, N, K, std=1 / math.sqrt(K)), blocks=True)
    bias = drawn(g, E, N).to(dtype)
    bias[0, N - 1] = NAN
    want = torch.zeros((E, C, N), dtype=torch.bool, device="cuda")
    want[1, 3], want[0, :, N - 1] = True, True
    assert torch.equal(torch.isnan(moe.matmul8(A, B, bias=bias, act=act, dtype=dtype)), want)
    got = moe.dequantize8(matmul8_to_8bits(moe, A, B, bias, act, moe._dtype_code(bias)), torch.float32)
    want[0, :, (N - 1) // 128 * 128:] = True                       # a block of the format is NaN as a whole
    assert torch.equal(torch.isnan(got), want)


@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("E,C,M,H", [(2, 40, 264, 136), (24, 453, 1040, 776)])
def test_expert_ffn8(moe, E, C, M, H, act):
    g = torch.Generator(device="cuda").manual_seed(H)
    x = drawn(g, E, C, M)
    x[1, 3, 5] = NAN
    X, _ = moe.quantize8(x)
    W1, W2 = (moe.quantize8(drawn(g, E, *s, std=1 / math.sqrt(s[0])), blocks=True, rows=False, transposed=True)[1] for s in ((M, H), (H, M)))
    Y = moe.expert_ffn8(X, W1, None, W2, None, act)
    want = torch.zeros((E, C, M), dtype=torch.bool, device="cuda")
    want[1, 3] = True
    assert torch.equal(torch.isnan(Y), want)


# the logits in the first product; slices of them; parts of the sums; more than 16 tokens, planned
@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("kind", ["bf16", "fp32", "8bit", "8bit_fp32"])
@pytest.mark.parametrize("T,M,H,E,k", [(5, 256, 512, 4, 1), (1, 4104, 264, 8, 2), (2, 1544, 1032, 4, 2), (40, 264, 2056, 9, 2)])
def test_few_tokens(moe, T, M, H, E, k, kind, act):
    """A NaN in one expert's first bias: the tokens that have this expert, and no others."""
    dt = torch.float32 if "fp32" in kind else torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(T + H)
    x, Wg = drawn(g, T, M).to(dt), drawn(g, M, E, std=1 / math.sqrt(M)).to(dt)
    W1, W2 = drawn(g, E, M, H, std=1 / math.sqrt(M)).to(dt), drawn(g, E, H, M, std=1 / math.sqrt(H)).to(dt)
    if kind.startswith("8bit"):
        W1, W2 = (moe.quantize8(w, blocks=True, rows=False, transposed=True)[1] for w in (W1, W2))
    b1 = drawn(g, E, H).to(dt)
    first = moe.FewTokenLayer(Wg, None, W1, b1, W2, None, T, k, float(E), 1, act, keep_routing=True)
    clean = first.forward(x).clone()
    assert torch.isfinite(clean).all()
    e = int(first.routing["idx"][0, 0])
    b1[e, H - 1] = NAN
    got = first.forward(x)
    has = (first.routing["idx"] == e).any(1)
    assert torch.isnan(got[has]).all() and torch.equal(got[~has], clean[~has])


@pytest.mark.parametrize("kind", ["bf16", "fp32", "8bit", "8bit_fp32"])
@pytest.mark.parametrize("T,M,H,E", [(3, 264, 520, 4), (40, 136, 264, 3)])
def test_few_tokens_infinity(moe, T, M, H, E, kind):
    """An infinite activation (an infinite bias under ReLU): infinities of the signs of its weights, NaN where a weight is zero."""
    dt = torch.float32 if "fp32" in kind else torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(T + H)
    x, Wg = drawn(g, T, M).to(dt), drawn(g, M, E, std=1 / math.sqrt(M)).to(dt)
    W1, W2 = drawn(g, E, M, H, std=1 / math.sqrt(M)).to(dt), drawn(g, E, H, M, std=1 / math.sqrt(H)).to(dt)
    W2[:, 5, 7] = 0
    row = W2[:, 5].float()
    if kind.startswith("8bit"):
        W1, W2 = (moe.quantize8(w, blocks=True, rows=False, transposed=True)[1] for w in (W1, W2))
        row = moe.dequantize8(W2, torch.float32)[:, :, 5]
    b1 = torch.zeros((E, H), dtype=dt, device="cuda")
    b1[:, 5] = float("inf")
    layer = moe.FewTokenLayer(Wg, None, W1, b1, W2, None, T, 1, float(E), 0, moe.ACT_RELU, keep_routing=True)
    got = layer.forward(x).float()
    want = row[layer.routing["idx"][:, 0].long()] * float("inf")
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.isnan(got[:, 7]).all()
    assert torch.equal(got.nan_to_num(0.0, 1.0, -1.0), want.nan_to_num(0.0, 1.0, -1.0))
