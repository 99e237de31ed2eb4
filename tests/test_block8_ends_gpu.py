"""The 8-bit format at the ends of its range: exponents from -126 to 120, fp32's subnormals to its largest value.  Codes and exponents are compared exactly with the oracle's; values
that bf16 or fp32 cannot hold come back rounded to nearest even, which for a block's largest above 248 * 2^120 is infinity."""
import numpy as np
import pytest
import torch

from oracle import block8_oracle as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def moe():
    assert torch.cuda.is_available(), "these tests need a GPU"
    from paper_2206_03382_amd import moe as m
    m.lib()
    return m


def values(m):
    raw, e = m.q.view(torch.uint8).cpu().numpy(), m.s.cpu().numpy().astype(np.int64) - 127
    return (B.e4m3_table()[raw] * 2.0 ** np.repeat(e, 128, axis=-1)[..., :raw.shape[-1]])[..., :m.width]


def rows_at_the_ends(dtype):
    """[.., 128]: a row for each power of two, with magnitudes that spread over twelve of them; then the line to infinity."""
    rng = np.random.default_rng(0)
    top = float(torch.finfo(dtype).max)
    v = [rng.uniform(1, 2, 128) * np.exp2(rng.uniform(-12, 0, 128) + p) * rng.choice([-1, 1], 128) for p in [*range(-149, -105), *range(100, 127)]]
    v += [np.full(128, s) for s in (top, -top, 247.9 * 2.0 ** 120, 248.0 * 2.0 ** 120, 249.0 * 2.0 ** 120)]
    x = torch.from_numpy(np.array(v).astype(np.float32)).to(dtype)
    assert torch.isfinite(x).all()
    return x


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_there_and_back(moe, dtype):
    x = rows_at_the_ends(dtype)
    ref, exps = B.quantize(x.double().numpy(), False)
    q, qt = moe.quantize8(x.cuda(), transposed=True)
    assert np.array_equal(q.s[:, :1].cpu().numpy().astype(np.int64) - 127, exps) and np.array_equal(values(q), ref)
    assert np.array_equal(values(qt), B.quantize(np.ascontiguousarray(x.double().numpy().T), False)[0])
    assert exps.min() == -126 and exps.max() == 120
    with np.errstate(over="ignore"):
        f32 = torch.from_numpy(ref.astype(np.float32))
    assert torch.isinf(f32[-5]).all() and torch.isfinite(f32[-3]).all() == (dtype == torch.float32)      # 247.9 is 248 in bf16
    assert torch.equal(moe.dequantize8(q, torch.float32).cpu(), f32) and torch.equal(moe.dequantize8(q).cpu(), f32.to(torch.bfloat16))
    held = (exps[:, 0] >= -124) & (np.abs(ref).max(1) < 2.0 ** 128)        # what bf16 holds without a rounding
    assert np.array_equal(moe.dequantize8(q).cpu().double().numpy()[held], ref[held])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_products(moe, dtype):
    """With powers of two on a diagonal, so that a result is one product: bf16 results of the stored values; fp32 results of the stored values rounded to bf16."""
    x = rows_at_the_ends(torch.float32)
    q, _ = moe.quantize8(x.cuda())
    ref = values(q)
    finite = np.abs(ref).max(1) < 2.0 ** 128
    ref, at = ref[finite], torch.from_numpy(finite).cuda()
    q = moe.Block8(q.q.view(torch.uint8)[at][None].view(torch.float8_e4m3fn), q.s[at][None], 128, False)
    used = torch.from_numpy(ref).to(torch.float32).to(torch.bfloat16).double().numpy() if dtype == torch.float32 else ref
    for p in (-8, 0, 40):
        eye, _ = moe.quantize8((torch.eye(128, device="cuda") * 2.0 ** p)[None])
        with np.errstate(over="ignore"):
            want = torch.from_numpy((used * 2.0 ** p).astype(np.float32)).to(dtype)
        assert torch.equal(moe.matmul8(q, eye, dtype=dtype)[0].cpu(), want), p


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("p", [-130, -127, -118, -100, 60, 100])
def test_few_tokens(moe, p, dtype):
    """8-bit weights of the layer for few tokens: rounded to bf16, whose subnormals are kept."""
    g = torch.Generator().manual_seed(p + 200)
    W = torch.randn((1, 128, 128), generator=g).abs().clamp(max=3) * 2.0 ** p
    W1, W2 = moe.quantize8(W.cuda(), blocks=True)[0], moe.quantize8(torch.eye(128, device="cuda")[None], blocks=True)[0]
    x = torch.zeros((4, 128))
    x[torch.arange(4), torch.arange(4)] = 2.0 ** (min(-p, 120) if p < 0 else -60)
    layer = moe.FewTokenLayer(torch.zeros((128, 1), dtype=dtype, device="cuda"), None, W1, None, W2, None, 4, 1, 4.0, 0, moe.ACT_RELU)
    want = x.double() @ moe.dequantize8(W1).cpu().double()[0].T
    assert torch.equal(layer.forward(x.to(dtype).cuda()).cpu(), want.to(dtype))
