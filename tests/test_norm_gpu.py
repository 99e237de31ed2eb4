"""RMS norm, its 8-bit output and its gradient against the 64-bit reference.

Tolerances.  A row's sum of squares is up to 32 fp32 additions in a lane, six across a wave and four to sixteen across waves, of positive terms: 56 roundings of
2^-24, half of which reaches the root; the reciprocal root, the mean and the products add at most eight: 36 * 2^-24 of y's size, in all 2.2e-6.  bf16 outputs add half
a unit in the last place, 2^-8.  Gradients: the dot product's roundings count against the sum of its magnitudes.
"""
import numpy as np
import pytest
import torch

from oracle import block8_oracle as B
from paper_2206_03382_amd import synth

pytestmark = pytest.mark.gpu

FP32 = 36 * 2.0 ** -24
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


@pytest.fixture(scope="module")
def moe():
    assert torch.cuda.is_available(), "these tests need a GPU"
    from paper_2206_03382_amd import moe as m
    m.lib()
    return m


def draw(rng, shape, dtype, scale=1.0):
    a = (rng.standard_normal(shape) * scale).astype(np.float32)
    t = torch.from_numpy(a).to(dtype)
    return t.cuda(), t.double().numpy()


def assert_within(got, ref, bound, what):
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all(), f"{what}: non-finite values"
    over = np.abs(got - ref) - bound
    assert over.max() <= 0, f"{what}: {np.abs(got - ref).max():.3e} off, {over.max():.3e} beyond the bound"


SHAPES = [(1, 8), (1, 4096), (3, 264), (5, 128), (7, 776), (16, 2048), (33, 520), (64, 1024), (300, 1000), (2, 16384), (3, 8200), (2100, 256), (2053, 2040), (2049, 4096), (17, 6144), (2100, 776)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,M", SHAPES)
def test_rms_norm(moe, T, M, dtype):
    rng = np.random.default_rng(T * 7 + M)
    x, x64 = draw(rng, (T, M), dtype)
    res, res64 = draw(rng, (T, M), dtype, 2.0)
    w, w64 = draw(rng, (M,), dtype, 0.5)
    x[0] *= 0                                                      # a row of zeros without a residual
    x64[0] = 0
    eps = 1e-5
    for residual, r64, weight, wt64 in ((res, res64, w, w64), (None, None, w, w64), (res, res64, None, None)):
        h64, y64 = B.rms_norm(x64, r64, wt64, eps)
        got = moe.rms_norm(x, weight, eps, residual=residual, want_8=True)
        if residual is not None:
            assert_within(got["h"], h64, UNIT[dtype] * np.abs(h64), "h")
        size = np.abs(y64)
        assert_within(got["y"], y64, (FP32 + UNIT[dtype]) * size, "y")
        only = moe.rms_norm(x, weight, eps, residual=residual, want_y=False, want_8=True)["y8"]
        assert torch.equal(only.q.view(torch.uint8), got["y8"].q.view(torch.uint8)) and torch.equal(only.s, got["y8"].s)
        # 8 bits: half an e4m3 step (2^-4 of a value, 2^-10 of the block's power of two below its normal range) of the fp32 value; exponents as the
        # reference's, or its neighbour's where the block's largest value is within fp32's error of the line between them
        assert_format(got["y8"], y64, FP32)


def assert_format(m, ref, slack):
    T, M = ref.shape
    exps = m.s.cpu().numpy().astype(np.int64) - 127
    nb = -(-M // 128)
    assert (exps[:, nb:] == 0).all()
    raw = m.q.view(torch.uint8).cpu().numpy()
    assert (raw[:, M:] == 0).all()
    val = B.e4m3_table()[raw[:, :M]]
    e = np.repeat(exps[:, :nb], 128, axis=1)[:, :M]
    pad = np.zeros((T, nb * 128))
    pad[:, :M] = np.abs(ref)
    amax = pad.reshape(T, nb, 128).max(-1)
    assert (amax <= 448.0 * 2.0 ** exps[:, :nb] * (1 + slack)).all()
    assert ((exps[:, :nb] == -126) | (amax > 224.0 * 2.0 ** exps[:, :nb] * (1 - slack))).all()
    bound = np.abs(ref) * (2.0 ** -4 * (1 + slack) + slack) + 2.0 ** (e - 10.0)
    assert (np.abs(val * 2.0 ** e - ref) <= bound).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,M", SHAPES + [(1500, 512), (5000, 264), (16500, 776), (16400, 264)])
def test_rms_norm_backward(moe, T, M, dtype):
    rng = np.random.default_rng(T * 5 + M)
    h, h64 = draw(rng, (T, M), dtype, 1.5)
    dy, dy64 = draw(rng, (T, M), dtype)
    dh, dh64 = draw(rng, (T, M), dtype)
    w, w64 = draw(rng, (M,), dtype, 0.5)
    eps = 1e-5
    for d, d64, weight, wt64 in ((dh, dh64, w, w64), (None, None, w, w64), (dh, dh64, None, None)):
        dx64, dw64 = B.rms_norm_backward(dy64, d64, h64, wt64, eps)
        got = moe.rms_norm_backward(dy, h, weight, eps, dh=d)
        r = 1.0 / np.sqrt(np.mean(h64 * h64, axis=1, keepdims=True) + eps)
        g = np.abs(dy64 if wt64 is None else dy64 * wt64)
        parts = r * g + np.abs(h64) * r ** 3 * np.sum(g * np.abs(h64), axis=1, keepdims=True) / M + (0 if d64 is None else np.abs(d64))
        assert_within(got["dx"], dx64, 3 * FP32 * parts + UNIT[dtype] * np.abs(dx64), "dx")
        # a column's sum: up to T / 1024 rows in a lane, then the slots, 32 groups of them: fewer roundings than 40 + T / 1000 + 32
        terms = np.sum(np.abs(dy64 * h64 * r), axis=0)
        assert_within(got["dweight"], dw64, (FP32 + (72 + T / 1000.0) * 2.0 ** -24) * terms + UNIT[dtype] * np.abs(dw64), "dweight")
        again = moe.rms_norm_backward(dy, h, weight, eps, dh=d)
        assert torch.equal(again["dx"], got["dx"]) and torch.equal(again["dweight"], got["dweight"])


def test_rms_norm_gradient_against_differences(moe):
    """The loss <y, dy> + <h, dh> along random directions of x and weight, by central differences in 64 bits: their error is step^2 times a third derivative, 1e-10 here."""
    rng = np.random.default_rng(3)
    T, M, eps, step = 9, 328, 1e-5, 1e-5
    h, h64 = draw(rng, (T, M), torch.float32)
    dy, dy64 = draw(rng, (T, M), torch.float32)
    dh, dh64 = draw(rng, (T, M), torch.float32)
    w, w64 = draw(rng, (M,), torch.float32)
    got = moe.rms_norm_backward(dy, h, w, eps, dh=dh)
    dx, dw = got["dx"].double().cpu().numpy(), got["dweight"].double().cpu().numpy()

    def loss(x, weight):
        s, y = B.rms_norm(x, None, weight, eps)
        return np.sum(y * dy64) + np.sum(s * dh64)
    for _ in range(4):
        a, b = rng.standard_normal((T, M)), rng.standard_normal(M)
        along = (loss(h64 + step * a, w64 + step * b) - loss(h64 - step * a, w64 - step * b)) / (2 * step)
        size = np.sum(np.abs(dx * a)) + np.sum(np.abs(dw * b))
        assert abs(np.sum(dx * a) + np.sum(dw * b) - along) <= 6 * FP32 * size + 1e-7


def test_rms_norm_extreme_values(moe):
    """Rows near the ends of the storage types, infinities and NaNs: a block that holds one is NaN, its neighbours are not touched by another row's."""
    x = torch.ones((6, 256), device="cuda")
    x[0] *= 1e-30
    x[1] *= 1e18
    x[2, 5] = float("inf")
    x[3, 7] = float("nan")
    x[4] *= 0
    got = moe.rms_norm(x, None, 1e-12, want_8=True)
    y = moe.dequantize8(got["y8"], torch.float32)
    assert torch.allclose(got["y"][0], torch.full((256,), 1e-24, device="cuda"), rtol=1e-5)
    assert torch.allclose(got["y"][1], torch.ones(256, device="cuda"), rtol=1e-5)
    assert torch.isnan(got["y"][3]).all() and torch.isnan(y[3]).all() and (got["y8"].s[3, :2] == 255).all()
    assert torch.isnan(got["y"][2, 5]) and torch.isnan(y[2, :128]).all() and (y[2, 128:] == 0).all()
    assert (got["y"][4] == 0).all() and (y[4] == 0).all() and (got["y8"].s[4, :2] == 1).all()
    assert torch.allclose(y[5], torch.ones(256, device="cuda"), rtol=2.0 ** -4)


def test_rms_norm_in_place_on_a_stream_of_its_own(moe):
    rng = np.random.default_rng(8)
    x, x64 = draw(rng, (130, 776), torch.bfloat16)
    res, res64 = draw(rng, (130, 776), torch.bfloat16)
    h64, y64 = B.rms_norm(x64, res64, None, 1e-6)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        out = dict(h=res, y=torch.empty_like(x), y8=None)
        moe.rms_norm(x, None, 1e-6, residual=res, out=out)          # the sum replaces the residual
    torch.cuda.current_stream().wait_stream(s)
    assert_within(res, h64, UNIT[torch.bfloat16] * np.abs(h64), "h")
    assert_within(out["y"], y64, (FP32 + UNIT[torch.bfloat16]) * np.abs(y64), "y")


def test_rms_norm_refusals(moe):
    x = torch.zeros((4, 16), device="cuda")
    with pytest.raises(ValueError):
        moe.rms_norm(x.t(), None, 1e-6)
    with pytest.raises(ValueError):
        moe.rms_norm(x, torch.zeros(15, device="cuda"), 1e-6)
    with pytest.raises(ValueError):
        moe.rms_norm(x, None, 1e-6, residual=x.bfloat16())
    with pytest.raises(moe.MoEError):
        moe.rms_norm(x, None, 0.0)
    with pytest.raises(moe.MoEError):
        moe.rms_norm(x, None, 1e-6, want_y=False)
    with pytest.raises(TypeError):
        moe.rms_norm(x.half(), None, 1e-6)
