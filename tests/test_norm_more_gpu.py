"""RMS norm: results used again as `out`, and the backward's several rows to a slot.  Bounds as in test_norm_gpu.py: 36 fp32 roundings of y's size, a storage rounding."""
import numpy as np
import pytest
import torch

import test_norm_gpu as checks
from oracle import block8_oracle as B

pytestmark = pytest.mark.gpu

FP32 = 36 * 2.0 ** -24
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


@pytest.fixture(scope="module")
def moe():
    assert torch.cuda.is_available(), "these tests need a GPU"
    from paper_2206_03382_amd import moe as m
    m.lib()
    return m


def drawn(rng, shape, dtype, scale=1.0):
    t = torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).to(dtype)
    return t.cuda(), t.double().numpy()


def assert_within(got, ref, bound):
    off = np.abs(got.double().cpu().numpy() - ref)
    assert np.isfinite(off).all() and (off <= bound).all(), (off - bound).max()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_results_used_again(moe, dtype):
    """Calls with and without a residual in turn through one result: each gives its own h, y and 8 bits, and writes into nobody's input."""
    rng = np.random.default_rng(12)
    T, M = 70, 520
    w, w64 = drawn(rng, (M,), dtype, 0.5)
    out, inputs = None, []
    for i, with_residual in enumerate((False, False, True, False, True, True)):
        x, x64 = drawn(rng, (T, M), dtype)
        res, res64 = drawn(rng, (T, M), dtype) if with_residual else (None, None)
        inputs += [(x, x64)] + ([(res, res64)] if with_residual else [])
        out = moe.rms_norm(x, w, 1e-5, residual=res, want_8=True, out=out)
        h64, y64 = B.rms_norm(x64, res64, w64, 1e-5)
        assert_within(out["h"], h64, UNIT[dtype] * np.abs(h64))
        assert_within(out["y"], y64, (FP32 + UNIT[dtype]) * np.abs(y64))
        assert_within(moe.dequantize8(out["y8"], torch.float32), y64, 2.0 ** -4 * (1 + 2 * FP32) * np.abs(y64) + 2.0 ** -14 * np.abs(y64).max(1, keepdims=True))
        for t, v in inputs:
            assert np.array_equal(t.double().cpu().numpy(), v)


@pytest.mark.parametrize("T", [8, 100])
def test_norm_layer_without_a_residual(moe, T):
    """x alone is x with a residual of zeros, and h is x, whatever an earlier forward left."""
    dt, M, H, E = torch.bfloat16, 256, 384, 4
    g = torch.Generator(device="cuda").manual_seed(T)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda").to(dt)     # noqa: E731
    W1, W2 = (moe.quantize8(rnd(*s) / 16, blocks=True, rows=False, transposed=True)[1] for s in ((E, M, H), (E, H, M)))
    layer = moe.NormMoELayer8(rnd(M), 1e-6, rnd(M, E) / 16, None, W1, None, W2, None, T, 2, 2.0, 1, moe.ACT_SILU)
    for _ in range(2):
        x = rnd(T, M)
        want, h = layer.forward(x, torch.zeros_like(x))
        want = want.clone()
        assert torch.equal(h, x) and h is not x
        layer.forward(rnd(T, M), rnd(T, M))
        got, h = layer.forward(x, None)
        assert h is x and torch.equal(got, want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_smallest_eps(moe, dtype):
    """eps down to fp32's subnormals, where r^2 alone is no fp32 number: rows of zeros and of values near sqrt(eps)."""
    rng = np.random.default_rng(2)
    for eps in (1e-37, 1e-40):
        h, h64 = drawn(rng, (6, 264), dtype, 1e-19)
        h[:3] = 0
        h64[:3] = 0
        dy, dy64 = drawn(rng, (6, 264), dtype, 1e-3)
        got = moe.rms_norm_backward(dy, h, None, eps)
        eps64 = float(np.float32(eps))
        dx64, dw64 = B.rms_norm_backward(dy64, None, h64, None, eps64)
        r = 1.0 / np.sqrt(np.mean(h64 * h64, axis=1, keepdims=True) + eps64)
        parts = r * np.abs(dy64) + np.abs(h64) * r ** 3 * np.sum(np.abs(dy64 * h64), axis=1, keepdims=True) / 264
        assert_within(got["dx"], dx64, (2.0 ** -7 + UNIT[dtype]) * parts)          # squares of 1e-19 have few bits in fp32
        y = moe.rms_norm(h, None, eps)["y"]
        assert_within(y, h64 * r, 2.0 ** -8 * np.abs(h64 * r) + UNIT[dtype] * np.abs(h64 * r))


@pytest.mark.parametrize("T,M,dtype", [(600, 8200, torch.bfloat16), (600, 6144, torch.float32), (700, 16384, torch.float32), (521, 16384, torch.bfloat16)])
def test_backward_of_wide_rows(moe, T, M, dtype):
    """1024 lanes to a row, several rows to a slot."""
    checks.test_rms_norm_backward(moe, T, M, dtype)
