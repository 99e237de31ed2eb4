"""The activations of products on experts' rows and of dense projections, and their derivatives, at every bf16 number of their range and at its ends, against the 64-bit reference.

One column of x through a row of ones makes the value before the activation exactly v; ones through the unit matrix make dx exactly the derivative, rounded once.

Tolerances, all of them relative to what they are beside, and one absolute step, the smallest normal number, since smaller results may become zero.  bf16: the fit of GeLU's tail 5e-5 of Phi(-|v|), 2e-4 beyond 13.2, where only the derivative has it; an
exponential's argument is rounded to 2^-23 of itself, which is v^2 / 2 or |v|, and at most 16 beside it; 2^-19 for the other operations.  fp32: 16 roundings, and of the exponentials' arguments v^2 and
2 |v| (erfc by way of its own argument, too).  Then half a step of the result.
"""
import numpy as np
import pytest
import torch
from scipy.special import log_ndtr

from oracle import rows_oracle as O
from test_rows_gpu import ACT, BF, F32, HALF, moe, up   # noqa: F401

pytestmark = pytest.mark.gpu

SMALLEST = 2.0 ** -126


def all_values(top, dtype):
    """Every bf16 number from 2^-24 up to `top`, both signs; as many more between them in fp32."""
    bits = np.arange(np.float32(2.0 ** -24).view(np.uint32) >> 16, (np.float32(top).view(np.uint32) >> 16) + 1, dtype=np.uint32) << 16
    v = bits.view(np.float32)
    if dtype == F32:
        v = np.concatenate([v, (bits | 0x5A5B).view(np.float32)])
    return np.concatenate([[np.float32(0.0)], v, -v])


def through(moe, v, act, dtype):   # noqa: F811
    """act(v) and act'(v) of the library."""
    x = torch.zeros((len(v), 8), dtype=dtype)
    x[:, 0] = torch.from_numpy(v).to(dtype)
    first = torch.zeros((8, 8), dtype=dtype)
    first[0] = 1
    x, first, eye = x.cuda(), first.cuda(), torch.eye(8, dtype=dtype, device="cuda")
    out, pre = moe.linear(x, first, act=ACT[act], keep_pre=True)
    assert torch.equal(pre, x[:, :1].expand(-1, 8))
    slope = moe.linear_backward(torch.ones_like(pre), x, eye, ACT[act], pre, want_dW=False, want_db=False)["dx"]
    assert torch.equal(out, out[:, :1].expand(-1, 8)) and torch.equal(slope, slope[:, :1].expand(-1, 8))
    return up(out[:, 0]), up(slope[:, 0])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("act,top", [("gelu", 13.5), ("silu", 100.0), ("relu", 4.0)])
def test_every_value(moe, act, top, dtype):   # noqa: F811
    v = all_values(top, dtype)
    out, slope = through(moe, v, act, dtype)
    v = v.astype(np.float64)
    ref, ref_slope = O.act(v, act)
    a = np.abs(v)
    if act == "relu":
        error = error_slope = 0.0 * a
    elif act == "gelu":
        tail, dens = np.exp(log_ndtr(-a)), a * np.exp(-0.5 * v * v) / np.sqrt(2.0 * np.pi)
        ref = np.maximum(v, 0.0) - a * tail                          # as exact as the tail is
        ref_slope = np.where(v < 0, tail - dens, 1.0 - tail + dens)
        if dtype == BF:
            t = 5e-5 + (v * v / 2 + 16) * 2.0 ** -23
            error, error_slope = a * tail * t + 2.0 ** -19 * np.abs(ref), tail * np.maximum(t, 2e-4 * (a > 13.2)) + dens * ((v * v / 2 + 16) * 2.0 ** -23 + 2.0 ** -19) + (v > 0) * 2.0 ** -22
        else:
            t = (16 + v * v + 2 * a) * 2.0 ** -24
            error, error_slope = np.abs(ref) * t, (tail + dens + (v > 0)) * t
    else:
        e = np.exp(-a)
        s = np.where(v < 0, e, 1.0) / (1.0 + e)
        ref, ref_slope = v * s, s * (1.0 + v * np.where(v < 0, 1.0, e) / (1.0 + e))
        t = (a + 16) * 2.0 ** -22 + 2.0 ** -19 if dtype == BF else (16 + 2 * a) * 2.0 ** -24
        error, error_slope = np.abs(ref) * t, s * (1.0 + a * np.where(v < 0, 1.0, e) / (1.0 + e)) * t
    for what, got, want, off in (("value", out, ref, error), ("derivative", slope, ref_slope, error_slope)):
        assert np.isfinite(got).all()
        over = np.abs(got - want) - (off + HALF[dtype] * (np.abs(want) + off) + SMALLEST)
        worst = int(over.argmax())
        assert over[worst] <= 0, f"{what} at {v[worst]}: {got[worst]} for {want[worst]}; {(over > 0).sum()} beyond the bound, from {v[over > 0].min()} to {v[over > 0].max()}"


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("act", ["gelu", "silu", "relu"])
def test_far_values(moe, act, dtype):   # noqa: F811
    """Where nothing is left of one of the two parts: zero and the value itself, derivatives zero and one."""
    v = np.array([110.0, 1e4, 1e30, 3e38], dtype=np.float32)
    v = torch.from_numpy(v).to(dtype).float().numpy()
    out, slope = through(moe, np.concatenate([v, -v]), act, dtype)
    assert (out == np.concatenate([v, 0 * v])).all() and (slope == [1] * 4 + [0] * 4).all()
    at = torch.zeros((2, 8), dtype=dtype, device="cuda")
    at[0, 0], at[1, 0] = float("inf"), float("nan")
    first = torch.ones((8, 8), dtype=dtype, device="cuda")
    got = moe.linear(at, first, act=ACT[act])
    assert (got[0] == float("inf")).all() and got[1].isnan().all()
