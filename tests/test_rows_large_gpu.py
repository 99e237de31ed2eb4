"""Products of experts' rows at the sizes whose rules name the 256 x 256 tile and the streamed ones, and offsets past 32 bits, against the formulas in 64 bits (torch, on the GPU).

Tolerances as in test_rows_gpu.py.  The experts' rows end everywhere in a tile of 256 and in its halves' sub-tiles of 32; which kernel a case takes is pinned by test_rows_rules.py.
"""
import math
from typing import NamedTuple

import numpy as np
import pytest
import torch

from test_rows_gpu import ACT, BF, F32, HALF, a_step, moe, sum_error   # noqa: F401

pytestmark = pytest.mark.gpu


class Case(NamedTuple):
    kernel: str
    R: int
    E: int
    K: int
    N: int
    act: str
    tokens: int = 0                                                 # of the matrix that rows are gathered from; 0: rows in place


LARGE = "256x256"
FORWARD = [Case(LARGE, 14000, 14, 832, 1792, "gelu", 4000), Case(LARGE, 14000, 14, 832, 1792, "gelu"), Case(LARGE, 7001, 3, 832, 1792, "silu", 5000), Case(LARGE, 6999, 4, 1024, 2048, "silu"),
           Case(LARGE, 6001, 5, 1024, 1536, "relu", 300), Case(LARGE, 8000, 12, 1088, 1536, "relu"), Case(LARGE, 7000, 3, 832, 1792, "none", 9000), Case(LARGE, 14000, 14, 832, 1792, "none"),
           Case("64x64 streamed", 64, 8, 2048, 2048, "silu"), Case("64x64 streamed", 90, 8, 2056, 2040, "gelu", 40), Case("64x64 streamed", 200, 8, 2048, 2056, "none"),
           Case("64x128 streamed", 128, 128, 1024, 1024, "relu"), Case("64x128 streamed", 1000, 128, 1032, 1032, "gelu", 300), Case("64x128 streamed", 300, 40, 1024, 1032, "none", 500)]
DENSE = [Case(LARGE, 8192, 1, 1024, 2048, "gelu"), Case(LARGE, 8229, 1, 832, 1792, "silu"), Case(LARGE, 4100, 1, 1024, 2048, "relu"), Case(LARGE, 8001, 1, 2048, 1536, "none")]
# K x N weights: gradients of N columns back to K; act is that of the projection before
BACK = [Case(LARGE, 14000, 14, 1792, 832, "gelu"), Case(LARGE, 12000, 4, 1024, 1536, "silu"), Case(LARGE, 7001, 3, 1792, 832, "relu"), Case(LARGE, 14000, 14, 1792, 832, "none"),
        Case("64x64 streamed", 64, 8, 2048, 2048, "gelu"), Case("64x64 streamed", 90, 8, 2056, 2048, "none"), Case("64x128 streamed", 128, 128, 1024, 1024, "silu"),
        Case("64x128 streamed", 300, 40, 1032, 1024, "relu")]
WEIGHTS = [Case(LARGE, 32768, 8, 2048, 2048, "none", 9000), Case(LARGE, 9003, 16, 1024, 1024, "none"), Case(LARGE, 9003, 16, 1024, 1024, "none", 5000), Case(LARGE, 6000, 3, 2048, 2304, "none")]

ENDS = [0, 1, 31, 33, 64, 65, 97, 128, 129, 161, 193, 225, 255, 63]


def fills_of(c):
    """Rows of the experts: ends of every kind, the rest in whole tiles to two of them; what then is left to the last one."""
    few = c.R <= 48 * c.E
    f = np.array([(e * 5 + 1) % 4 * (c.R // c.E) // 2 if few else ENDS[e % len(ENDS)] for e in range(c.E)])
    while f.sum() > c.R:
        f[int(f.argmax())] //= 2
    for e in (c.E // 2, c.E // 3):
        f[e] += 0 if few else (c.R - f.sum()) // 512 * 256
    f[-1] += c.R - f.sum()
    assert f.sum() == c.R and f.min() >= 0
    return f


def inputs(c, seed, behind=5):
    """offsets, A, W, gather with rows of memory behind the last expert's; and the rows of A in 64 bits."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s, scale=1.0: (torch.randn(s, device="cuda", generator=g) * scale).to(BF)   # noqa: E731
    offsets = [0, *np.cumsum(fills_of(c)).tolist()]
    A = normal(c.tokens or c.R + behind, c.K)
    gather = torch.randint(0, c.tokens, (c.R + behind,), device="cuda", generator=g, dtype=torch.int32) if c.tokens else None
    rows = (A if gather is None else A[gather.long()])[:c.R].double()
    if gather is None:
        A[c.R:] = float("nan")
    else:
        gather[c.R:] = -1
    return normal, offsets, torch.tensor(offsets, dtype=torch.int32, device="cuda"), A, rows, gather, normal(c.E, c.K, c.N, scale=1.0 / math.sqrt(c.K))


def activation(v, act):
    if act == "relu":
        return v.clamp(min=0.0), (v > 0).double()
    if act == "gelu":
        cdf = 0.5 * torch.special.erfc(-v / math.sqrt(2.0))
        return v * cdf, cdf + v * torch.exp(-0.5 * v * v) / math.sqrt(2.0 * math.pi)
    if act == "silu":
        s = torch.sigmoid(v)
        return v * s, s * (1.0 + v * (1.0 - s))
    return v, torch.ones_like(v)


def act_error(act, v, y):
    return 0.0 * y.abs() if act in ("none", "relu") else y.abs() * (5e-5 + v.abs() * 2.0 ** -22)


def products(rows, W, offsets, bias=None):
    """rows through their expert's weights, and the sums of the magnitudes."""
    v, S = rows.new_empty(rows.shape[0], W.shape[2]), rows.new_empty(rows.shape[0], W.shape[2])
    for e in range(W.shape[0]):
        at, w = slice(offsets[e], offsets[e + 1]), W[e].double()
        v[at], S[at] = rows[at] @ w, rows[at].abs() @ w.abs()
        if bias is not None:
            v[at] += bias[e].double()
            S[at] += bias[e].double().abs()
    return v, S


def assert_within(got, ref, bound, what):
    assert got.shape == ref.shape and torch.isfinite(got).all(), what
    over = (got.double() - ref).abs() - bound
    assert over.max() <= 0, f"{what}: {over.max().item():.3e} beyond the bound in {(over > 0).sum().item()} of {over.numel()}, first at {(over > 0).nonzero()[0].tolist()}"


@pytest.mark.parametrize("c", FORWARD, ids=str)
def test_forward(moe, c):   # noqa: F811
    normal, offsets, off, A, rows, gather, W = inputs(c, 1)
    b = normal(c.E, c.N, scale=0.3)
    out = torch.full((c.R + 5, c.N), 77.0, dtype=BF, device="cuda")
    got, pre = moe.ragged_matmul(A, W, off, b, ACT[c.act], gather=gather, keep_pre=True, out=out)
    assert got is out and (out[c.R:] == 77.0).all()
    v, S = products(rows, W, offsets, b)
    y, _ = activation(v, c.act)
    e = sum_error(BF, c.K) * S
    if pre is not None:
        assert_within(pre[:c.R], v, e + HALF[BF] * v.abs(), "pre")
    assert_within(out[:c.R], y, 1.13 * e + act_error(c.act, v, y) + HALF[BF] * y.abs(), "out")
    for _ in range(2):
        assert torch.equal(moe.ragged_matmul(A, W, off, b, ACT[c.act], gather=gather)[:c.R], out[:c.R])      # without kept values


@pytest.mark.parametrize("c", DENSE, ids=str)
def test_dense(moe, c):   # noqa: F811
    normal, offsets, _, A, rows, _, W = inputs(c, 2, behind=0)
    b, res = normal(c.N, scale=0.3), normal(c.R, c.N, scale=2.0)
    v, S = products(rows, W, offsets, b[None])
    y, _ = activation(v, c.act)
    e = sum_error(BF, c.K) * S
    error = 1.13 * e + act_error(c.act, v, y)
    r = res.double()
    got, pre = moe.linear(A, W[0], b, ACT[c.act], residual=res, keep_pre=True)
    if pre is not None:
        assert_within(pre, v, e + HALF[BF] * v.abs(), "pre")
    assert_within(got, y + r, error + 2.0 ** -23 * r.abs() + HALF[BF] * (y + r).abs(), "out")
    assert torch.equal(moe.linear(A, W[0], b, ACT[c.act], residual=res), got)
    assert_within(moe.linear(A, W[0], b, ACT[c.act]), y, error + HALF[BF] * y.abs(), "without a residual")
    own = res.clone()                                               # onto the residual itself
    assert torch.equal(moe.linear(A, W[0], b, ACT[c.act], residual=own, out=own), got)
    v0, S0 = products(rows, W, offsets)
    assert_within(moe.linear(A, W[0], residual=res), v0 + r, sum_error(BF, c.K) * S0 + 2.0 ** -23 * r.abs() + HALF[BF] * (v0 + r).abs(), "without bias and activation")


@pytest.mark.parametrize("c", BACK, ids=str)
def test_gradient_of_rows(moe, c):   # noqa: F811
    normal, offsets, off, _, _, _, W = inputs(c, 3)
    dy, x, x_pre = normal(c.R + 5, c.N), normal(c.R + 5, c.K), normal(c.R + 5, c.K, scale=1.5)
    dy[c.R:], x_pre[c.R:] = float("nan"), float("nan")
    x_pre[0] = 0                                                    # ReLU'(0) = 0
    with_act = {} if c.act == "none" else dict(x_act=ACT[c.act], x_pre=x_pre)
    got = moe.ragged_matmul_backward(dy, x, W, off, want_dW=False, want_db=False, **with_act)["dx"]
    d, S = products(dy[:c.R].double(), W.transpose(1, 2), offsets)
    p = x_pre[:c.R].double()
    _, slope = activation(p, c.act)
    ref = d * slope
    e = sum_error(BF, c.N) * S
    off_slope = 0.0 if c.act in ("none", "relu") else 2e-5
    assert_within(got[:c.R], ref, 1.13 * e + (d.abs() + e) * off_slope + HALF[BF] * (1 + 2.0 ** -7) * ref.abs() + 2.0 ** -120, "dx")
    assert torch.equal(moe.ragged_matmul_backward(dy, x, W, off, want_dW=False, want_db=False, **with_act)["dx"][:c.R], got[:c.R])


@pytest.mark.parametrize("c", WEIGHTS, ids=str)
def test_gradient_of_weights(moe, c):   # noqa: F811
    normal, offsets, off, A, rows, gather, W = inputs(c, 4)
    dy = normal(c.R + 5, c.N)
    d = dy[:c.R].double()
    dy[c.R:] = float("nan")
    got = moe.ragged_matmul_backward(dy, A, W, off, gather=gather, want_dx=False, want_db=False)["dW"]
    for e in range(c.E):
        at = slice(offsets[e], offsets[e + 1])
        ref, S = rows[at].T @ d[at], rows[at].abs().T @ d[at].abs()
        assert_within(got[e], ref, sum_error(BF, offsets[e + 1] - offsets[e]) * S + HALF[BF] * ref.abs(), f"dW of expert {e}")
        if at.start == at.stop:
            assert (got[e] == 0).all()
    assert torch.equal(moe.ragged_matmul_backward(dy, A, W, off, gather=gather, want_dx=False, want_db=False)["dW"], got)


def test_captured_steps_on_the_large_tile(moe):   # noqa: F811
    """Forward and all gradients of a dense projection and of experts' rows, captured and replayed with eager work in between."""
    c = Case(LARGE, 6000, 3, 2048, 2304, "gelu", 9000)
    normal, _, off, A, _, gather, W = inputs(c, 5, behind=0)
    b, dy, res = normal(c.E, c.N), normal(c.R, c.N), normal(c.R, c.N)
    x = normal(c.R, c.K)

    def step():
        out, pre = moe.ragged_matmul(A, W, off, b, moe.ACT_GELU, gather=gather, keep_pre=True)
        g = moe.ragged_matmul_backward(dy, A, W, off, moe.ACT_GELU, pre, gather=gather)
        return [out, pre, *g.values(), *a_step(moe, x, W[0], b[0], res, dy, moe.ACT_SILU)]

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for i in range(3):
        A.mul_(1.125), x.mul_(0.875)
        off[1] += 37 * i
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, step())), f"replay {i}"


# ---- past 32 bits ------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF, F32])
def test_rows_gathered_from_more_than_4_gib(moe, dtype):   # noqa: F811
    """Rows from both ends of a token matrix beyond 4 GiB: the products' and weight gradients' bits are those of the rows copied."""
    K, R = 4096, 700
    tokens = ((1 << 32) // (K * (2 if dtype == BF else 4))) + 9
    g = torch.Generator(device="cuda").manual_seed(6)
    A = torch.empty((tokens, K), dtype=dtype, device="cuda")
    gather = torch.randint(0, 40, (R,), device="cuda", generator=g, dtype=torch.int32)
    gather[::2] += tokens - 40
    A[:40], A[tokens - 40:] = torch.randn((40, K), device="cuda", generator=g).to(dtype), torch.randn((40, K), device="cuda", generator=g).to(dtype)
    off = torch.tensor([0, 333, R], dtype=torch.int32, device="cuda")
    for N in (136, 1544):
        W, dy = torch.randn((2, K, N), device="cuda", generator=g).to(dtype), torch.randn((R, N), device="cuda", generator=g).to(dtype)
        copied = A[gather.long()].contiguous()
        assert torch.equal(moe.ragged_matmul(A, W, off, act=moe.ACT_SILU, gather=gather), moe.ragged_matmul(copied, W, off, act=moe.ACT_SILU))
        got, want = (moe.ragged_matmul_backward(dy, a, W, off, gather=n, want_dx=False)["dW"] for a, n in ((A, gather), (copied, None)))
        assert torch.equal(got, want)


def test_more_than_2_to_the_31_results(moe):   # noqa: F811
    """Rows of results, kept values and gradients whose elements' numbers pass 31 bits: the first and last rows against the formulas, all weight gradients."""
    R, K, N = (1 << 20) + 77, 64, 2056
    assert R * N > 1 << 31
    g = torch.Generator(device="cuda").manual_seed(7)
    normal = lambda *s, scale=1.0: torch.randn(s, dtype=BF, device="cuda", generator=g) * scale   # noqa: E731
    A, W, dy = normal(R, K), normal(2, K, N, scale=0.125), normal(R, N)
    half = R // 2 + 5
    off = torch.tensor([0, half, R], dtype=torch.int32, device="cuda")
    out, pre = moe.ragged_matmul(A, W, off, act=moe.ACT_RELU, keep_pre=True)
    got = moe.ragged_matmul_backward(dy, A, W, off, moe.ACT_RELU, pre)
    for at, e in ((slice(0, 300), 0), (slice(half - 3, half), 0), (slice(half, half + 3), 1), (slice(R - 300, R), 1)):
        v, S = products(A[at].double(), W[e][None], [0, at.stop - at.start])
        assert_within(pre[at], v, sum_error(BF, K) * S + HALF[BF] * v.abs(), "pre")
        assert torch.equal(out[at], pre[at].clamp(min=0))
        d = dy[at].double() * (pre[at] > 0)
        v, S = products(d, W[e].T[None], [0, at.stop - at.start])
        assert_within(got["dx"][at], v, sum_error(BF, N) * S + HALF[BF] * v.abs(), "dx")
    for e, at in ((0, slice(0, half)), (1, slice(half, R))):
        ref, S = A.new_zeros((K, N), dtype=torch.float64), A.new_zeros((K, N), dtype=torch.float64)
        db, Sb = A.new_zeros(N, dtype=torch.float64), A.new_zeros(N, dtype=torch.float64)
        for r in range(at.start, at.stop, 1 << 16):
            part = slice(r, min(r + (1 << 16), at.stop))
            d, a = dy[part].double() * (pre[part] > 0), A[part].double()
            ref += a.T @ d
            S += a.abs().T @ d.abs()
            db += d.sum(0)
            Sb += d.abs().sum(0)
        n = at.stop - at.start
        assert_within(got["dW"][e], ref, sum_error(BF, n) * S + HALF[BF] * ref.abs(), "dW")
        assert_within(got["db"][e], db, (n / 8 + 96) * 2.0 ** -24 * Sb + HALF[BF] * db.abs(), "db")


def test_combine_of_more_than_2_to_the_31_elements(moe):   # noqa: F811
    T, k, M = (1 << 18) + 3, 2, 4096
    assert T * k * M > 1 << 31
    g = torch.Generator(device="cuda").manual_seed(8)
    Y, d = torch.randn((T * k, M), dtype=BF, device="cuda", generator=g), torch.randn((T, M), dtype=BF, device="cuda", generator=g)
    row_of = (T * k - 1 - torch.arange(T * k, device="cuda", dtype=torch.int32)).reshape(T, k)
    w = torch.rand((T, k), device="cuda", generator=g)
    out = moe.ragged_combine(Y, row_of, w)
    dY, dw = moe.ragged_combine_backward(d, Y, row_of, w)
    for at in (slice(0, 50), slice(T - 50, T)):
        y, weight, dout = Y[row_of[at].long()].double(), w[at].double()[:, :, None], d[at].double()[:, None]
        ref = (y * weight).sum(1)
        assert_within(out[at], ref, (k + 3) * 2.0 ** -24 * (y * weight).abs().sum(1) + HALF[BF] * ref.abs(), "out")
        assert_within(dY[row_of[at].long()], weight * dout, (HALF[BF] + 3 * 2.0 ** -24) * (weight * dout).abs(), "dY")
        assert_within(dw[at], (dout * y).sum(2), (M / 64 + 24) * 2.0 ** -24 * (dout * y).abs().sum(2), "dgate_w")
