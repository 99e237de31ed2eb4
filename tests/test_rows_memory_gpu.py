"""What workspaces and results hold before a call makes no difference, and experts without any rows at all: products of experts' rows and dense projections on each of their kernels."""
import numpy as np
import pytest
import torch

from test_rows_gpu import ACT, BF, F32, a_step, draw, fills_of, moe   # noqa: F401

pytestmark = pytest.mark.gpu

# rows, experts, K, N
SIZES = [(3, 2, 64, 64), (16, 8, 1024, 512), (700, 9, 1000, 776), (5000, 140, 64, 512), (9001, 5, 136, 128), (6000, 3, 2048, 2304), (128, 128, 1024, 1024), (32768, 2, 512, 512)]
DENSE = [(1, 4096, 4096), (50, 4096, 2056), (300, 776, 264), (20001, 264, 256), (8192, 1024, 2048)]


def poison(nbytes):
    """Memory that the allocator will hand out again holds NaNs, in bf16 as in fp32."""
    blocks = [torch.full((n // 4,), float("nan"), device="cuda") for n in (nbytes, nbytes // 4, nbytes // 16, 1 << 20, 1 << 16, 1 << 12, 512) for _ in range(4)]
    blocks = [b.view(torch.int32).fill_(-1) for b in blocks]
    torch.cuda.synchronize()
    del blocks


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("R,E,K,N", SIZES)
def test_rows(moe, R, E, K, N, dtype):   # noqa: F811
    rng = np.random.default_rng(R)
    A, W, b, dy = (draw(rng, s, dtype)[0] for s in ((R, K), (E, K, N), (E, N), (R, N)))
    gather = torch.from_numpy(rng.integers(0, R, R).astype(np.int32)).cuda()
    off = torch.from_numpy(np.concatenate([[0], np.cumsum(fills_of("skewed", E, R, rng))]).astype(np.int32)).cuda()

    def step(offsets, act=moe.ACT_SILU):
        out, pre = moe.ragged_matmul(A, W, offsets, b, act, gather=gather, keep_pre=True)
        g = moe.ragged_matmul_backward(dy, A, W, offsets, act, pre, gather=gather)
        h = moe.ragged_matmul_backward(dy, A, W, offsets, x_act=act, x_pre=A)
        return out, pre, g, h

    first = step(off)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    poison(max(R * max(K, N), E * K * N) * 4)
    second = step(off)
    for x, y in zip(first[:2] + tuple(first[2].values()) + tuple(first[3].values()), second[:2] + tuple(second[2].values()) + tuple(second[3].values())):
        assert torch.equal(x, y) and torch.isfinite(x).all()

    for at in (0, R):                                               # nobody has rows: in front of them all, and behind
        none = torch.full((E + 1,), at, dtype=torch.int32, device="cuda")
        out = torch.full((R, N), 77.0, dtype=dtype, device="cuda")
        assert (moe.ragged_matmul(A, W, none, b, moe.ACT_SILU, gather=gather, out=out) == 77.0).all()
        for kept in (dict(gather=gather), dict()):
            g = moe.ragged_matmul_backward(dy, A, W, none, moe.ACT_SILU, first[1], **kept)
            assert (g["dW"] == 0).all() and (g["db"] == 0).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,K,N", DENSE)
def test_dense(moe, T, K, N, dtype):   # noqa: F811
    rng = np.random.default_rng(T)
    x, W, b, res, dy = (draw(rng, s, dtype)[0] for s in ((T, K), (K, N), (N,), (T, N), (T, N)))
    first = a_step(moe, x, W, b, res, dy, moe.ACT_GELU)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    poison(max(T * max(K, N), K * N) * 4)
    for x_, y in zip(first, a_step(moe, x, W, b, res, dy, moe.ACT_GELU)):
        assert torch.equal(x_, y) and torch.isfinite(x_).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("R,E,K,N", SIZES + [(9003, 16, 1024, 1024), (14000, 14, 832, 1792)])
def test_nan_stays_with_its_expert(moe, R, E, K, N, dtype):   # noqa: F811
    """One expert's rows of x, dy and kept values hold NaNs, and so do its weights: the other experts' results and gradients have the bits that they have without, wherever tiles end."""
    rng = np.random.default_rng(R + 1)
    fills = fills_of("skewed", E, R, rng)
    offsets = np.concatenate([[0], np.cumsum(fills)])
    off = torch.from_numpy(offsets.astype(np.int32)).cuda()
    A, W, dy, x_pre = (draw(rng, s, dtype)[0] for s in ((R, K), (E, K, N), (R, N), (R, K)))
    pre = draw(rng, (R, N), dtype)[0]

    def step():
        g = moe.ragged_matmul_backward(dy, A, W, off, moe.ACT_GELU, pre)
        back = moe.ragged_matmul_backward(dy, A, W, off, x_act=moe.ACT_SILU, x_pre=x_pre)
        rows = (moe.ragged_matmul(A, W, off, act=moe.ACT_RELU), g["dx"], back["dx"])
        return rows, (g["dW"], g["db"], back["dW"], back["db"])

    rows, weights = step()
    bad = int(np.flatnonzero(fills)[-1] if fills[0] == R else np.flatnonzero(fills[1:])[0] + 1)
    at = slice(int(offsets[bad]), int(offsets[bad + 1]))
    for t in (A, dy, pre, x_pre):
        t[at] = float("nan")
    W[bad] = float("nan")
    rows_, weights_ = step()
    others = torch.ones(R, dtype=torch.bool, device="cuda")
    others[at] = False
    for a, b in zip(rows, rows_):
        assert torch.equal(a[others], b[others]) and b[at].isnan().all()
    for a, b in zip(weights, weights_):
        assert torch.equal(a[:bad], b[:bad]) and torch.equal(a[bad + 1:], b[bad + 1:]) and b[bad].isnan().all()
