"""A padded batch: choices of padding tokens are marked by an expert that does not exist, while the counts still announce their rows.  Forward and backward of a projection on the rows that choices
have, against the 64-bit reference; the rows that no choice has add nothing to the gradients if dY is cleared, as the bindings' documentation asks.  Tolerances: test_rows_gpu.py's."""
import numpy as np
import pytest
import torch

from oracle import rows_oracle as O
from test_rows_gpu import BF, F32, HALF, assert_within, draw, moe, route, sum_error   # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,E,k,K,N", [(70, 5, 2, 64, 72), (9, 8, 3, 328, 136), (1500, 3, 1, 256, 512)])
def test_padded_batch(moe, T, E, k, K, N, dtype):   # noqa: F811
    rng = np.random.default_rng(T)
    idx, loc, counts = route(rng, T, E, k)
    real = T // 2
    idx[real:] = -1
    x, x64 = draw(rng, (T, K), dtype)
    W, W64 = draw(rng, (E, K, N), dtype, 1.0 / np.sqrt(K))
    dout, dout64 = draw(rng, (T, N), dtype)
    w, w64 = draw(rng, (T, k), F32)
    poison = [torch.full((T * k, n), float("nan"), dtype=dtype, device="cuda") for n in (K, N, N)]       # what fresh memory may hold
    del poison
    rows = moe.ragged_rows(*(torch.from_numpy(a).cuda() for a in (idx, loc, counts)))
    Y = moe.ragged_matmul(x, W, rows.offsets, gather=rows.row_src)
    out = moe.ragged_combine(Y, rows.row_of, w)
    dY, dw = moe.ragged_combine_backward(dout, Y, rows.row_of, w, dY=torch.zeros_like(Y))
    g = moe.ragged_matmul_backward(dY, x, W, rows.offsets, gather=rows.row_src)
    dx = moe.ragged_combine(g["dx"], rows.row_of, None)

    h, u = HALF[dtype], 2.0 ** -24
    dW, eW, db, eb = np.zeros(W64.shape), np.zeros(W64.shape), np.zeros((E, N)), np.zeros((E, N))
    for t in range(T):
        ref, bound, ref_dx, bound_dx = np.zeros(N), np.zeros(N), np.zeros(K), np.zeros(K)
        for j in range(k if t < real else 0):
            e = idx[t, j]
            y, S = x64[t] @ W64[e], np.abs(x64[t]) @ np.abs(W64[e])
            ref += w64[t, j] * y
            bound += np.abs(w64[t, j]) * (sum_error(dtype, K) * S + h * (np.abs(y) + S * 2.0 ** -10)) + (k + 3) * u * np.abs(w64[t, j] * y) * 1.01
            d = w64[t, j] * dout64[t]
            off = (h + 4 * u) * np.abs(d)                            # dY's rounding
            dW[e] += np.outer(x64[t], d)
            eW[e] += np.outer(np.abs(x64[t]), off + (sum_error(dtype, int(counts[e])) * 1.01) * np.abs(d))
            db[e] += d
            eb[e] += off + (counts[e] / 8 + 96) * u * 1.01 * np.abs(d)
            back, S = d @ W64[e].T, np.abs(d) @ np.abs(W64[e].T)
            ref_dx += back
            bound_dx += off @ np.abs(W64[e].T) + sum_error(dtype, N) * S * 1.01 + h * (np.abs(back) + S * 2.0 ** -6) + (k + 3) * u * S
        assert_within(out[t], ref, bound + h * (np.abs(ref) + bound), f"out of token {t}")
        assert_within(dx[t], ref_dx, bound_dx + h * (np.abs(ref_dx) + bound_dx), f"dx of token {t}")
    assert_within(g["dW"], dW, eW + h * (np.abs(dW) + eW), "dW")
    assert_within(g["db"], db, eb + h * (np.abs(db) + eb), "db")
    assert (dw[real:] == 0).all() and (out[real:] == 0).all() and (dx[real:] == 0).all()
