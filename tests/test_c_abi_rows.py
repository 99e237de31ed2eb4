"""Argument checks of the operators on experts' rows, of dense projections and of dropout, on the host: nothing is launched, no GPU is needed."""
import os

import pytest

FAKE, OUT = 4096, 1 << 20                                           # non-null, aligned, never dereferenced; results have addresses of their own


@pytest.fixture(scope="module")
def moe():
    from paper_2206_03382_amd import moe as m
    if not os.path.exists(m.LIB_PATH):
        from paper_2206_03382_amd.build import build_library
        build_library(verbose=False)
    m.lib()
    return m


def test_rows_refusals(moe):
    L = moe.lib()
    rows = lambda idx=FAKE, loc=FAKE, counts=FAKE, T=8, E=4, k=2, C=0, off=FAKE, src=FAKE, of=FAKE: L.moe_ragged_rows(idx, loc, counts, T, E, k, C, off, src, of, None)   # noqa: E731
    assert rows(idx=None) == rows(loc=None) == rows(counts=None) == rows(off=None) == rows(src=None) == rows(of=None) == moe.INVALID_ARG
    assert rows(T=0) == rows(E=0) == rows(k=0) == rows(k=5) == rows(C=-1) == moe.INVALID_ARG
    assert rows(E=513) == rows(T=1 << 30) == rows(T=1 << 29, k=2) == rows(idx=FAKE + 2) == rows(of=FAKE + 1) == moe.UNSUPPORTED


def test_product_refusals(moe):
    L = moe.lib()

    def product(A=FAKE, gather=None, rows=0, W=FAKE, bias=None, act=-1, dt=1, off=FAKE, R=8, E=2, K=64, N=64, pre=None, out=OUT):
        return L.moe_ragged_matmul(A, gather, rows, W, bias, act, dt, off, R, E, K, N, pre, out, None)

    assert product(A=None) == product(W=None) == product(off=None) == product(out=None) == product(out=FAKE) == product(pre=FAKE) == product(pre=OUT) == product(bias=OUT) == product(dt=2) == product(act=3) == product(act=-2) == moe.INVALID_ARG
    assert product(gather=FAKE) == product(R=0) == product(E=0) == product(K=0) == product(N=-8) == moe.INVALID_ARG
    assert product(K=12) == product(N=20) == product(E=513) == product(R=1 << 30) == product(K=1 << 21) == product(K=1 << 16, N=1 << 16) == moe.UNSUPPORTED
    assert product(A=FAKE + 8) == product(out=FAKE + 4) == product(bias=FAKE + 2) == product(pre=FAKE + 8) == product(off=FAKE + 2) == moe.UNSUPPORTED
    assert product(R=1 << 29, N=1 << 14) == product(gather=FAKE, rows=1 << 30) == product(gather=FAKE + 2, rows=8) == moe.UNSUPPORTED      # more tiles than a grid; rows

    def back(dy=FAKE, x=FAKE, gather=None, rows=0, W=FAKE, pre=None, act=-1, x_pre=None, x_act=-1, dt=1, off=FAKE, R=8, E=2, K=64, N=64, ws=FAKE, n=1 << 40, dx=OUT, dW=OUT + 256, db=OUT + 512):
        return L.moe_ragged_matmul_backward(dy, x, gather, rows, W, pre, act, x_pre, x_act, dt, off, R, E, K, N, ws, n, dx, dW, db, None)

    assert back(dy=None) == back(off=None) == back(ws=None) == back(x=None) == back(W=None) == back(dx=None, dW=None, db=None) == back(dt=7) == back(act=5) == moe.INVALID_ARG
    assert back(act=1) == back(pre=FAKE) == back(x_act=0) == back(x_pre=FAKE) == back(x_pre=FAKE, x_act=1, dx=None) == back(gather=FAKE) == moe.INVALID_ARG
    assert back(K=4) == back(dW=FAKE + 8) == back(ws=FAKE + 16) == back(x_pre=FAKE + 8, x_act=0) == moe.UNSUPPORTED
    assert back(pre=FAKE, act=1, n=64) == moe.WORKSPACE_TOO_SMALL
    assert back(dx=FAKE) == back(dW=FAKE) == back(db=FAKE) == back(dx=OUT + 256) == back(dW=OUT + 512) == moe.INVALID_ARG
    size = L.moe_ragged_matmul_backward_workspace_bytes
    assert size(8, 2, 64, 64, 1, 1) >= 8 * 64 * 2 and size(8, 2, 64, 64, -1, 1) > 0
    assert size(8, 2, 60, 64, 1, 1) == size(0, 2, 64, 64, 1, 1) == size(8, 2, 64, 64, 9, 1) == size(8, 2, 64, 64, 1, 5) == 0


def test_linear_refusals(moe):
    L = moe.lib()
    lin = lambda x=FAKE, W=FAKE, b=None, act=-1, res=None, dt=1, T=1, K=64, N=64, ws=None, n=0, pre=None, out=OUT: L.moe_linear(   # noqa: E731
        x, W, b, act, res, dt, T, K, N, ws, n, pre, out, None)
    assert lin(x=None) == lin(W=None) == lin(out=None) == lin(out=FAKE) == lin(pre=OUT) == lin(pre=FAKE) == lin(b=OUT) == lin(res=OUT + 256, pre=OUT + 256) == lin(act=4) == lin(dt=-1) == lin(T=0) == lin(K=0) == moe.INVALID_ARG
    assert lin(K=4) == lin(N=4) == lin(x=FAKE + 8) == lin(res=FAKE + 4) == lin(b=FAKE + 8) == lin(K=1 << 20, N=1 << 12) == moe.UNSUPPORTED
    need = L.moe_linear_workspace_bytes(1, 4096, 64, 1)
    assert need > 0 and L.moe_linear_workspace_bytes(1, 64, 64, 1) == L.moe_linear_workspace_bytes(1, 4096, 64, 0) == L.moe_linear_workspace_bytes(1, 4096, 60, 1) == 0
    assert lin(K=4096) == moe.INVALID_ARG and lin(K=4096, ws=FAKE, n=need - 1) == moe.WORKSPACE_TOO_SMALL and lin(K=4096, ws=FAKE + 128, n=need) == moe.UNSUPPORTED
    back = lambda dy=FAKE, x=FAKE, W=FAKE, pre=None, act=-1, T=4, K=64, ws=FAKE, n=1 << 40, dx=OUT, dW=OUT + 256, db=OUT + 512: L.moe_linear_backward(   # noqa: E731
        dy, x, W, pre, act, 1, T, K, 64, ws, n, dx, dW, db, None)
    assert back(dy=None) == back(x=None) == back(W=None) == back(ws=None) == back(act=0) == back(pre=FAKE) == back(dx=None, dW=None, db=None) == back(T=0) == moe.INVALID_ARG
    assert back(dx=FAKE) == back(dW=FAKE) == back(db=FAKE) == back(db=OUT) == moe.INVALID_ARG
    assert back(K=12) == back(ws=FAKE + 128) == back(db=FAKE + 8) == moe.UNSUPPORTED and back(n=16) == moe.WORKSPACE_TOO_SMALL
    assert L.moe_linear_backward_workspace_bytes(4, 64, 64, 0, 1) > 0 and L.moe_linear_backward_workspace_bytes(4, 64, 62, 0, 1) == 0


def test_dropout_and_combine_refusals(moe):
    L = moe.lib()
    drop = lambda x=FAKE, res=None, p=0.5, seed=FAKE, dt=1, n=64, out=OUT: L.moe_dropout(x, res, p, seed, dt, n, out, None)   # noqa: E731
    assert drop(x=None) == drop(out=None) == drop(p=-0.1) == drop(p=1.5) == drop(p=float("nan")) == drop(seed=None) == drop(dt=3) == drop(n=0) == moe.INVALID_ARG
    assert drop(n=12) == drop(n=1 << 40) == drop(x=FAKE + 8) == drop(res=FAKE + 2) == drop(seed=FAKE + 4) == moe.UNSUPPORTED
    comb = lambda Y=FAKE, R=8, of=FAKE, w=None, res=None, p=0.0, seed=None, dt=1, T=4, M=64, k=2, out=OUT: L.moe_ragged_combine(Y, R, of, w, res, p, seed, dt, T, M, k, out, None)   # noqa: E731
    assert comb(Y=None) == comb(of=None) == comb(out=None) == comb(out=FAKE) == comb(p=0.5) == comb(R=0) == comb(T=0) == comb(k=0) == comb(dt=2) == moe.INVALID_ARG
    assert comb(M=12) == comb(k=513) == comb(T=1 << 30) == comb(R=1 << 30) == comb(Y=FAKE + 8) == comb(w=FAKE + 2) == comb(M=1 << 21) == moe.UNSUPPORTED
    back = lambda d=FAKE, Y=FAKE, R=8, of=FAKE, p=0.0, seed=None, T=4, M=64, k=2, dY=OUT, dw=OUT + 256: L.moe_ragged_combine_backward(d, Y, R, of, None, p, seed, 1, T, M, k, dY, dw, None)   # noqa: E731
    assert back(d=None) == back(Y=None) == back(of=None) == back(dY=None) == back(dY=FAKE) == back(dw=None) == back(p=0.1) == back(T=0) == moe.INVALID_ARG
    assert back(M=4) == back(dY=FAKE + 8) == back(dw=FAKE + 1) == back(p=0.1, seed=FAKE + 4) == moe.UNSUPPORTED
