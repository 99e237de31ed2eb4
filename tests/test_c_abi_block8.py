"""Argument checks of the norm, the 8-bit matrices and the few-token layer, on the host: nothing is launched, no GPU is needed."""
import os

import pytest

FAKE = 4096                                                         # non-null, aligned, never dereferenced


@pytest.fixture(scope="module")
def moe():
    from paper_2206_03382_amd import moe as m
    if not os.path.exists(m.LIB_PATH):
        from paper_2206_03382_amd.build import build_library
        build_library(verbose=False)
    m.lib()
    return m


def test_norm_refusals(moe):
    L = moe.lib()
    norm = lambda x=FAKE, res=None, w=FAKE, eps=1e-6, dt=1, T=8, M=64, h=None, y=FAKE, q=None, s=None: L.moe_rms_norm(x, res, w, eps, dt, T, M, h, y, q, s, None)   # noqa: E731
    assert norm(x=None) == norm(eps=0.0) == norm(eps=1e-60) == norm(eps=float("nan")) == norm(dt=2) == norm(T=0) == moe.INVALID_ARG
    assert norm(y=None) == norm(q=FAKE) == norm(s=FAKE) == norm(res=FAKE) == moe.INVALID_ARG
    assert norm(M=60) == norm(M=16392) == norm(T=1 << 22) == norm(x=FAKE + 4) == norm(w=FAKE + 8) == norm(y=FAKE + 2) == moe.UNSUPPORTED
    back = lambda dy=FAKE, h=FAKE, ws=FAKE, n=1 << 30, dx=FAKE, dw=FAKE, M=64, T=8: L.moe_rms_norm_backward(dy, None, h, FAKE, 1e-6, 1, T, M, ws, n, dx, dw, None)   # noqa: E731
    assert back(dy=None) == back(h=None) == back(dx=None) == back(ws=None) == back(T=0) == moe.INVALID_ARG
    assert back(n=16) == moe.WORKSPACE_TOO_SMALL
    assert back(M=4) == back(ws=FAKE + 16) == moe.UNSUPPORTED
    assert L.moe_rms_norm_backward_workspace_bytes(8, 64) >= 8 * 64 * 4 and L.moe_rms_norm_backward_workspace_bytes(8, 60) == 0


def test_format_sizes(moe):
    L = moe.lib()
    assert [L.moe_row_bytes8(k) for k in (1, 128, 129, 4096, 0)] == [128, 128, 256, 4096, -1]
    assert [L.moe_row_scales8(k) for k in (1, 512, 513, 4096, 0)] == [4, 4, 8, 32, -1]


def test_matrix_refusals(moe):
    L = moe.lib()
    quant = lambda src=FAKE, dt=1, E=2, R=8, K=64, mode=0, q=FAKE, s=FAKE, qt=None, st=None: L.moe_quantize8(src, dt, None, E, R, K, mode, q, s, qt, st, None)   # noqa: E731
    assert quant(src=None) == quant(dt=3) == quant(E=0) == quant(R=0) == quant(mode=2) == quant(q=None) == quant(s=None) == quant(qt=FAKE) == moe.INVALID_ARG
    assert quant(q=None, s=None) == quant(E=65536) == moe.INVALID_ARG
    assert quant(K=12) == quant(src=FAKE + 8) == quant(q=FAKE + 8) == quant(R=1 << 30, K=1 << 20) == moe.UNSUPPORTED
    assert L.moe_dequantize8(None, FAKE, 0, 1, 8, 64, 1, FAKE, None) == L.moe_dequantize8(FAKE, FAKE, 5, 1, 8, 64, 1, FAKE, None) == moe.INVALID_ARG
    assert L.moe_dequantize8(FAKE, FAKE, 0, 1, 8, 60, 1, FAKE, None) == moe.UNSUPPORTED
    mm = lambda A=FAKE, As=FAKE, mode=1, act=-1, dt=1, gather=None, rows=0, E=2, C=8, K=64, N=64, out=FAKE, o8=None, os=None: L.moe_matmul8(   # noqa: E731
        A, As, FAKE, FAKE, mode, None, act, dt, None, None, gather, rows, E, C, K, N, out, o8, os, None)
    assert mm(A=None) == mm(As=None) == mm(mode=2) == mm(act=3) == mm(dt=9) == mm(gather=FAKE) == mm(E=0) == mm(C=0) == mm(K=0) == moe.INVALID_ARG
    assert mm(out=None) == mm(o8=FAKE, os=FAKE) == mm(out=None, o8=FAKE) == moe.INVALID_ARG
    assert mm(N=12) == mm(A=FAKE + 8) == mm(As=FAKE + 1) == mm(N=1 << 20, K=4096) == moe.UNSUPPORTED


def test_linear8_refusals(moe):
    L = moe.lib()
    assert L.moe_expert_linear8_state_bytes(2, 8, 64, 64) >= 2 * (64 * 128 + 64 * 128 + 64 * 128 + 8 * 128)
    assert L.moe_expert_linear8_state_bytes(2, 8, 60, 64) == L.moe_expert_linear8_state_bytes(2, 8, 64, 12) == L.moe_expert_linear8_state_bytes(0, 8, 64, 64) == 0
    train = lambda x=FAKE, W=FAKE, dt=1, E=2, C=8, K=64, N=64, y=FAKE, st=FAKE, n=1 << 30: L.moe_expert_linear8_train(x, W, dt, None, E, C, K, N, y, st, n, None)   # noqa: E731
    assert train(x=None) == train(W=None) == train(y=None) == train(st=None) == train(dt=7) == train(E=0) == train(C=0) == moe.INVALID_ARG
    assert train(K=12) == train(N=20) == train(x=FAKE + 8) == train(st=FAKE + 16) == train(K=1 << 16, N=1 << 16) == moe.UNSUPPORTED
    assert train(n=64) == moe.WORKSPACE_TOO_SMALL
    back = lambda dy=FAKE, dt=1, K=64, st=FAKE, n=1 << 30, dx=FAKE, dW=FAKE: L.moe_expert_linear8_backward(dy, dt, None, 2, 8, K, 64, st, n, dx, dW, None)   # noqa: E731
    assert back(dy=None) == back(st=None) == back(dx=None, dW=None) == back(dt=-1) == moe.INVALID_ARG
    assert back(K=4) == back(dW=FAKE + 4) == moe.UNSUPPORTED and back(n=0) == moe.WORKSPACE_TOO_SMALL


def test_layer_refusals(moe):
    L = moe.lib()
    ffn = lambda x=FAKE, act=0, M=64, H=64, slots=None, T=0, hid=FAKE: L.moe_expert_ffn8(x, FAKE, slots, T, FAKE, FAKE, None, FAKE, FAKE, None, act, 1, None, 2, 8, M, H, hid, FAKE, FAKE, None)   # noqa: E731
    assert ffn(x=None) == ffn(act=-1) == ffn(slots=FAKE) == ffn(hid=None) == moe.INVALID_ARG
    assert ffn(M=12) == ffn(H=12) == ffn(x=FAKE + 4) == moe.UNSUPPORTED
    few = lambda T=4, s1=None, s2=None, M=64, n=1 << 30, k=1, f=1.0, E=4, ws=FAKE: L.moe_layer_forward_few(   # noqa: E731
        FAKE, FAKE, None, FAKE, s1, None, FAKE, s2, None, T, M, 64, E, k, f, 0, 0, 1, FAKE, None, None, None, None, None, ws, n, None)
    assert few(s1=FAKE) == few(k=5) == few(f=0.0) == few(T=0) == few(ws=None) == moe.INVALID_ARG
    assert few(T=moe.FEW_MAX_TOKENS + 1) == few(M=12) == few(E=513) == few(ws=FAKE + 16) == moe.UNSUPPORTED
    assert few(n=64) == moe.WORKSPACE_TOO_SMALL
    assert L.moe_layer_few_workspace_bytes(64, 64, 64, 4, 1, 1) > 0 and L.moe_layer_few_workspace_bytes(65, 64, 64, 4, 1, 1) == 0
    full = lambda x8=FAKE, n=1 << 40, M=64, f=1.0: L.moe_layer_forward8(FAKE, x8, FAKE, FAKE, None, FAKE, FAKE, None, FAKE, FAKE, None, 100, M, 64, 4, 1, f, 0, 0, 1, FAKE, None, None, None, None, None, FAKE, n, None)   # noqa: E731
    assert full(x8=None) == full(f=-1.0) == moe.INVALID_ARG
    assert full(M=20) == moe.UNSUPPORTED and full(n=64) == moe.WORKSPACE_TOO_SMALL
    assert L.moe_layer8_workspace_bytes(100, 64, 64, 4, 1, 25, 1) > 0 and L.moe_layer8_workspace_bytes(100, 60, 64, 4, 1, 25, 1) == 0
