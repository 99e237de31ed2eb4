"""The 8-bit block format, its products and the layers on them against 64-bit references.

Tolerances.  Quantising involves no sum: values and exponents are compared exactly.  Products of bf16 results: half a unit in the last place, 2^-8 of the result,
and what the instruction loses of a step's 128 products, which it aligns to the largest: taken as 2^-14 of the sum of the magnitudes, which is no less
than 128 times an alignment to 21 bits.  fp32 results: exact products and fp32 sums of at most K / 32 + 40 roundings.  Activations in 8 bits between two products: an fp32 sum off
by a little may round to the other neighbour, a step of 2^-3 of the value; the reference is therefore evaluated on the hidden activations that the library stored, which are
checked by themselves.
"""
import math

import numpy as np
import pytest
import torch

from oracle import block8_oracle as B
from oracle import moe_oracle as O
from paper_2206_03382_amd import synth

pytestmark = pytest.mark.gpu

UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


@pytest.fixture(scope="module")
def moe():
    assert torch.cuda.is_available(), "these tests need a GPU"
    from paper_2206_03382_amd import moe as m
    m.lib()
    return m


def values(m):
    """float64 values of a Block8, from its bytes."""
    raw = m.q.view(torch.uint8).cpu().numpy()
    exps = m.s.cpu().numpy().astype(np.int64) - 127
    R = raw.shape[-2]
    e = np.repeat(exps, 128, axis=-1)[..., :raw.shape[-1]]
    if m.blocks:
        e = np.repeat(e, 128, axis=-2)[..., :R, :]
    return (B.e4m3_table()[raw] * 2.0 ** e)[..., :m.width]


def assert_stored(m, v, blocks, rows=None):
    """A Block8 holds what the reference stores of v, zeros past the width and 1 as the exponents past the blocks."""
    ref, exps = B.quantize(v, blocks)
    nb = exps.shape[-1]
    got = m.s.cpu().numpy().astype(np.int64) - 127
    assert np.array_equal(got[..., :nb], exps) and (got[..., nb:] == 0).all()
    raw = m.q.view(torch.uint8).cpu().numpy()
    assert (raw[..., m.width:] == 0).all()
    assert np.array_equal(values(m), ref)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("E,R,K", [(1, 1, 8), (1, 5, 128), (2, 130, 136), (3, 128, 520), (1, 257, 264), (2, 77, 1032)])
def test_quantize(moe, E, R, K, dtype):
    rng = np.random.default_rng(R + K)
    v = rng.standard_normal((E, R, K)) * np.exp2(rng.integers(-40, 40, (E, R, 1)))
    v[0, 0] = 0
    v[-1, -1, :8] = [448.0, -448.0, 449.0, 2.0 ** -9, 1.0625, 1.1875, 240.0, 464.0]          # the line between exponents, ties
    x = torch.from_numpy(v.astype(np.float32)).to(dtype)
    v = x.double().numpy()
    for blocks in (False, True):
        q, qt = moe.quantize8(x.cuda(), blocks=blocks, rows=True, transposed=True)
        assert_stored(q, v, blocks)
        assert_stored(qt, np.ascontiguousarray(v.transpose(0, 2, 1)), blocks)
        one, none = moe.quantize8(x.cuda(), blocks=blocks)
        other, two = moe.quantize8(x.cuda(), blocks=blocks, rows=False, transposed=True)
        assert none is None and other is None
        for a, b in ((one, q), (two, qt)):
            assert torch.equal(a.q.view(torch.uint8), b.q.view(torch.uint8)) and torch.equal(a.s, b.s)
        back = moe.dequantize8(q, torch.float32)
        assert np.array_equal(back.double().cpu().numpy(), values(q))
        assert torch.equal(moe.dequantize8(q).float(), back)


def test_quantize_ties_and_small_values(moe):
    """Every midpoint between neighbours of the format, and its neighbours in fp32, at a block whose exponent is 0."""
    mags = B.e4m3_table()[:127]
    mid = (mags[1:] + mags[:-1]) / 2
    v = np.concatenate([mid, np.nextafter(mid.astype(np.float32), np.float32(0)), np.nextafter(mid.astype(np.float32), np.float32(500)), mags]).astype(np.float32)
    v = v[v <= 448]
    v = np.concatenate([v, -v])
    rows = np.full((-(-len(v) // 127), 128), 0, dtype=np.float32)
    rows[:, 0] = 448.0
    for i, row in enumerate(rows):
        part = v[i * 127:(i + 1) * 127]
        row[1:1 + len(part)] = part
    q, _ = moe.quantize8(torch.from_numpy(rows).cuda())
    assert (q.s[:, 0] == 127).all()
    assert_stored(q, rows.astype(np.float64), False)


def test_quantize_nonfinite(moe):
    x = torch.ones((3, 304), device="cuda")
    x[0, 3] = float("nan")
    x[1, 130] = float("-inf")
    q, qt = moe.quantize8(x, transposed=True)
    assert q.s[0].tolist()[:3] == [255, 119, 119] and q.s[1].tolist()[:3] == [119, 255, 119]
    back = moe.dequantize8(q)
    assert torch.isnan(back[0, :128]).all() and torch.isnan(back[1, 128:256]).all()
    assert (back[0, 128:] == 1).all() and (back[2] == 1).all()
    assert [int(s) for s in (qt.s[3, 0], qt.s[130, 0], qt.s[4, 0])] == [255, 255, 119]
    ones, _ = moe.quantize8(torch.ones((1, 8, 304), device="cuda"))
    for dtype in (torch.float32, torch.bfloat16):
        y = moe.matmul8(moe.Block8(q.q[None], q.s[None], 304, False), ones, dtype=dtype)
        assert torch.isnan(y[0, :2]).all() and (y[0, 2] == 304).all()


def test_quantize_counts(moe):
    """Rows past an expert's fill: not written; zeros in the transposed form up to the end of their block."""
    rng = np.random.default_rng(0)
    E, R, K = 5, 300, 136
    x = torch.from_numpy(rng.standard_normal((E, R, K)).astype(np.float32)).cuda()
    x[2, 130:] = float("nan")                                      # what a slab holds past its fill must not matter
    counts = torch.tensor([0, 1, 130, 400, -3], dtype=torch.int32, device="cuda")
    q, qt = moe.quantize8(x, transposed=True, counts=counts)
    v = x.double().cpu().numpy()
    for e, n in enumerate((0, 1, 130, 300, 0)):
        if n == 0:
            continue
        live = np.where(np.arange(R)[:, None] < n, v[e], 0.0)
        assert_stored(moe.Block8(q.q[e, :n], q.s[e, :n], K, False), live[:n], False)
        upto = -(-n // 128)
        ref, exps = B.quantize(np.ascontiguousarray(live.T), False)
        got = values(moe.Block8(qt.q[e], qt.s[e], R, False))
        assert np.array_equal(got[:, :min(R, upto * 128)], ref[:, :min(R, upto * 128)])


def operand(moe, rng, E, R, K, blocks, spread=3):
    v = rng.standard_normal((E, R, K)) * np.exp2(rng.integers(-spread, spread + 1, (E, R, 1)))
    q, _ = moe.quantize8(torch.from_numpy(v.astype(np.float32)).cuda(), blocks=blocks)
    return q, values(q)


def assert_product(got, ref, mags, K, dtype, what="product"):
    got = got.double().cpu().numpy()
    lost = 2.0 ** -14 if dtype == torch.bfloat16 else (K / 32 + 40) * 2.0 ** -24
    over = np.abs(got - ref) - (UNIT[dtype] * np.abs(ref) + lost * mags + 1e-30)
    assert np.isfinite(got).all() and over.max() <= 0, f"{what}: {over.max():.3e} beyond the bound, at {np.argwhere(over > 0)[:3]}"


MATMULS = [(1, 1, 8, 8), (1, 3, 128, 16), (2, 17, 136, 40), (1, 129, 640, 136), (3, 256, 512, 256), (1, 300, 1032, 520), (2, 520, 264, 264), (5, 64, 1288, 1000),
           (1, 1024, 2048, 512), (9, 40, 384, 1152),
           (24, 453, 1040, 776), (1, 2100, 8328, 4104), (1, 200, 8328, 264)]          # the large tile, with more exponents than LDS holds at a time; the small one with them


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("E,C,K,N", MATMULS)
def test_matmul8(moe, E, C, K, N, dtype):
    rng = np.random.default_rng(C + K)
    A, a = operand(moe, rng, E, C, K, False)
    for blocks in (False, True):
        W, w = operand(moe, rng, E, N, K, blocks)
        bias = torch.from_numpy(rng.standard_normal((E, N)).astype(np.float32)).to(dtype)
        b = bias.double().numpy()[:, None, :]
        ref, mags = a @ w.transpose(0, 2, 1), np.abs(a) @ np.abs(w).transpose(0, 2, 1)
        assert_product(moe.matmul8(A, W, dtype=dtype), ref, mags, K, dtype)
        got = moe.matmul8(A, W, bias=bias.cuda(), act=moe.ACT_RELU, dtype=dtype)
        assert_product(got, np.maximum(ref + b, 0), mags + np.abs(b), K, dtype, "bias and relu")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_matmul8_counts_and_gather(moe, dtype):
    rng = np.random.default_rng(5)
    E, C, K, N, T = 7, 300, 392, 264, 500
    counts = torch.tensor([0, 1, 16, 129, 300, 900, -1], dtype=torch.int32, device="cuda")
    fills = [0, 1, 16, 129, 300, 300, 0]
    W, w = operand(moe, rng, E, N, K, True)
    A, a = operand(moe, rng, E, C, K, False)
    out = torch.full((E, C, N), 7.0, dtype=dtype, device="cuda")
    moe.matmul8(A, W, dtype=dtype, counts=counts, out=out)
    X, x = operand(moe, rng, 1, T, K, False)
    X = moe.Block8(X.q[0], X.s[0], K, False)
    gather = rng.integers(-1, T + 1, (E, C)).astype(np.int32)       # out of range: row 0
    out2 = torch.full((E, C, N), 7.0, dtype=dtype, device="cuda")
    moe.matmul8(X, W, dtype=dtype, counts=counts, gather=torch.from_numpy(gather).cuda(), out=out2)
    rows = np.where((gather < 0) | (gather >= T), 0, gather)
    for e, n in enumerate(fills):
        assert (out[e, n:] == 7).all() and (out2[e, n:] == 7).all()
        if n:
            assert_product(out[e, :n], a[e, :n] @ w[e].T, np.abs(a[e, :n]) @ np.abs(w[e]).T, K, dtype)
            z = x[0][rows[e, :n]]
            assert_product(out2[e, :n], z @ w[e].T, np.abs(z) @ np.abs(w[e]).T, K, dtype, "gathered")


def test_matmul8_many_experts(moe):
    """More experts than the tile search takes."""
    rng = np.random.default_rng(6)
    E, C, K, N = 600, 5, 128, 24
    A, a = operand(moe, rng, E, C, K, False)
    W, w = operand(moe, rng, E, N, K, False)
    counts = rng.integers(0, C + 2, E).astype(np.int32)
    got = moe.matmul8(A, W, counts=torch.from_numpy(counts).cuda())
    live = np.arange(C)[None, :, None] < counts[:, None, None]
    assert_product(got, np.where(live, a @ w.transpose(0, 2, 1), 0), np.abs(a) @ np.abs(w).transpose(0, 2, 1), K, torch.bfloat16)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("E,C,K,N,ragged", [(1, 8, 8, 8, False), (3, 37, 136, 264, True), (2, 300, 520, 392, True), (4, 256, 256, 512, False), (1, 1, 128, 128, False), (17, 453, 776, 1544, True)])
def test_linear8_training_pass(moe, E, C, K, N, ragged, dtype):
    """y, dx and dW from the operands as the format holds them, and the gradients against differences of <y, dy> (bilinear in the stored operands, so that a difference
    is exact but for its own roundings)."""
    rng = np.random.default_rng(C + N)
    x = torch.from_numpy(rng.standard_normal((E, C, K)).astype(np.float32)).to(dtype)
    W = torch.from_numpy((rng.standard_normal((E, K, N)) / math.sqrt(K)).astype(np.float32)).to(dtype)
    dy = torch.from_numpy(rng.standard_normal((E, C, N)).astype(np.float32)).to(dtype)
    fills = [int(n) for n in rng.integers(0, C + C // 2 + 2, E)] if ragged else [C] * E
    counts = torch.tensor(fills, dtype=torch.int32, device="cuda") if ragged else None
    y, kept = moe.expert_linear8_train(x.cuda(), W.cuda(), counts=counts)
    dx, dW = moe.expert_linear8_backward(dy.cuda(), kept)
    live = np.arange(C)[None, :, None] < np.array(fills)[:, None, None]
    x64, W64, dy64 = np.where(live, x.double().numpy(), 0), W.double().numpy(), np.where(live, dy.double().numpy(), 0)
    qx, qW, qdy = B.quantize(x64, False)[0], B.quantize(W64, True)[0], B.quantize(dy64, False)[0]
    tr = lambda v: np.ascontiguousarray(v.transpose(0, 2, 1))       # noqa: E731
    qxt, qdyt = B.quantize(tr(x64), False)[0], B.quantize(tr(dy64), False)[0]
    assert_product(y, qx @ qW, np.abs(qx) @ np.abs(qW), K, dtype, "y")
    assert_product(dx, qdy @ tr(qW), np.abs(qdy) @ np.abs(tr(qW)), N, dtype, "dx")
    assert_product(dW, qxt @ tr(qdyt), np.abs(qxt) @ np.abs(tr(qdyt)), C, dtype, "dW")
    lost = 2.0 ** -8 + 2.0 ** -13 if dtype == torch.bfloat16 else 2.0 ** -16
    d = rng.standard_normal((E, C, K))
    along = np.sum(((qx + d) @ qW - (qx - d) @ qW) / 2 * qdy)
    gx = dx.double().cpu().numpy()
    assert abs(np.sum(gx * d) - along) <= lost * np.sum(np.abs(qdy) @ np.abs(tr(qW)) * np.abs(d))
    d = rng.standard_normal((E, K, N))
    along = np.sum(((tr(qxt) @ (qW + d)) - (tr(qxt) @ (qW - d))) / 2 * tr(qdyt))
    gw = dW.double().cpu().numpy()
    assert abs(np.sum(gw * d) - along) <= lost * np.sum(np.abs(qxt) @ np.abs(tr(qdyt)) * np.abs(d)) + 1e-30


ACTS = {0: lambda v: np.maximum(v, 0), 1: lambda v: O.activation(v, 1), 2: lambda v: O.activation(v, 2)}


def ffn8_reference(z, W1, b1, W2, b2, act, hidden):
    """The two products in float64; the second one on `hidden`, the activations as the library stored them, after those have been checked: each within a step of
    the format and the first product's own error of its value."""
    up = z @ W1.T + (0 if b1 is None else b1)
    h = ACTS[act](up)
    mags = np.abs(z) @ np.abs(W1).T + (0 if b1 is None else np.abs(b1))
    pad = np.zeros((h.shape[0], -(-h.shape[1] // 128) * 128))
    pad[:, :h.shape[1]] = np.abs(h) + 1.2 * 2.0 ** -14 * mags
    amax = np.repeat(pad.reshape(h.shape[0], -1, 128).max(-1), 128, axis=1)[:, :h.shape[1]]
    assert (np.abs(hidden - h) <= 2.0 ** -4 * np.abs(h) + 1.3 * 2.0 ** -14 * mags + amax / 224.0 * 2.0 ** -10).all()   # slopes of the activations: at most 1.13
    return hidden @ W2.T + (0 if b2 is None else b2), np.abs(hidden) @ np.abs(W2).T + (0 if b2 is None else np.abs(b2))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("E,C,M,H,T,act,bias", [(2, 5, 64, 136, 9, 0, True), (3, 70, 264, 520, 100, 1, True), (4, 300, 256, 384, 700, 2, False), (1, 513, 512, 1024, 513, 1, True), (24, 453, 1040, 776, 900, 1, True)])
def test_expert_ffn8(moe, E, C, M, H, T, act, bias, dtype):
    rng = np.random.default_rng(C + H)
    X, x = operand(moe, rng, 1, T, M, False, spread=1)
    X = moe.Block8(X.q[0], X.s[0], M, False)
    W = [torch.from_numpy((rng.standard_normal((E, a, b)) / math.sqrt(a)).astype(np.float32)).cuda() for a, b in ((M, H), (H, M))]
    W1, W2 = (moe.quantize8(w, blocks=True, rows=False, transposed=True)[1] for w in W)
    b1 = torch.from_numpy(rng.standard_normal((E, H)).astype(np.float32) * 0.1).to(dtype) if bias else None
    b2 = torch.from_numpy(rng.standard_normal((E, M)).astype(np.float32) * 0.1).to(dtype) if bias else None
    dev = lambda t: None if t is None else t.cuda()                 # noqa: E731
    slots = torch.from_numpy(rng.integers(0, T, (E, C)).astype(np.int32))
    fills = [min(C, int(n)) for n in rng.integers(0, C + C // 2 + 1, E)]
    fills[0] = C
    counts = torch.tensor(fills, dtype=torch.int32, device="cuda")
    L = moe.lib()
    code = moe.F32 if dtype == torch.float32 else moe.BF16
    hid = moe._alloc8((E,), C, H, False, "cuda")
    Y = torch.full((E, C, M), float("nan"), dtype=dtype, device="cuda")
    p = lambda t: None if t is None else t.data_ptr()               # noqa: E731
    b1d, b2d, sd = dev(b1), dev(b2), slots.cuda()
    assert L.moe_expert_ffn8(p(X.q), p(X.s), p(sd), T, p(W1.q), p(W1.s), p(b1d), p(W2.q), p(W2.s), p(b2d), act, code, p(counts), E, C, M, H,
                             p(hid.q), p(hid.s), p(Y), torch.cuda.current_stream().cuda_stream) == moe.OK
    same = moe.expert_ffn8(X, W1, b1d, W2, b2d, act, dtype, counts=counts, slot_src=sd)
    w1, w2, hv = values(W1), values(W2), values(hid)
    for e, n in enumerate(fills):
        assert torch.isnan(Y[e, n:]).all()
        if n == 0:
            continue
        assert torch.equal(Y[e, :n], same[e, :n])
        f64 = lambda b: None if b is None else b[e].double().numpy()        # noqa: E731
        ref, mags = ffn8_reference(x[0][slots[e, :n].numpy()], w1[e], f64(b1), w2[e], f64(b2), act, hv[e, :n])
        assert_product(Y[e, :n], ref, mags, H, dtype, "Y")
    # slabs instead of gathered rows: the same numbers
    Z = moe.Block8(X.q[sd.long()].contiguous(), X.s[sd.long()].contiguous(), M, False)
    slabs = moe.expert_ffn8(Z, W1, b1d, W2, b2d, act, dtype, counts=counts)
    for e, n in enumerate(fills):
        assert torch.equal(slabs[e, :n], Y[e, :n])


def dev_of(a, dt):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(dt).cuda()


@pytest.mark.parametrize("T", [300, 33])
def test_norm_layer8_runs_the_path(moe, T):
    """The pre-norm block on 8-bit experts: routing exactly as the gate's on the normalised tokens, output as the 8-bit experts' in 64 bits on that routing.  The activations'
    own rounding to 8 bits is 2^-4 of each at most and independent from one to the next: 2.7 % of the result, measured as a 2-norm, and less where few tokens keep them in bf16."""
    cfg = synth.CONFIGS[1].scaled(T=T, M=256, H=512, E=8)
    inp = synth.make_inputs(cfg, seed=4, bias_std=0.1)
    dt = torch.bfloat16
    W = [moe.quantize8(dev_of(inp[n], dt), blocks=True, rows=False, transposed=True)[1] for n in ("W1", "W2")]
    g = np.random.default_rng(1)
    w = synth.round_to_bf16(1 + 0.1 * g.standard_normal(256).astype(np.float32))
    res = synth.round_to_bf16(g.standard_normal((T, 256)).astype(np.float32))
    layer = moe.NormMoELayer8(dev_of(w, dt), 1e-6, dev_of(inp["Wg"], dt), None, W[0], dev_of(inp["b1"], dt), W[1], dev_of(inp["b2"], dt), T, cfg.k, cfg.f,
                              cfg.normalize, cfg.act, keep_routing=True)
    assert (layer.few is not None) == (T <= moe.FEW_MAX_TOKENS)
    out, h = layer.forward(dev_of(inp["x"], dt), dev_of(res, dt))
    h64, y64 = B.rms_norm(inp["x"].astype(np.float64), res.astype(np.float64), w.astype(np.float64), 1e-6)
    assert np.abs(h.double().cpu().numpy() - h64).max() <= 2.0 ** -8 * np.abs(h64).max()
    y = layer.normed["y"].float().cpu().numpy()                    # the gate's input: bf16
    assert np.abs(y - y64).max() <= (2.0 ** -8 + 1e-5) * np.abs(y64).max()
    w1, w2 = (np.ascontiguousarray(values(m).transpose(0, 2, 1)) for m in W)
    tokens = y.astype(np.float64) if layer.few else values(layer.normed["y8"])
    r = O.moe_layer(y, inp["Wg"], None, inp["W1"], inp["b1"], inp["W2"], inp["b2"], cfg.k, cfg.f, cfg.normalize, cfg.act)
    for key in ("idx", "loc", "counts"):
        assert np.array_equal(layer.routing[key].cpu().numpy(), r[key])
    ref = O.token_outputs_direct(range(T), tokens, r["idx"], r["loc"], r["gate_w"], r["C"], w1, inp["b1"], w2, inp["b2"], cfg.act)
    got = out.double().cpu().numpy()
    off = np.linalg.norm(got - ref) / np.linalg.norm(ref)
    assert off <= (6e-3 if layer.few else 4.5e-2), off


def test_norm_layer8_in_hip_graph(moe):
    """The block captured in a graph: several replays with new inputs, the program's own work in between, each equal to the eager result."""
    cfg = synth.CONFIGS[1].scaled(T=200, M=256, H=384, E=4)
    inp = synth.make_inputs(cfg, seed=9)
    dt = torch.bfloat16
    W = [moe.quantize8(dev_of(inp[n], dt), blocks=True, rows=False, transposed=True)[1] for n in ("W1", "W2")]
    make = lambda T: moe.NormMoELayer8(None, 1e-6, dev_of(inp["Wg"], dt), None, W[0], None, W[1], None, T, cfg.k, cfg.f, cfg.normalize, cfg.act)   # noqa: E731
    for T in (200, 16):
        layer, eager = make(T), make(T)
        x, res = torch.zeros((T, 256), dtype=dt, device="cuda"), torch.zeros((T, 256), dtype=dt, device="cuda")
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            layer.forward(x, res)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            layer.forward(x, res)
        for i in range(4):
            x.normal_()
            res.normal_()
            graph.replay()
            torch.cuda.synchronize()
            want, h = eager.forward(x, res)
            assert torch.equal(layer.out, want) and torch.equal(layer.normed["h"], h)


def test_refusals(moe):
    q, _ = moe.quantize8(torch.zeros((2, 16, 128), device="cuda"))
    w, _ = moe.quantize8(torch.zeros((2, 16, 128), device="cuda"), blocks=True)
    assert moe.matmul8(q, w).shape == (2, 16, 16)
    with pytest.raises(ValueError):
        moe.matmul8(w, q)                                          # A needs an exponent for each row
    with pytest.raises(ValueError):
        moe.matmul8(q, moe.Block8(w.q, w.s, 100, False))
    with pytest.raises(ValueError):
        moe.matmul8(q, moe.Block8(w.q.view(torch.uint8), w.s, 128, True))
    with pytest.raises(ValueError):
        moe.matmul8(q, w, counts=torch.zeros(2, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        moe.quantize8(torch.zeros((128, 16), device="cuda").t())
    with pytest.raises(moe.MoEError):
        moe.quantize8(torch.zeros((4, 12), device="cuda"))
    with pytest.raises(ValueError):
        moe.expert_ffn8(q, w, None, w, None, 0)                    # W2 must be [E,M,H]


def test_refuses_outputs_of_other_shapes(moe):
    x, w = torch.ones((4, 256), device="cuda"), torch.ones(256, device="cuda")
    out = moe.rms_norm(x, w, 1e-6, residual=x, want_8=True)
    wide = moe.rms_norm(torch.ones((4, 512), device="cuda"), None, 1e-6, want_8=True)
    for key, bad in [("h", x[:2]), ("y", x.bfloat16()), ("y8", wide["y8"])]:
        with pytest.raises(ValueError):
            moe.rms_norm(x, w, 1e-6, residual=x, out={**out, key: bad})
    grads = moe.rms_norm_backward(x, x, w, 1e-6)
    for key, bad in [("dx", x[:2]), ("dweight", w[:8])]:
        with pytest.raises(ValueError):
            moe.rms_norm_backward(x, x, w, 1e-6, out={**grads, key: bad})
    A, B_ = moe.quantize8(torch.ones((1, 8, 128), device="cuda"))[0], moe.quantize8(torch.ones((1, 16, 128), device="cuda"))[0]
    with pytest.raises(ValueError):
        moe.matmul8(A, B_, out=torch.empty((1, 8, 8), device="cuda"))


@pytest.mark.parametrize("counts", [None, [0, 5, 40, 900]])
def test_linear8_is_its_pieces(moe, counts):
    """The training pass is the quantisations and products that a caller could make one by one, bit for bit; either gradient alone is the same."""
    E, C, K, N = 4, 300, 200, 328
    g = torch.Generator(device="cuda").manual_seed(3)
    x, W, dy = (torch.randn(s, generator=g, device="cuda").bfloat16() for s in ((E, C, K), (E, K, N), (E, C, N)))
    n = None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda")
    y, kept = moe.expert_linear8_train(x, W, counts=n)
    dx, dW = moe.expert_linear8_backward(dy, kept)
    x8, xt8 = moe.quantize8(x, transposed=True, counts=n)
    W8, Wt8 = moe.quantize8(W, blocks=True, transposed=True)
    dy8, dyt8 = moe.quantize8(dy, transposed=True, counts=n)
    assert torch.equal(y, moe.matmul8(x8, Wt8, counts=n)) and torch.equal(dx, moe.matmul8(dy8, W8, counts=n)) and torch.equal(dW, moe.matmul8(xt8, dyt8, k_counts=n))
    for alone in (0, 1):
        out = [torch.full_like(dx, 7), torch.full_like(dW, 7)]
        p = [o.data_ptr() if i == alone else None for i, o in enumerate(out)]
        st = moe.lib().moe_expert_linear8_backward(dy.data_ptr(), moe.BF16, None if n is None else n.data_ptr(), E, C, K, N, kept.state.data_ptr(), kept.state.numel(), *p, moe._stream())
        assert st == moe.OK and torch.equal(out[alone], (dx, dW)[alone]) and (out[1 - alone] == 7).all()
    with pytest.raises(ValueError):
        moe.expert_linear8_backward(dy[:, :8], kept)
    with pytest.raises(ValueError):
        moe.expert_linear8_train(x, W[:, :8])


def test_linear8_in_hip_graph(moe):
    E, C, K, N = 3, 130, 136, 264
    x, W, dy = torch.randn((E, C, K), device="cuda"), torch.randn((E, K, N), device="cuda"), torch.randn((E, C, N), device="cuda")
    counts = torch.tensor([130, 0, 17], dtype=torch.int32, device="cuda")

    def step():
        y, kept = moe.expert_linear8_train(x, W, counts=counts)
        return (y, *moe.expert_linear8_backward(dy, kept))
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for i in range(3):
        x.normal_()
        counts.copy_(torch.tensor([17 * i, 130, 129 - i], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(captured, step()):
            assert torch.equal(a, b)
