"""Products of experts' rows that lie one behind the other, dense projections, dropout, the rows of a router's choices and their combine, against the 64-bit reference.

Tolerances.  A product's sum over K is a chain of matrix instructions.  bf16 operands: 32 exact products each (16 in the 32-row form, which has twice as many instructions), added up with at most an ulp of
the partial sum, 2^-23, each, then one addition of 2^-24 to the chain: (32 * 2^-23 + K / 16 * 2^-24) of the sum of the magnitudes S.  fp32 operands: two products an instruction, each
rounded: K * 2^-24 of S, and four parts' sums more where the reduction is split.  An activation's slope is at most 1.13; its own error is 5e-5 of the value for bf16 results (GeLU's fit; SiLU 2e-6 + |v| 2^-23 of the exponential's
argument), 16 roundings of fp32 for fp32 results, whose erfc is near 0 by way of its argument's rounding: |v| 2^-23 of the exponent v^2 / 2 more.  Each result is rounded once, half a step: 2^-8 or 2^-24 of it.
Gradients go by the stored pre-activations.  dp is rounded to the storage type, so every term of a sum may be off by 2^-8 (2^-24) and the derivative's error, 2e-5 absolute for bf16, 16 * 2^-24 for fp32 on top of the
exponent's; R rows are added like K products, in chunks for db.
"""
import numpy as np
import pytest
import torch

from oracle import rows_oracle as O

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
HALF = {BF: 2.0 ** -8, F32: 2.0 ** -24}
ACT = {"none": -1, "relu": 0, "gelu": 1, "silu": 2}


@pytest.fixture(scope="module")
def moe():
    assert torch.cuda.is_available(), "these tests need a GPU"
    from paper_2206_03382_amd import moe as m
    m.lib()
    return m


def draw(rng, shape, dtype, scale=1.0):
    t = torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).to(dtype)
    return t.cuda(), t.double().numpy()


def up(t):
    return t.double().cpu().numpy()


def assert_within(got, ref, bound, what):
    got = up(got)
    assert got.shape == ref.shape, f"{what}: {got.shape} for {ref.shape}"
    assert np.isfinite(got).all(), f"{what}: non-finite values"
    over = np.abs(got - ref) - bound
    assert over.size == 0 or over.max() <= 0, f"{what}: {np.abs(got - ref).max():.3e} off, {over.max():.3e} beyond the bound"


def sum_error(dtype, K):
    return 32 * 2.0 ** -23 + K / 16 * 2.0 ** -24 if dtype == BF else (K + 8) * 2.0 ** -24


def act_error(dtype, act, v, y):
    """Of the activation's own evaluation at v."""
    if act in ("none", "relu"):
        return 0.0 * np.abs(y)
    if dtype == BF:
        return np.abs(y) * (5e-5 + np.abs(v) * 2.0 ** -22)
    return np.abs(y) * (16 + v * v + 2 * np.abs(v)) * 2.0 ** -24 + 2.0 ** -126


def grad_error(dtype, act, v):
    if act in ("none", "relu"):
        return 0.0 * v
    return 2e-5 + 0.0 * v if dtype == BF else 32 * 2.0 ** -24 + 0.0 * v


def fills_of(kind, E, R, rng):
    if kind == "even":
        f = np.full(E, R // E)
        f[:R % E] += 1
    elif kind == "one":                                             # everything at one expert
        f = np.zeros(E, dtype=int)
        f[E // 2] = R
    else:                                                           # most at the first, some without any
        w = rng.random(E) ** 4
        w[rng.integers(0, E, max(1, E // 4))] = 0
        w[0] = 2.0
        f = np.floor(w / w.sum() * R).astype(int)
        f[0] += R - f.sum()
    return f


# (rows, experts, K, N, fills, rows of memory behind the last expert's): every tile and both sides of its edges
PRODUCTS = [
    (1, 1, 8, 8, "even", 0), (1, 3, 64, 256, "one", 3), (2, 4, 8, 2056, "even", 0), (5, 2, 264, 72, "skewed", 7), (16, 8, 1024, 512, "even", 0),
    (17, 5, 328, 1000, "skewed", 1), (33, 3, 64, 64, "even", 5), (63, 1, 4096, 256, "even", 0), (64, 4, 128, 128, "skewed", 0), (65, 7, 776, 136, "skewed", 2),
    (127, 2, 512, 264, "even", 0), (129, 16, 2048, 320, "skewed", 3), (255, 2, 192, 768, "even", 0), (257, 3, 256, 512, "skewed", 1),
    (513, 2, 320, 1024, "one", 9), (700, 9, 1000, 776, "skewed", 4), (1111, 17, 64, 256, "skewed", 13), (2048, 4, 512, 1024, "even", 0), (4099, 3, 128, 2560, "skewed", 5),
    (6000, 70, 192, 512, "skewed", 0), (5000, 140, 64, 512, "skewed", 1), (30000, 2, 64, 256, "skewed", 0), (20000, 4, 256, 512, "skewed", 0),
    (1, 3, 1024, 72, "one", 2), (8, 128, 1032, 1024, "even", 0), (16, 5, 1544, 136, "skewed", 2), (11, 2, 2048, 1032, "one", 1),
    (4000, 3, 256, 264, "even", 3), (9001, 5, 136, 128, "skewed", 0), (5000, 40, 1024, 1032, "even", 0), (9000, 3, 264, 520, "skewed", 5), (4097, 5, 256, 1288, "even", 0), (8200, 4, 768, 512, "skewed", 2),                     # shared reductions over rows; many tiles, 125 rows each
]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("R,E,K,N,kind,behind", PRODUCTS)
def test_ragged_product_and_gradients(moe, R, E, K, N, kind, behind, dtype):
    rng = np.random.default_rng(R + 13 * E + K)
    fills = fills_of(kind, E, R, rng)
    offsets = np.concatenate([[0], np.cumsum(fills)]).astype(np.int32)
    act = ["none", "relu", "gelu", "silu"][(R + E) % 4]
    gathered = R % 2 == 1
    tokens = max(1, R // 2)
    A, A64 = draw(rng, (tokens if gathered else R + behind, K), dtype)
    W, W64 = draw(rng, (E, K, N), dtype, 1.0 / np.sqrt(K))
    b, b64 = draw(rng, (E, N), dtype, 0.2)
    gather = gather64 = None
    if gathered:
        gather64 = rng.integers(0, tokens, R + behind)
        gather = torch.from_numpy(gather64.astype(np.int32)).cuda()
    off = torch.from_numpy(offsets).cuda()
    mark = 77.0
    out = torch.full((R + behind, N), mark, dtype=dtype, device="cuda")
    got, pre = moe.ragged_matmul(A, W, off, b, ACT[act], gather=gather, keep_pre=True, out=out)
    assert got is out and (out[R:] == mark).all() and (pre is None) == (act == "none")
    if pre is None:                                                 # the values before no activation
        pre = out.clone()
    v, S = O.product(A64, gather64, W64, b64, offsets)
    y, _ = O.act(v, act)
    e = sum_error(dtype, K) * S
    assert_within(pre[:R], v[:R], (e + HALF[dtype] * np.abs(v))[:R], "pre")
    assert_within(out[:R], y[:R], (1.13 * e + act_error(dtype, act, v, y) + HALF[dtype] * np.abs(y))[:R], "out")
    again = moe.ragged_matmul(A, W, off, b, ACT[act], gather=gather)
    assert torch.equal(again[:R], out[:R])
    plain = moe.ragged_matmul(A, W, off, None, gather=gather)
    v0, S0 = O.product(A64, gather64, W64, None, offsets)
    assert_within(plain[:R], v0[:R], (sum_error(dtype, K) * S0 + HALF[dtype] * np.abs(v0))[:R], "without bias and activation")

    # gradients, of the stored pre-activations; memory behind the last expert's rows may hold anything
    dy, dy64 = draw(rng, (R + behind, N), dtype)
    if behind:
        dy[R:], dy64[R:] = float("nan"), 0.0
        pre[R:] = float("nan")
        if gathered:
            gather[R:] = -1
    p64 = up(pre)
    p64[R:] = 0.0
    _, slope = O.act(p64, act)
    d = dy64 * slope
    dx, dW, db = O.product_backward(d, A64, gather64, W64, offsets)
    off_d = np.abs(dy64) * grad_error(dtype, act, p64) + np.abs(d) * (HALF[dtype] if act != "none" else 0.0)    # of a term of the sums
    size = np.abs(d) + off_d
    sx, sW, sb = O.product_backward(size, np.abs(A64), gather64, np.abs(W64), offsets)
    ex, eW, eb = O.product_backward(off_d, np.abs(A64), gather64, np.abs(W64), offsets)
    g = moe.ragged_matmul_backward(dy, A, W, off, ACT[act], None if act == "none" else pre, gather=gather)
    assert_within(g["dx"][:R], dx[:R], (ex + sum_error(dtype, N) * sx + HALF[dtype] * np.abs(dx))[:R], "dx")
    longest = int(fills.max())
    assert_within(g["dW"], dW, eW + sum_error(dtype, longest) * sW + HALF[dtype] * np.abs(dW), "dW")
    assert_within(g["db"], db, eb + (longest / 8 + 96) * 2.0 ** -24 * sb + HALF[dtype] * np.abs(db), "db")
    for want in ("dx", "dW", "db"):                                  # each by itself, the same bits
        only = moe.ragged_matmul_backward(dy, A, W, off, ACT[act], None if act == "none" else pre, gather=gather, **{f"want_{w}": w == want for w in ("dx", "dW", "db")})
        rows = slice(0, R) if want == "dx" else slice(None)
        assert torch.equal(only[want][rows], g[want][rows]) and sum(t is not None for t in only.values()) == 1


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("kind", ["one", "even", "skewed", "gaps"])
@pytest.mark.parametrize("R,E,N", [(1, 300, 64), (8, 40, 264), (9, 40, 264), (128, 8, 72), (128, 9, 72), (129, 2, 520), (257, 200, 64), (513, 5, 264), (2049, 33, 64), (12300, 70, 64), (50000, 3, 1288)])
def test_bias_gradient_of_experts_that_share_or_cross_chunks(moe, R, E, N, kind, dtype):
    """A few rows and many experts, a hot expert among small ones, experts without rows in front, between and behind; rows behind the last one are not read."""
    rng = np.random.default_rng(R + 7 * E + N)
    share = {"one": np.eye(1, E, E // 2)[0], "even": np.ones(E), "skewed": 1.0 / np.arange(1, E + 1) ** 2, "gaps": (np.arange(E) % 3 == 1) + 1e-9}[kind]
    fills = np.bincount(rng.choice(E, R, p=share / share.sum()), minlength=E)
    if kind == "even" and R >= E:
        fills = np.full(E, R // E)                                   # borders on those of the chunks, where these divide
    offsets = np.concatenate([[0], np.cumsum(fills)]).astype(np.int32)
    used, behind = int(offsets[-1]), 70
    off = torch.from_numpy(offsets).cuda()
    dy, dy64 = draw(rng, (used + behind, N), dtype)
    pre, p64 = draw(rng, (used + behind, N), dtype)
    dy[used:], pre[used:] = float("nan"), float("nan")
    A = torch.zeros(used + behind, 64, dtype=dtype, device="cuda")
    W = torch.zeros(E, 64, N, dtype=dtype, device="cuda")
    d64 = dy64[:used] * (p64[:used] > 0)                             # exact in the storage type
    ids = np.repeat(np.arange(E), fills)
    want, size = np.zeros((E, N)), np.zeros((E, N))
    for e in np.unique(ids):
        want[e], size[e] = d64[offsets[e]:offsets[e + 1]].sum(0), np.abs(d64[offsets[e]:offsets[e + 1]]).sum(0)
    got = moe.ragged_matmul_backward(dy, A, W, off, ACT["relu"], pre, want_dx=False, want_dW=False)["db"]
    assert_within(got, want, (int(fills.max()) / 8 + 96) * 2.0 ** -24 * size + HALF[dtype] * np.abs(want), "db")
    again = moe.ragged_matmul_backward(dy, A, W, off, ACT["relu"], pre, want_dx=False, want_dW=False)["db"]
    assert torch.equal(got, again)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
@pytest.mark.parametrize("R,E,K,N", [(5, 2, 72, 64), (130, 4, 256, 512), (700, 3, 328, 200), (3000, 4, 512, 256), (9001, 3, 520, 264), (8000, 3, 512, 776)])
def test_gradient_of_the_projection_before(moe, R, E, K, N, act, dtype):
    """dx times the derivative of the activation that made x, in one rounding."""
    rng = np.random.default_rng(R + K)
    offsets = np.concatenate([[0], np.cumsum(fills_of("skewed", E, R, rng))]).astype(np.int32)
    dy, dy64 = draw(rng, (R, N), dtype)
    x, _ = draw(rng, (R, K), dtype)
    xp, xp64 = draw(rng, (R, K), dtype, 1.5)
    xp[0] *= 0                                                      # ReLU'(0) = 0
    xp64[0] = 0
    W, W64 = draw(rng, (E, K, N), dtype, 1.0 / np.sqrt(K))
    off = torch.from_numpy(offsets).cuda()
    g = moe.ragged_matmul_backward(dy, x, W, off, x_act=ACT[act], x_pre=xp, want_dW=False, want_db=False)
    dx, _, _ = O.product_backward(dy64, xp64, None, W64, offsets)
    S, _, _ = O.product_backward(np.abs(dy64), xp64, None, np.abs(W64), offsets)
    _, slope = O.act(xp64, act)
    ref = dx * slope
    assert_within(g["dx"], ref, 1.13 * sum_error(dtype, N) * S + (np.abs(dx) + sum_error(dtype, N) * S) * grad_error(dtype, act, xp64) + HALF[dtype] * (1 + 2.0 ** -7) * np.abs(ref) + 2.0 ** -120, "dx")


LINEAR = [(1, 8, 8), (1, 4096, 264), (1, 264, 4096), (2, 64, 64), (3, 1000, 776), (8, 2048, 512), (15, 72, 1032), (16, 1024, 1024), (17, 512, 256), (31, 776, 1544), (33, 4096, 136), (64, 256, 2048), (65, 64, 64),
          (100, 1024, 4096), (127, 128, 256), (256, 320, 512), (300, 776, 264), (1000, 512, 1024), (2049, 192, 256), (4100, 1024, 1280), (9000, 64, 512),
          (1, 4096, 4096), (19, 2056, 1032), (50, 4096, 2056), (110, 2568, 4096), (290, 4096, 1000), (8193, 520, 264), (20001, 264, 256), (10000, 512, 776)]          # few rows, the reduction shared by blocks


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,K,N", LINEAR)
def test_linear_and_gradients(moe, T, K, N, dtype):
    rng = np.random.default_rng(T + K + 3 * N)
    act = ["none", "relu", "gelu", "silu"][(T + K // 8) % 4]
    x, x64 = draw(rng, (T, K), dtype)
    W, W64 = draw(rng, (K, N), dtype, 1.0 / np.sqrt(K))
    b, b64 = draw(rng, (N,), dtype, 0.2)
    res, res64 = draw(rng, (T, N), dtype, 2.0)
    offsets = [0, T]
    v, S = O.product(x64, None, W64[None], b64[None], offsets)
    y, _ = O.act(v, act)
    e = sum_error(dtype, K) * S
    bound = 1.13 * e + act_error(dtype, act, v, y) + 2.0 ** -23 * np.abs(res64)
    got, pre = moe.linear(x, W, b, ACT[act], residual=res, keep_pre=True)
    assert (pre is None) == (act == "none")
    if pre is not None:
        assert_within(pre, v, e + HALF[dtype] * np.abs(v), "pre")
    assert_within(got, y + res64, bound + HALF[dtype] * np.abs(y + res64), "out")
    assert torch.equal(moe.linear(x, W, b, ACT[act], residual=res), got)
    assert_within(moe.linear(x, W, b, ACT[act]), y, bound + HALF[dtype] * np.abs(y), "without a residual")
    v0, S0 = O.product(x64, None, W64[None], None, offsets)
    assert_within(moe.linear(x, W, residual=res), v0 + res64, sum_error(dtype, K) * S0 + 2.0 ** -23 * np.abs(res64) + HALF[dtype] * np.abs(v0 + res64), "without bias and activation")
    own = res.clone()                                               # onto the residual itself
    assert moe.linear(x, W, b, ACT[act], residual=own, out=own) is own and torch.equal(own, got)

    dy, dy64 = draw(rng, (T, N), dtype)
    p64 = v if pre is None else up(pre)
    _, slope = O.act(p64, act)
    d = dy64 * slope
    dx, dW, db = O.product_backward(d, x64, None, W64[None], offsets)
    off_d = np.abs(dy64) * grad_error(dtype, act, p64) + np.abs(d) * (HALF[dtype] if act != "none" else 0.0)
    size = np.abs(d) + off_d
    sx, sW, sb = O.product_backward(size, np.abs(x64), None, np.abs(W64)[None], offsets)
    ex, eW, eb = O.product_backward(off_d, np.abs(x64), None, np.abs(W64)[None], offsets)
    g = moe.linear_backward(dy, x, W, ACT[act], None if act == "none" else pre)
    assert_within(g["dx"], dx, ex + sum_error(dtype, N) * sx + HALF[dtype] * np.abs(dx), "dx")
    assert_within(g["dW"], dW[0], (eW + sum_error(dtype, T) * sW)[0] + HALF[dtype] * np.abs(dW[0]), "dW")
    assert_within(g["db"], db[0], (eb + (T / 8 + 96) * 2.0 ** -24 * sb)[0] + HALF[dtype] * np.abs(db[0]), "db")


def test_gradients_against_differences(moe):
    """The loss <out, dy> of a projection with activation along random directions of x, W and bias, by central differences in 64 bits: their error is step^2 times a third derivative."""
    rng = np.random.default_rng(5)
    T, K, N, step = 9, 40, 24, 1e-5
    x, x64 = draw(rng, (T, K), F32)
    W, W64 = draw(rng, (K, N), F32, 0.3)
    b, b64 = draw(rng, (N,), F32)
    dy, dy64 = draw(rng, (T, N), F32)
    for act in ("gelu", "silu"):
        _, pre = moe.linear(x, W, b, ACT[act], keep_pre=True)
        g = moe.linear_backward(dy, x, W, ACT[act], pre)
        for name, at in (("dx", 0), ("dW", 1), ("db", 2)):
            args = [x64, W64, b64]
            way = rng.standard_normal(args[at].shape)

            def loss(s):
                moved = [a + s * way if i == at else a for i, a in enumerate(args)]
                return float((O.act(moved[0] @ moved[1] + moved[2], act)[0] * dy64).sum())

            slope = (loss(step) - loss(-step)) / (2 * step)
            mine = float((up(g[name]) * way).sum())
            # fp32 gradients: 2^-20 of the magnitudes of the terms; differences: 1e-10 of them and 1e-11 / step of the loss's own rounding
            terms = float((np.abs(up(g[name])) * np.abs(way)).sum()) + float(np.abs(dy64).sum())
            assert abs(slope - mine) <= (2.0 ** -18 + 1e-6) * terms, (act, name, slope, mine)


# ---- dropout ---------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,M,p", [(1, 8, 0.5), (1, 8, 0.0), (3, 264, 0.1), (16, 1024, 0.25), (7, 776, 1.0), (5, 40, 2.0 ** -17), (33, 520, 0.999)])
def test_dropout(moe, T, M, p, dtype):
    rng = np.random.default_rng(T + M)
    x, x64 = draw(rng, (T, M), dtype)
    res, res64 = draw(rng, (T, M), dtype, 2.0)
    for seed, offset in ((0, 0), (0x123456789ABCDEF0, 0x0FEDCBA987654321), (-1, -(2 ** 63))):
        numbers = torch.tensor([seed, offset], dtype=torch.int64, device="cuda")
        m = O.multiplier(T * M, p, seed & (2 ** 64 - 1), offset & (2 ** 64 - 1)).reshape(T, M)
        ref = x64 * m
        got = moe.dropout(x, p, numbers)
        assert_within(got, ref, (HALF[dtype] + 2.0 ** -23) * np.abs(ref), "out")
        assert ((up(got) == 0) == ((m == 0) | (x64 == 0))).all()
        ref = ref + res64
        assert_within(moe.dropout(x, p, numbers, residual=res), ref, 2.0 ** -22 * (np.abs(x64 * m) + np.abs(res64)) + HALF[dtype] * np.abs(ref), "with the residual")
        for target in ("x", "residual"):                            # in place
            a, r = x.clone(), res.clone()
            into = a if target == "x" else r
            assert moe.dropout(a, p, numbers, residual=r, out=into) is into
            assert torch.equal(into, moe.dropout(x, p, numbers, residual=res))


def test_dropped_infinities_are_zero(moe):
    x = torch.full((4, 64), float("inf"), device="cuda")
    x[2] = float("nan")
    numbers = torch.tensor([3, 4], dtype=torch.int64, device="cuda")
    m = O.multiplier(256, 0.5, 3, 4).reshape(4, 64)
    got = moe.dropout(x, 0.5, numbers, residual=torch.ones_like(x)).cpu().numpy()
    assert (got[m == 0] == 1).all() and not np.isfinite(got[m > 0]).any() and (m == 0).any() and (m > 0).any()


def test_dropout_of_many_groups(moe):
    """More groups than a grid has threads (2^28) and element numbers past 32 bits, the share that is kept, and another offset's mask: of n elements, within five standard deviations,
    5 sqrt(p (1 - p) / n)."""
    n, p = (1 << 31) + (1 << 14), 0.125
    x = torch.ones((n // 1024, 1024), dtype=BF, device="cuda")
    a = moe.dropout(x, p, torch.tensor([9, 0], dtype=torch.int64, device="cuda")) != 0
    b = moe.dropout(x, p, torch.tensor([9, 1], dtype=torch.int64, device="cuda")) != 0
    for kept, of in ((a.sum().item(), 1 - p), ((a & b).sum().item(), (1 - p) ** 2)):
        assert abs(kept / n - of) <= 5 * np.sqrt(of * (1 - of) / n)
    flat = a.view(-1)
    for g in (n // 8 - 1, (1 << 28) + 3, 12345678):                 # groups anywhere have the reference's bits
        w = O.philox((9, 0), (g, 0, 0, 0))
        assert flat[8 * g:8 * g + 8].tolist() == [(w[i // 2] >> 16 * (i % 2) & 0xFFFF) >= 8192 for i in range(8)]


# ---- rows and combine ------------------------------------------------------------------------------------------------------

def route(rng, T, E, k):
    idx = np.argsort(rng.random((T, E)) - 0.3 * (np.arange(E) == 0), axis=1)[:, :k].astype(np.int32)
    loc, seen = np.zeros((T, k), dtype=np.int32), np.zeros(E, dtype=np.int32)
    for j in range(k):
        for t in range(T):
            loc[t, j] = seen[idx[t, j]]
            seen[idx[t, j]] += 1
    return idx, loc, seen


ROUTES = [(1, 1, 1, 8), (1, 8, 8, 64), (5, 3, 2, 264), (64, 4, 1, 1032), (100, 128, 8, 512), (333, 17, 3, 776), (1000, 512, 9, 72), (700, 300, 16, 136), (2049, 6, 4, 4096)]


@pytest.mark.parametrize("T,E,k,M", ROUTES)
def test_ragged_rows(moe, T, E, k, M):
    rng = np.random.default_rng(T + E)
    idx, loc, counts = route(rng, T, E, k)
    t = [torch.from_numpy(a).cuda() for a in (idx, loc, counts)]
    for C in (0, 1, max(1, T * k // (2 * E))):
        got = moe.ragged_rows(*t, C=C)
        for mine, ref in zip(got, O.rows(idx, loc, counts, C)):
            assert np.array_equal(mine.cpu().numpy(), ref)
    # choices of padding tokens, marked by an expert that does not exist: the others keep their rows
    idx[T // 2:], loc2 = -1, loc
    ref = O.rows(idx, loc2, counts, 0)
    got = moe.ragged_rows(torch.from_numpy(idx).cuda(), t[1], t[2])
    assert np.array_equal(got.row_of.cpu().numpy(), ref[2]) and np.array_equal(got.offsets.cpu().numpy(), ref[0])
    # the routers' own outputs
    logits = torch.from_numpy(rng.standard_normal((T, E)).astype(np.float32)).cuda()
    r = moe.gate_topk(logits, k, 1, 0)
    got = moe.ragged_rows(r["idx"], r["loc"], r["counts"])
    for mine, ref in zip(got, O.rows(*(r[n].cpu().numpy() for n in ("idx", "loc", "counts")), 0)):
        assert np.array_equal(mine.cpu().numpy(), ref)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,E,k,M", ROUTES)
def test_ragged_combine(moe, T, E, k, M, dtype):
    rng = np.random.default_rng(T + M)
    idx, loc, counts = route(rng, T, E, k)
    C = 0 if T % 2 else max(1, T * k // (2 * E))
    offsets, _, row_of64 = O.rows(idx, loc, counts, C)
    R = int(offsets[-1]) + 2
    Y, Y64 = draw(rng, (R, M), dtype)
    res, res64 = draw(rng, (T, M), dtype, 2.0)
    dout, dout64 = draw(rng, (T, M), dtype)
    w, w64 = draw(rng, (T, k), F32)
    row_of = torch.from_numpy(row_of64).cuda()
    numbers = torch.tensor([T, M], dtype=torch.int64, device="cuda")
    few = T * M <= 60000                                            # the reference generator is a loop in Python
    for drop in (None, (0.2, numbers)) if few else (None,):
        m = np.ones((T, M)) if drop is None else O.multiplier(T * M, 0.2, T, M).reshape(T, M)
        for weights, weights64 in ((w, w64), (None, None)):
            total, size = O.combine(Y64, row_of64, weights64)
            # k products and sums in fp32, the scale and the residual's addition
            bound = (k + 3) * 2.0 ** -24 * size * m
            ref = total * m
            assert_within(moe.ragged_combine(Y, row_of, weights, dropout=drop), ref, bound + HALF[dtype] * np.abs(ref), "out")
            ref = ref + res64
            got = moe.ragged_combine(Y, row_of, weights, residual=res, dropout=drop)
            assert_within(got, ref, bound + 2.0 ** -23 * (np.abs(res64) + size * m) + HALF[dtype] * np.abs(ref), "with the residual")
            own = res.clone()
            assert torch.equal(moe.ragged_combine(Y, row_of, weights, residual=own, dropout=drop, out=own), got)
            dY = torch.full((R, M), 55.0, dtype=dtype, device="cuda")
            _, dw = moe.ragged_combine_backward(dout, Y, row_of, weights, dropout=drop, dY=dY)
            d = dout64 * m
            rY, rw, sw = np.full((R, M), 55.0), np.zeros((T, k)), np.zeros((T, k))
            for t in range(T):
                for j in range(k):
                    r = row_of64[t, j]
                    if r >= 0:
                        rY[r] = (1.0 if weights is None else w64[t, j]) * d[t]
                        rw[t, j], sw[t, j] = d[t] @ Y64[r], np.abs(d[t]) @ np.abs(Y64[r])
            assert_within(dY, rY, (HALF[dtype] + 3 * 2.0 ** -24) * np.abs(rY), "dY")       # rows without a choice keep what they held
            # a lane's share of the products, six additions over the lanes, four waves
            assert_within(dw, rw, (M / 64 + 24) * 2.0 ** -24 * sw, "dgate_w")


def test_combine_leaves_out_what_is_not_there(moe):
    """Rows out of range, both ways, and what lies in rows that no choice has."""
    Y = torch.full((4, 64), float("nan"), device="cuda")
    Y[1] = 2.0
    row_of = torch.tensor([[1, -1], [-1, -5], [4, 1], [2 ** 31 - 1, 1]], dtype=torch.int32, device="cuda")
    w = torch.tensor([[1.0, float("nan")], [float("inf"), 1.0], [float("nan"), 0.5], [1.0, 2.0]], device="cuda")
    out = moe.ragged_combine(Y, row_of, w)
    assert out[:, 0].tolist() == [2.0, 0.0, 1.0, 4.0]
    dY, dw = moe.ragged_combine_backward(torch.ones((4, 64), device="cuda"), Y, row_of[:3].contiguous().repeat(2, 1)[:4], w, dY=torch.zeros_like(Y))
    assert torch.isfinite(dY[0]).all() and (dY[2:] == 0).all() and dw[1].tolist() == [0.0, 0.0] and dw[0].tolist() == [128.0, 0.0]


def test_offsets_that_lie_and_tokens_out_of_range(moe):
    """Descending offsets and offsets beyond the rows end at the rows that exist, tokens out of range read token 0: results are whatever they are, in bounds."""
    rng = np.random.default_rng(0)
    x, x64 = draw(rng, (50, 64), BF)
    W, W64 = draw(rng, (3, 64, 256), BF, 0.125)
    guard = torch.full((64, 256), 3.0, dtype=BF, device="cuda")
    moe.ragged_matmul(x, W, torch.tensor([0, 70, 20, 1000], dtype=torch.int32, device="cuda"), out=guard[:50])
    assert (guard[50:] == 3.0).all()
    moe.ragged_matmul(x, W, torch.tensor([-5, -3, 60, -1], dtype=torch.int32, device="cuda"), out=guard[:50])
    assert (guard[50:] == 3.0).all()
    gather = torch.tensor([-1, 50, 2 ** 31 - 1, -2 ** 31, 7], dtype=torch.int32, device="cuda")
    got = moe.ragged_matmul(x, W, torch.tensor([0, 5, 5, 5], dtype=torch.int32, device="cuda"), gather=gather)
    v, S = O.product(x64, np.array([0, 0, 0, 0, 7]), W64, None, [0, 5, 5, 5])
    assert_within(got, v, sum_error(BF, 64) * S + HALF[BF] * np.abs(v), "out")


@pytest.mark.parametrize("dtype", [BF, F32])
def test_in_a_graph_and_on_another_stream(moe, dtype):
    """The whole run of the operators captured once and replayed on other inputs, seeds and routings, with eager work in between; and on a stream of its own."""
    rng = np.random.default_rng(1)
    T, E, k, M, H = 70, 5, 2, 128, 256
    x, _ = draw(rng, (T, M), dtype)
    W1, _ = draw(rng, (E, M, H), dtype, 0.1)
    W2, _ = draw(rng, (E, H, M), dtype, 0.1)
    b1, _ = draw(rng, (E, H), dtype)
    dout, _ = draw(rng, (T, M), dtype)
    numbers = torch.tensor([1, 2], dtype=torch.int64, device="cuda")
    idx, loc, counts = (torch.from_numpy(a).cuda() for a in route(rng, T, E, k))
    w = torch.rand((T, k), device="cuda")

    def step():
        rows = moe.ragged_rows(idx, loc, counts)
        hidden, pre = moe.ragged_matmul(x, W1, rows.offsets, b1, moe.ACT_GELU, gather=rows.row_src, keep_pre=True)
        Y = moe.ragged_matmul(hidden, W2, rows.offsets)
        out = moe.ragged_combine(Y, rows.row_of, w, residual=x, dropout=(0.25, numbers))
        dY, dw = moe.ragged_combine_backward(dout, Y, rows.row_of, w, dropout=(0.25, numbers))
        g2 = moe.ragged_matmul_backward(dY, hidden, W2, rows.offsets, x_act=moe.ACT_GELU, x_pre=pre)
        g1 = moe.ragged_matmul_backward(g2["dx"], x, W1, rows.offsets, gather=rows.row_src)
        dx = moe.ragged_combine(g1["dx"], rows.row_of, None, residual=dout)
        return [out, dw, dx, g1["dW"], g1["db"], g2["dW"], g2["db"], moe.dropout(dout, 0.25, numbers)]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        first = step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, step()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for i in range(4):
        numbers += i
        x.mul_(1.25)
        new = route(np.random.default_rng(i), T, E, k)
        for t, a in zip((idx, loc, counts), new):
            t.copy_(torch.from_numpy(a))
        graph.replay()
        torch.cuda.synchronize()
        eager = step()
        assert all(torch.equal(a, b) for a, b in zip(captured, eager)), f"replay {i}"


# Sizes whose launches share a reduction through a workspace, forward (few rows, many columns) and backward (many rows, few columns), and those of the tiles of one stage
SHARED = [(40, 4096, 256), (6000, 256, 264), (3000, 264, 776)]


def a_step(moe, x, W, b, res, dy, act):
    out, pre = moe.linear(x, W, b, act, residual=res, keep_pre=True)
    g = moe.linear_backward(dy, x, W, act, pre)
    return [out, pre, g["dx"], g["dW"], g["db"]]


@pytest.mark.parametrize("dtype", [BF, F32])
def test_two_graphs_and_eager_calls_in_between(moe, dtype):
    """Two captured steps, replayed in turn on inputs that change, with eager steps and a synchronization in between: every replay has the eager result's bits."""
    rng = np.random.default_rng(9)
    for T, K, N in SHARED:
        sets = [[draw(rng, s, dtype)[0] for s in ((T, K), (K, N), (N,), (T, N), (T, N))] for _ in range(2)]
        for s in sets:
            a_step(moe, *s, moe.ACT_SILU)
        torch.cuda.synchronize()
        graphs = []
        for s in sets:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                graphs.append((graph, s, a_step(moe, *s, moe.ACT_SILU)))
        for i in range(3):
            for graph, s, _ in graphs:
                s[0].mul_(1.0 + 0.125 * i)
                graph.replay()
            torch.cuda.synchronize()
            for j, (_, s, captured) in enumerate(graphs):
                assert all(torch.equal(a, b) for a, b in zip(captured, a_step(moe, *s, moe.ACT_SILU))), f"{T} x {K} x {N}: graph {j}, replay {i}"


@pytest.mark.parametrize("dtype", [BF, F32])
def test_two_streams_at_a_time(moe, dtype):
    """Steps on two streams at once, several of each, have the bits of one by itself."""
    rng = np.random.default_rng(10)
    for T, K, N in SHARED:
        sets = [[draw(rng, s, dtype)[0] for s in ((T, K), (K, N), (N,), (T, N), (T, N))] for _ in range(2)]
        alone = [a_step(moe, *s, moe.ACT_GELU) for s in sets]
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in sets]
        results = [[], []]
        for _ in range(4):
            for s, stream, r in zip(sets, streams, results):
                with torch.cuda.stream(stream):
                    r.append(a_step(moe, *s, moe.ACT_GELU))
        torch.cuda.synchronize()
        for want, r in zip(alone, results):
            assert all(torch.equal(a, b) for got in r for a, b in zip(got, want)), f"{T} x {K} x {N}"


@pytest.mark.parametrize("T", [1, 300, 9000])
def test_nan_and_infinity_stay_in_their_rows(moe, T):
    """A NaN or an infinity in one row of x reaches that row of the result and no other, at edges of tiles; ReLU keeps a NaN."""
    K, N = 328, 264
    x = torch.zeros((T, K), dtype=BF, device="cuda")
    W = torch.ones((K, N), dtype=BF, device="cuda")
    x[T - 1, K - 1] = float("nan")
    x[T // 2, 0] = float("inf") if T > 1 else float("nan")
    for act in (moe.ACT_NONE, moe.ACT_RELU, moe.ACT_GELU, moe.ACT_SILU):
        out = moe.linear(x, W, act=act).float()
        assert out[T - 1].isnan().all()
        rest = torch.ones(T, dtype=torch.bool, device="cuda")
        rest[T - 1] = rest[T // 2] = False
        assert (out[rest] == 0).all() and (T == 1 or out[T // 2].isinf().all())
