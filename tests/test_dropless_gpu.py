"""The layer without a capacity, forward and backward, against the 64-bit reference given its routing, and captured into a graph.

Tolerances: every quantity of the reference carries a bound of its error, put together by the rules of the operators' own tests (a product of matrices: the errors of both operands times
the other's magnitudes, and sum_error of the sum of the magnitudes; an activation: 1.13 of its argument's error and its own evaluation; a derivative: the second derivative is
below 1; half a step of every rounding to the storage type).  The routing (idx, loc, gate_w, logits) is the layer's own, taken as exact; the gate's backward makes its probabilities
from those logits again, to 2^-18 of them.  With normalised weights it goes on through all of them, dlogits_e = p_e (dp_e - sum_i dp_i p_i) with dp_j p_j = w_j (dw_j - sum_i w_i dw_i): the sum
over i is zero in exact arithmetic, and in fp32 a rounding of its terms' magnitudes, at most 2 sum_j w_j |dw_j|, which reaches every expert times p_e, the ones that were not chosen as well.
"""
import numpy as np
import pytest
import torch

from oracle import rows_oracle as O
from test_rows_gpu import ACT, BF, F32, HALF, act_error, assert_within, draw, grad_error, moe, sum_error, up   # noqa: F401

pytestmark = pytest.mark.gpu


class Q:
    """Values with a bound of their error."""

    def __init__(self, v, e=0.0):
        self.v, self.e = v, np.zeros_like(v) + e

    def rounded(self, dtype):
        return Q(self.v, self.e + HALF[dtype] * (np.abs(self.v) + self.e))

    @property
    def T(self):
        return Q(self.v.T, self.e.T)

    def __getitem__(self, at):
        return Q(self.v[at], self.e[at])


def mm(a, b, dtype, bias=None):
    size = np.abs(a.v) @ np.abs(b.v)
    e = np.abs(a.v) @ b.e + a.e @ np.abs(b.v) + a.e @ b.e
    v = a.v @ b.v
    if bias is not None:
        v, size = v + bias, size + np.abs(bias)
    return Q(v, e + sum_error(dtype, a.v.shape[1]) * (size + e))


def times(a, b):
    return Q(a.v * b.v, np.abs(a.v) * b.e + a.e * np.abs(b.v) + a.e * b.e)


def activation(v, act, dtype):
    y, slope = O.act(v.v, act)
    return Q(y, 1.13 * v.e + act_error(dtype, act, v.v, y)), Q(slope, v.e + HALF[dtype] * np.abs(v.v) + grad_error(dtype, act, v.v))


def expert(x, W1, b1, W2, b2, act, dtype):
    pre = mm(x, W1, dtype, b1)
    hidden, slope = activation(pre, act, dtype)
    hidden = hidden.rounded(dtype)
    return hidden, slope, mm(hidden, W2, dtype, b2)


def expert_backward(x, W1, W2, hidden, slope, dY, dtype):
    dp = times(mm(dY, W2.T, dtype), slope).rounded(dtype)
    n = x.v.shape[0]
    sums = lambda d: Q(d.v.sum(0), d.e.sum(0) + (n / 8 + 96) * 2.0 ** -24 * (np.abs(d.v) + d.e).sum(0)).rounded(dtype)   # noqa: E731
    return mm(dp, W1.T, dtype), mm(x.T, dp, dtype).rounded(dtype), sums(dp), mm(hidden.T, dY, dtype).rounded(dtype), sums(dY)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,E,k,M,H,act,normalize,p,shared,bias", [
    (1, 4, 2, 64, 72, "gelu", 1, 0.0, False, True), (70, 5, 2, 128, 192, "silu", 1, 0.25, True, False), (33, 8, 8, 264, 136, "gelu", 0, 0.1, True, True),
    (257, 17, 3, 136, 320, "silu", 0, 0.0, False, False), (600, 3, 1, 256, 256, "gelu", 1, 0.5, True, True)])
def test_layer(moe, T, E, k, M, H, act, normalize, p, shared, bias, dtype):   # noqa: F811
    rng = np.random.default_rng(T + E)
    x, x64 = draw(rng, (T, M), dtype)
    res, res64 = draw(rng, (T, M), dtype)
    Wg, Wg64 = draw(rng, (M, E), dtype, 1.0 / np.sqrt(M))
    W1, W1_64 = draw(rng, (E, M, H), dtype, 1.0 / np.sqrt(M))
    W2, W2_64 = draw(rng, (E, H, M), dtype, 1.0 / np.sqrt(H))
    S1, S1_64 = draw(rng, (M, 2 * H), dtype, 1.0 / np.sqrt(M))
    S2, S2_64 = draw(rng, (2 * H, M), dtype, 1.0 / np.sqrt(2 * H))
    b = [draw(rng, shape, dtype, 0.3) if bias else (None, None) for shape in ((E, H), (E, M), (2 * H,), (M,))]
    dout, dout64 = draw(rng, (T, M), dtype)
    gate_bias = torch.from_numpy(rng.standard_normal(E).astype(np.float32)).cuda()
    numbers = torch.tensor([11, T], dtype=torch.int64, device="cuda")
    layer = moe.DroplessLayer(Wg, gate_bias, W1, b[0][0], W2, b[1][0], k, normalize, ACT[act], shared=(S1, b[2][0], S2, b[3][0]) if shared else None)
    drop = (p, numbers) if p else None
    out, kept = layer.forward(x, residual=res, dropout=drop, keep=True)
    assert torch.equal(layer.forward(x, residual=res, dropout=drop), out)
    g = layer.backward(kept, dout)

    idx, w = kept.routing["idx"].cpu().numpy(), up(kept.routing["gate_w"])
    offsets, row_src, row_of = O.rows(idx, kept.routing["loc"].cpu().numpy(), kept.routing["counts"].cpu().numpy(), 0)
    assert offsets[-1] == T * k and (row_of >= 0).all() and (row_src == kept.rows.row_src.cpu().numpy()).all() and (row_of == kept.rows.row_of.cpu().numpy()).all()
    m = O.multiplier(T * M, p, 11, T).reshape(T, M) if p else np.ones((T, M))
    u = 2.0 ** -24
    # forward
    xr = Q(x64[row_src])
    parts = [expert(xr[offsets[e]:offsets[e + 1]], Q(W1_64[e]), b[0][1][e] if bias else None, Q(W2_64[e]), b[1][1][e] if bias else None, act, dtype) for e in range(E)]
    Y = Q(np.concatenate([q[2].v for q in parts]), np.concatenate([q[2].e for q in parts])).rounded(dtype)
    base, sh = Q(res64), None
    if shared:
        sh = expert(Q(x64), Q(S1_64), b[2][1], Q(S2_64), b[3][1], act, dtype)
        base = Q(sh[2].v + res64, sh[2].e + 2 * u * np.abs(res64)).rounded(dtype)
    routed = (w[:, :, None] * Y.v[row_of]).sum(1)
    size = (np.abs(w)[:, :, None] * (np.abs(Y.v) + Y.e)[row_of]).sum(1)
    ref = Q(base.v + m * routed, base.e + m * (np.abs(w)[:, :, None] * Y.e[row_of]).sum(1) + (k + 4) * u * (m * size + np.abs(base.v) + base.e)).rounded(dtype)
    assert_within(out, ref.v, ref.e, "out")

    # backward
    d = Q(dout64 * m, 2 * u * np.abs(dout64 * m))
    dY = Q(np.zeros((T * k, M)))
    flat = row_of.reshape(-1)
    weighted = times(Q(np.repeat(d.v, k, 0), np.repeat(d.e, k, 0)), Q(w.reshape(-1, 1), u * w.reshape(-1, 1)))
    dY.v[flat], dY.e[flat] = weighted.v, weighted.e
    dY = dY.rounded(dtype)
    dw = Q(np.einsum("tm,tjm->tj", d.v, Y.v[row_of]))
    dw.e = np.einsum("tm,tjm->tj", np.abs(d.v), Y.e[row_of]) + np.einsum("tm,tjm->tj", np.abs(d.v) + d.e, (np.abs(Y.v) + Y.e)[row_of]) * (M + 8) * u
    rows_dx = Q(np.zeros((T * k, M)))
    for e in range(E):
        at = slice(offsets[e], offsets[e + 1])
        gx, gW1, gb1, gW2, gb2 = expert_backward(xr[at], Q(W1_64[e]), Q(W2_64[e]), parts[e][0], parts[e][1], dY[at], dtype)
        gx = gx.rounded(dtype)
        rows_dx.v[at], rows_dx.e[at] = gx.v, gx.e
        for name, q in (("dW1", gW1), ("db1", gb1), ("dW2", gW2), ("db2", gb2)):
            assert_within(g[name][e], q.v, q.e, f"{name} of expert {e}")
    dx = Q(rows_dx.v[row_of].sum(1), rows_dx.e[row_of].sum(1))
    size = (np.abs(rows_dx.v) + rows_dx.e)[row_of].sum(1)
    if shared:
        gx, gW1, gb1, gW2, gb2 = expert_backward(Q(x64), Q(S1_64), Q(S2_64), sh[0], sh[1], Q(dout64), dtype)
        gx = gx.rounded(dtype)
        dx, size = Q(dx.v + gx.v, dx.e + gx.e), size + np.abs(gx.v) + gx.e
        for name, q in (("dWs1", gW1), ("dbs1", gb1), ("dWs2", gW2), ("dbs2", gb2)):
            assert_within(g[name], q.v, q.e, name)
    dx = Q(dx.v, dx.e + (k + 2) * u * size).rounded(dtype)
    logits = up(kept.routing["logits"])
    prob = np.exp(logits - logits.max(1, keepdims=True))
    prob /= prob.sum(1, keepdims=True)
    at = np.arange(T)[:, None]
    chosen = np.zeros((T, E))
    chosen[at, idx] = 1.0
    q = prob * chosen / (prob * chosen).sum(1, keepdims=True) if normalize else prob            # dlogits = q (dw - sum of dw q over the choices), dw = 0 elsewhere
    full, full_e = np.zeros((T, E)), np.zeros((T, E))
    full[at, idx], full_e[at, idx] = dw.v, dw.e
    dl = Q(q * (full - (full * q).sum(1, keepdims=True)))
    weight = ((np.abs(full) + full_e) * q).sum(1, keepdims=True)
    dl.e = q * (full_e + (full_e * q).sum(1, keepdims=True)) + 2.0 ** -18 * (q * (np.abs(full) + full_e + weight) + 2 * prob * weight)
    part = mm(dl, Q(Wg64.T), F32)
    total = Q(dx.v + part.v, dx.e + part.e + 2 * u * (np.abs(dx.v) + np.abs(part.v))).rounded(dtype)
    assert_within(g["dx"], total.v, total.e, "dx")
    gWg = mm(Q(x64.T), dl, F32)
    gWg.e += sum_error(BF, T) * (np.abs(x64.T) @ (np.abs(dl.v) + dl.e))                        # on the matrix cores, in either type
    gWg = gWg.rounded(dtype)
    assert_within(g["dWg"], gWg.v, gWg.e, "dWg")
    assert_within(g["dgate_bias"], dl.v.sum(0), dl.e.sum(0) + (T + 8) * u * (np.abs(dl.v) + dl.e).sum(0), "dgate_bias")


def test_layer_in_a_graph(moe):   # noqa: F811
    """Captured forward and backward, replayed on other tokens (and so other routings) and masks, with eager work between the replays."""
    rng = np.random.default_rng(2)
    T, E, k, M, H = 90, 6, 2, 128, 256
    x, dout = draw(rng, (T, M), BF)[0], draw(rng, (T, M), BF)[0]
    Wg, W1, W2 = draw(rng, (M, E), BF, 0.1)[0], draw(rng, (E, M, H), BF, 0.1)[0], draw(rng, (E, H, M), BF, 0.1)[0]
    S1, S2 = draw(rng, (M, H), BF, 0.1)[0], draw(rng, (H, M), BF, 0.1)[0]
    numbers = torch.tensor([5, 0], dtype=torch.int64, device="cuda")
    layer = moe.DroplessLayer(Wg, None, W1, None, W2, None, k, 1, moe.ACT_GELU, shared=(S1, None, S2, None))

    def step():
        out, kept = layer.forward(x, residual=x, dropout=(0.1, numbers), keep=True)
        return [out, *layer.backward(kept, dout).values()]

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for i in range(4):
        numbers += 1
        x.copy_(draw(np.random.default_rng(100 + i), (T, M), BF)[0])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, step())), f"replay {i}"


def test_layer_refusals(moe):   # noqa: F811
    z = lambda *s, dtype=BF: torch.zeros(s, dtype=dtype, device="cuda")   # noqa: E731
    args = dict(Wg=z(16, 4), gate_bias=None, W1=z(4, 16, 24), b1=None, W2=z(4, 24, 16), b2=None, k=2, normalize=1, act=moe.ACT_SILU)
    layer = moe.DroplessLayer(**args)
    for bad in (dict(Wg=z(16, 5)), dict(W2=z(4, 16, 24)), dict(W2=z(4, 24, 16, dtype=F32)), dict(b1=z(4, 16)), dict(gate_bias=z(4)), dict(shared=(z(24, 8), None, z(8, 16), None)),
                dict(shared=(z(16, 8), None, z(16, 8), None)), dict(shared=(z(16, 8, dtype=F32), None, z(8, 16), None))):
        with pytest.raises(ValueError):
            moe.DroplessLayer(**{**args, **bad})
    for x in (z(3, 24), z(3, 16, dtype=F32), z(16)):
        with pytest.raises(ValueError):
            layer.forward(x)
    with pytest.raises(ValueError):
        layer.forward(z(3, 16), residual=z(2, 16))
