"""The operators on experts' rows that lie one behind the other, dense projections and dropout, in 64 bits and plain loops: the reference of their tests."""
import numpy as np
from scipy.special import erfc


def act(v, name):
    """The activation and its derivative."""
    if name == "relu":
        return np.maximum(v, 0.0), (v > 0).astype(np.float64)
    if name == "gelu":
        cdf = 0.5 * erfc(-v / np.sqrt(2.0))
        return v * cdf, cdf + v * np.exp(-0.5 * v * v) / np.sqrt(2.0 * np.pi)
    if name == "silu":
        s = 0.5 * (1.0 + np.tanh(0.5 * v))
        return v * s, s * (1.0 + v * (1.0 - s))
    return v, np.ones_like(v)


def rows(idx, loc, counts, C):
    """offsets, row_src, row_of."""
    T, k = idx.shape
    offsets = [0]
    for c in counts:
        offsets.append(offsets[-1] + (min(int(c), C) if C else int(c)))
    row_of = np.full((T, k), -1, dtype=np.int32)
    row_src = np.full(T * k, -1, dtype=np.int32)
    for t in range(T):
        for j in range(k):
            e, place = int(idx[t, j]), int(loc[t, j])
            if 0 <= e < len(counts) and 0 <= place < offsets[e + 1] - offsets[e]:
                row_of[t, j] = offsets[e] + place
                row_src[row_of[t, j]] = t
    return np.array(offsets, dtype=np.int32), row_src, row_of


def product(A, gather, W, bias, offsets):
    """Values before the activation and, for error bounds, the sums of the magnitudes."""
    R = A.shape[0] if gather is None else len(gather)
    v, size = np.zeros((R, W.shape[2])), np.zeros((R, W.shape[2]))
    for e in range(len(offsets) - 1):
        at = slice(offsets[e], offsets[e + 1])
        a = A[at] if gather is None else A[gather[at]]
        v[at] = a @ W[e] + (0 if bias is None else bias[e])
        size[at] = np.abs(a) @ np.abs(W[e]) + (0 if bias is None else np.abs(bias[e]))
    return v, size


def product_backward(d, A, gather, W, offsets):
    """dx, dW, db of d, the gradient of the values before the activation."""
    dx, dW, db = np.zeros((d.shape[0], W.shape[1])), np.zeros(W.shape), np.zeros((W.shape[0], W.shape[2]))
    for e in range(len(offsets) - 1):
        at = slice(offsets[e], offsets[e + 1])
        a = A[at] if gather is None else A[gather[at]]
        dx[at], dW[e], db[e] = d[at] @ W[e].T, a.T @ d[at], d[at].sum(0)
    return dx, dW, db


def philox(key, counter):
    """Philox4x32-10 (Salmon, Moraes, Dror, Shaw, SC 2011) in Python's integers."""
    c, k, word = list(counter), list(key), 0xFFFFFFFF
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & word, (a >> 32) ^ c[3] ^ k[1], a & word]
        k = [(k[0] + 0x9E3779B9) & word, (k[1] + 0xBB67AE85) & word]
    return c


def multiplier(n, p, seed, offset):
    """What each of n elements is multiplied by: 0 or 1 / (1 - p)."""
    word, below = 0xFFFFFFFF, int(np.rint(p * 65536))
    out = np.zeros(n)
    for g in range(n // 8):
        w = philox((seed & word, seed >> 32 & word), (g & word, g >> 32, offset & word, offset >> 32 & word))
        for i in range(8):
            if (w[i // 2] >> 16 * (i % 2) & 0xFFFF) >= below:
                out[8 * g + i] = 65536.0 / (65536 - below)
    return out


def combine(Y, row_of, gate_w):
    """The weighted sums and the sums of their terms' magnitudes."""
    T, k = row_of.shape
    out, size = np.zeros((T, Y.shape[1])), np.zeros((T, Y.shape[1]))
    for t in range(T):
        for j in range(k):
            if 0 <= row_of[t, j] < Y.shape[0]:
                term = (1.0 if gate_w is None else gate_w[t, j]) * Y[row_of[t, j]]
                out[t] += term
                size[t] += np.abs(term)
    return out, size
