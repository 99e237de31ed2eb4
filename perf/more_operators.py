"""The operators of a layer without capacity, as cases that can be timed and checked: what each one stands for, its inputs, one pass in
plain torch and one through the public entry points, and the work that the pass cannot do without.

A case is a dict of plain values.  Every case has
  op       "ragged"         one projection of the experts on rows of their own number, which are gathered from the tokens:
                            y[r] = act(x[row_src[r]] W[e] + b[e]) for the rows offsets[e] <= r < offsets[e + 1] (ragged_matmul)
           "ragged_train"   the same with its gradients dx (by row), dW and db (ragged_matmul, ragged_matmul_backward)
           "linear"         y = act(x W + b) + residual (linear)
           "linear_train"   the same with dx, dW and db (linear, linear_backward)
           "dropout"        y = residual + dropout(x), from a counter-based generator (dropout)
           "dropout_train"  the same with dx, whose mask is made again (dropout)
           "combine"        the rows of a router's choices and the weighted sum of their results, dropped out and added to the
                            residual (ragged_rows, ragged_combine)
           "combine_train"  the same with the gradients of the rows' results and of the weights (ragged_combine_backward)
  dtype    "bf16" or "fp32" storage
and the sizes of its op: T tokens, K and N a projection's input and output widths, M model dim, E experts, k choices per token,
p the probability of dropping, f a capacity factor (0: none, nothing is dropped).

The generator is Philox4x32-10 (Salmon, Moraes, Dror, Shaw, SC 2011): the key is the seed, the counter the number of a group of eight
elements and an offset; an element takes 16 of the 128 bits and is dropped where they are below p 2^16.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
_ES = {"bf16": 2, "fp32": 4}


def _ragged(name, op, dtype, T, K, N, E, k, act, zipf, bias):
    return dict(name=name, op=op, dtype=dtype, T=T, K=K, N=N, E=E, k=k, act=act, zipf=zipf, bias=bias)


def _linear(name, op, dtype, T, K, N, act, bias, residual):
    return dict(name=name, op=op, dtype=dtype, T=T, K=K, N=N, act=act, bias=bias, residual=residual)


def _dropout(name, op, dtype, T, M, p, residual):
    return dict(name=name, op=op, dtype=dtype, T=T, M=M, p=p, residual=residual)


def _combine(name, op, dtype, T, M, E, k, f, p, residual):
    return dict(name=name, op=op, dtype=dtype, T=T, M=M, E=E, k=k, f=f, p=p, residual=residual)


def listed():
    return [
        # one token through its eight of 128 fine-grained experts: their weights are read for a row each
        _ragged("ragged_decode", "ragged", "bf16", 1, 4096, 1024, 128, 8, "silu", False, False),
        # a quarter of the largest workload's tokens, none dropped
        _ragged("ragged_finegrained", "ragged", "bf16", 32768, 4096, 1024, 128, 8, "silu", False, False),
        # the middle workload's first projection, trained
        _ragged("ragged_train", "ragged_train", "bf16", 16384, 2048, 2048, 8, 2, "gelu", False, True),
        # odd widths, an odd number of experts, most rows at the first of them and some without any
        _ragged("ragged_train_fp32", "ragged_train", "fp32", 1501, 776, 1544, 17, 2, "relu", True, True),
        # one token through the dense projection that closes a block, onto its residual stream: the lowest latency there is
        _linear("linear_decode", "linear", "bf16", 1, 4096, 4096, "none", True, True),
        # a prefill of many sequences through a dense expert beside the routed ones
        _linear("linear_large", "linear", "bf16", 16384, 4096, 4096, "gelu", True, True),
        # a dense expert's projection in a training step
        _linear("linear_train", "linear_train", "bf16", 8192, 2048, 2048, "gelu", True, True),
        # sizes that are no multiple of anything but 8, fp32
        _linear("linear_odd_fp32", "linear", "fp32", 1001, 776, 1544, "relu", True, True),
        # a handful of rows, where the call itself is what counts
        _dropout("dropout_small", "dropout", "bf16", 16, 4096, 0.1, True),
        # half of the largest workload's tokens and the residual stream, forward and backward
        _dropout("dropout_large", "dropout_train", "bf16", 65536, 4096, 0.1, True),
        # one decode step of a small batch
        _combine("combine_decode", "combine", "bf16", 16, 2048, 8, 2, 0.0, 0.0, True),
        # the fine-grained experts' results for 16384 tokens, trained
        _combine("combine_train", "combine_train", "bf16", 16384, 4096, 128, 8, 0.0, 0.1, True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, step):
    return max(256, _log_int(rng, 256, 4096) // step * step)


def draw(rng):
    """One more case of the same ranges: sizes spread over their logarithm, a third of the widths multiples of 8 only."""
    while True:
        op = rng.choice(["ragged", "ragged", "ragged_train", "ragged_train", "linear", "linear", "linear_train", "dropout", "dropout_train",
                         "combine", "combine_train"])
        step = rng.choice([8, 64, 256])
        dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
        es, most = _ES[dtype], 2.2e12 if dtype == "bf16" else 1.4e11
        K, N = _width(rng, step), _width(rng, step)
        E = rng.choice([4, 8, 16, 32, 64, 128, _log_int(rng, 3, 128)])
        k = min(E, rng.choice([1, 1, 2, 2, 4, 8]))
        act = rng.choice(["none", "relu", "gelu", "silu"])
        bias, residual = rng.random() < 0.5, rng.random() < 0.7
        p = rng.choice([0.0, 0.1, 0.1, rng.uniform(0.01, 0.6)])
        if op in ("ragged", "ragged_train"):
            T = rng.choice([_log_int(rng, 1, 64), _log_int(rng, 1, 32768), _log_int(rng, 16, 32768)])
            c = _ragged("", op, dtype, T, K, N, E, k, act, rng.random() < 0.3, bias)
            if (2.0 if op == "ragged" else 6.0) * T * k * K * N > most or E * K * N > 5.4e8 or T * k * (K + N) * es > 2.7e9:
                continue
        elif op in ("linear", "linear_train"):
            T = rng.choice([_log_int(rng, 1, 64), _log_int(rng, 1, 32768), _log_int(rng, 16, 32768)])
            c = _linear("", op, dtype, T, K, N, act, bias, residual)
            if (2.0 if op == "linear" else 6.0) * T * K * N > most / 4:
                continue
        elif op in ("dropout", "dropout_train"):
            c = _dropout("", op, dtype, _log_int(rng, 1, 65536), K, p, residual)
            if c["T"] * K * es > 5.4e8:
                continue
        else:
            c = _combine("", op, dtype, _log_int(rng, 1, 32768), K, E, k, rng.choice([0.0, 0.0, 1.0, 1.25]), p, residual)
            if c["T"] * k * K * es > 1.08e9:
                continue
        return {n: v for n, v in c.items() if n != "name"}


# ---- inputs ------------------------------------------------------------------------------------------------------------

def _routing(g, T, E, k, zipf):
    """A router's decisions: distinct experts, normalised weights, arrival positions in the order (choice, token), arrivals."""
    logits = torch.randn((T, E), generator=g, device="cuda")
    if zipf:
        logits -= 2.4 * torch.log(torch.arange(1, E + 1, device="cuda", dtype=torch.float32))
    top = torch.topk(logits, k, dim=1)
    idx = top.indices.to(torch.int32)
    flat = idx.t().reshape(-1).long()
    order = torch.argsort(flat, stable=True)
    counts = torch.bincount(flat, minlength=E)
    start = torch.cumsum(counts, 0) - counts
    place = torch.empty_like(flat)
    place[order] = torch.arange(T * k, device="cuda") - start[flat[order]]
    loc = place.view(k, T).t().contiguous().to(torch.int32)
    return idx, torch.softmax(top.values, dim=1).contiguous(), loc, counts.to(torch.int32)


def _capacity(case):
    return math.ceil(case["k"] * case["f"] * case["T"] / case["E"]) if case["f"] > 0 else 0


def prepare(case, seed):
    """Tokens, weights and a router's decisions on the GPU, as a program has them before the call."""
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    op, dt = case["op"], _DTYPES[case["dtype"]]

    def stored(*shape, std=1.0):                 # in pieces of the first dimension: no fp32 copy of a large tensor
        out = torch.empty(shape, dtype=dt, device="cuda")
        rows = max(1, min(shape[0], (1 << 26) // max(1, math.prod(shape[1:]))))
        for i in range(0, shape[0], rows):
            out[i:i + rows] = torch.randn(out[i:i + rows].shape, generator=g, device="cuda").mul_(std)
        return out

    def numbers():                               # the generator's seed and offset, on the device as a captured step needs them
        return torch.randint(0, 1 << 62, (2,), generator=g, device="cuda", dtype=torch.int64)

    s = dict(case=case)
    T = case["T"]
    if op in ("dropout", "dropout_train"):
        M = case["M"]
        s.update(x=stored(T, M), residual=stored(T, M, std=2.0) if case["residual"] else None, seed=numbers(),
                 dy=stored(T, M) if op == "dropout_train" else None)
        return s
    if op in ("linear", "linear_train"):
        K, N = case["K"], case["N"]
        s.update(x=stored(T, K), W=stored(K, N, std=1.0 / math.sqrt(K)), bias=stored(N, std=0.1) if case["bias"] else None,
                 residual=stored(T, N, std=2.0) if case["residual"] else None, dy=stored(T, N) if op == "linear_train" else None)
        return s
    E, k = case["E"], case["k"]
    idx, gate_w, loc, counts = _routing(g, T, E, k, case.get("zipf", False))
    if op in ("combine", "combine_train"):
        M, C = case["M"], _capacity(case)
        R = int((counts.clamp(max=C) if C else counts).sum())
        s.update(idx=idx, gate_w=gate_w, loc=loc, counts=counts, C=C, Y=stored(R, M), residual=stored(T, M, std=2.0) if case["residual"] else None,
                 seed=numbers(), dy=stored(T, M) if op == "combine_train" else None)
        return s
    K, N = case["K"], case["N"]
    offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = torch.cumsum(counts, 0)
    row_src = torch.empty(T * k, dtype=torch.int32, device="cuda")
    row_src[(offsets[idx.long()] + loc).reshape(-1).long()] = torch.arange(T, dtype=torch.int32, device="cuda").repeat_interleave(k)
    s.update(offsets=offsets, row_src=row_src, fills=counts.tolist(), x=stored(T, K), W=stored(E, K, N, std=1.0 / math.sqrt(K)),
             bias=stored(E, N, std=0.1) if case["bias"] else None, dy=stored(T * k, N) if op == "ragged_train" else None)
    return s


# ---- one pass in plain torch ---------------------------------------------------------------------------------------------

def _act(v, act):
    if act == "relu":
        return torch.relu(v)
    if act == "gelu":
        return 0.5 * v * (1.0 + torch.erf(v * math.sqrt(0.5)))
    if act == "silu":
        return v * torch.sigmoid(v)
    return v


def _act_grad(v, act):
    if act == "relu":
        return (v > 0).to(v.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(v * math.sqrt(0.5))) + v * torch.exp(-0.5 * v * v) * (1.0 / math.sqrt(2.0 * math.pi))
    if act == "silu":
        sg = torch.sigmoid(v)
        return sg * (1.0 + v * (1.0 - sg))
    return torch.ones_like(v)


def _by_expert(s):
    """(expert, first row, one past the last), the experts that have rows."""
    at = 0
    for e, n in enumerate(s["fills"]):
        if n:
            yield e, at, at + n
        at += n


def _pre(x, W, b):
    v = x @ W.float()
    return v if b is None else v + b.float()


def _plain_ragged(s, case):
    dt = s["x"].dtype
    src = s["row_src"].long()
    y = torch.empty((src.shape[0], case["N"]), dtype=dt, device="cuda")
    train = case["op"] == "ragged_train"
    if train:
        dx = torch.empty((src.shape[0], case["K"]), dtype=dt, device="cuda")
        dW = torch.zeros_like(s["W"])
        db = torch.zeros((case["E"], case["N"]), dtype=dt, device="cuda") if case["bias"] else None
    for e, lo, hi in _by_expert(s):
        x = s["x"][src[lo:hi]].float()
        v = _pre(x, s["W"][e], None if s["bias"] is None else s["bias"][e])
        y[lo:hi] = _act(v, case["act"])
        if train:
            d = s["dy"][lo:hi].float() * _act_grad(v, case["act"])
            dx[lo:hi] = d @ s["W"][e].float().t()
            dW[e] = x.t() @ d
            if case["bias"]:
                db[e] = d.sum(0)
    return dict(y=y, dx=dx, dW=dW, db=db) if train else dict(y=y)


def _plain_linear(s, case):
    dt, x = s["x"].dtype, s["x"].float()
    v = _pre(x, s["W"], s["bias"])
    y = _act(v, case["act"])
    y = (y if s["residual"] is None else y + s["residual"].float()).to(dt)
    if case["op"] == "linear":
        return dict(y=y)
    d = s["dy"].float() * _act_grad(v, case["act"])
    return dict(y=y, dx=(d @ s["W"].float().t()).to(dt), dW=(x.t() @ d).to(dt), db=d.sum(0).to(dt) if case["bias"] else None)


_LOW = 0xFFFFFFFF


def _philox(key, counter):
    """Philox4x32-10 on int64 tensors that hold 32 bits each; the product of two of them wraps around, which leaves its 64 bits in place."""
    c0, c1, c2, c3 = counter
    k0, k1 = key
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & _LOW) ^ c1 ^ k0, b & _LOW, ((a >> 32) & _LOW) ^ c3 ^ k1, a & _LOW
        k0, k1 = (k0 + 0x9E3779B9) & _LOW, (k1 + 0xBB67AE85) & _LOW
    return c0, c1, c2, c3


def _below(p):
    return int(round(p * 65536))


def _kept(seed, T, M, p):
    """[T, M]: whether the element is kept."""
    group = torch.arange(T * M // 8, device="cuda", dtype=torch.int64)
    words = _philox((seed[0] & _LOW, (seed[0] >> 32) & _LOW),
                    (group & _LOW, group >> 32, (seed[1] & _LOW).expand_as(group), ((seed[1] >> 32) & _LOW).expand_as(group)))
    bits = torch.stack([h for w in words for h in (w & 0xFFFF, w >> 16)], dim=1)
    return (bits >= _below(p)).view(T, M)


def _drop(v, seed, p):
    if p == 0.0:
        return v
    return torch.where(_kept(seed, *v.shape, p), v * (65536.0 / (65536 - _below(p))), 0.0)


def _plain_dropout(s, case):
    dt, p = s["x"].dtype, case["p"]
    y = _drop(s["x"].float(), s["seed"], p)
    y = (y if s["residual"] is None else y + s["residual"].float()).to(dt)
    return dict(y=y) if case["op"] == "dropout" else dict(y=y, dx=_drop(s["dy"].float(), s["seed"], p).to(dt))


def _plain_combine(s, case):
    dt, p, C, Y = s["Y"].dtype, case["p"], s["C"], s["Y"]
    counts = s["counts"].clamp(max=C) if C else s["counts"]
    offsets = torch.zeros(case["E"] + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = torch.cumsum(counts, 0)
    live = s["loc"] < C if C else torch.ones_like(s["loc"], dtype=torch.bool)
    row_of = torch.where(live, offsets[s["idx"].long()] + s["loc"], -1)
    row_src = torch.full((row_of.numel() + 1,), -1, dtype=torch.int32, device="cuda")     # one more, for choices without a row
    row_src[torch.where(live, row_of, row_of.numel()).reshape(-1).long()] = torch.arange(case["T"], dtype=torch.int32, device="cuda").repeat_interleave(case["k"])
    row_src = torch.where(torch.arange(row_of.numel(), device="cuda") < offsets[-1], row_src[:-1], -1)
    at, w = row_of.clamp(min=0).long(), torch.where(live, s["gate_w"], 0.0)
    out = torch.zeros((case["T"], case["M"]), device="cuda")
    for j in range(case["k"]):
        out += w[:, j, None] * Y[at[:, j]].float()
    out = _drop(out, s["seed"], p)
    out = (out if s["residual"] is None else out + s["residual"].float()).to(dt)
    r = dict(offsets=offsets, row_src=row_src, row_of=row_of, out=out)
    if case["op"] == "combine_train":
        d = _drop(s["dy"].float(), s["seed"], p)
        dY, dw = torch.empty((Y.shape[0] + 1, case["M"]), dtype=dt, device="cuda"), torch.empty_like(w)
        for j in range(case["k"]):
            dY[torch.where(live[:, j], row_of[:, j], Y.shape[0]).long()] = (w[:, j, None] * d).to(dt)
            dw[:, j] = torch.where(live[:, j], (d * Y[at[:, j]].float()).sum(1), 0.0)
        r.update(dY=dY[:-1], dgate_w=dw)
    return r


_PLAIN = {"ragged": _plain_ragged, "ragged_train": _plain_ragged, "linear": _plain_linear, "linear_train": _plain_linear,
          "dropout": _plain_dropout, "dropout_train": _plain_dropout, "combine": _plain_combine, "combine_train": _plain_combine}


# ---- one pass through the framework ---------------------------------------------------------------------------------------

def _own(s, case):
    from paper_2206_03382_amd import moe
    op = case["op"]
    if op in ("dropout", "dropout_train"):
        y = moe.dropout(s["x"], case["p"], s["seed"], residual=s["residual"])
        return dict(y=y) if op == "dropout" else dict(y=y, dx=moe.dropout(s["dy"], case["p"], s["seed"]))
    if op in ("combine", "combine_train"):
        rows = moe.ragged_rows(s["idx"], s["loc"], s["counts"], C=s["C"])
        drop = (case["p"], s["seed"]) if case["p"] > 0 else None
        out = moe.ragged_combine(s["Y"], rows.row_of, s["gate_w"], residual=s["residual"], dropout=drop)
        r = dict(offsets=rows.offsets, row_src=rows.row_src, row_of=rows.row_of, out=out)
        if op == "combine_train":
            r["dY"], r["dgate_w"] = moe.ragged_combine_backward(s["dy"], s["Y"], rows.row_of, s["gate_w"], dropout=drop)
        return r
    act = {"none": moe.ACT_NONE, "relu": moe.ACT_RELU, "gelu": moe.ACT_GELU, "silu": moe.ACT_SILU}[case["act"]]
    if op == "linear":
        return dict(y=moe.linear(s["x"], s["W"], s["bias"], act, residual=s["residual"]))
    if op == "linear_train":
        y, pre = moe.linear(s["x"], s["W"], s["bias"], act, residual=s["residual"], keep_pre=True)
        g = moe.linear_backward(s["dy"], s["x"], s["W"], act, pre, want_db=case["bias"])
        return dict(y=y, dx=g["dx"], dW=g["dW"], db=g["db"])
    if op == "ragged":
        return dict(y=moe.ragged_matmul(s["x"], s["W"], s["offsets"], s["bias"], act, gather=s["row_src"]))
    y, pre = moe.ragged_matmul(s["x"], s["W"], s["offsets"], s["bias"], act, gather=s["row_src"], keep_pre=True)
    g = moe.ragged_matmul_backward(s["dy"], s["x"], s["W"], s["offsets"], act, pre, gather=s["row_src"], want_db=case["bias"])
    return dict(y=y, dx=g["dx"], dW=g["dW"], db=g["db"])


def run(state):
    case = state["case"]
    return _own(state, case) if own else _PLAIN[case["op"]](state, case)


# ---- the work, and the result in 64 bits -----------------------------------------------------------------------------------

def work(case):
    op, es, T = case["op"], _ES[case["dtype"]], float(case["T"])
    train = op.endswith("_train")
    if op in ("dropout", "dropout_train"):
        n = T * case["M"]
        return dict(bytes=n * es * ((3 if case["residual"] else 2) + (2 if train else 0)), flops=n * (4 if train else 2))
    if op in ("combine", "combine_train"):
        k, M = case["k"], case["M"]
        rows = float(_fills(case).sum())
        bytes_ = rows * M * es + T * M * es * (2 if case["residual"] else 1) + T * k * 20
        if train:                                # the rows' results are one input of both directions
            bytes_ += T * M * es + rows * M * es + T * k * 4
        return dict(bytes=bytes_, flops=(5.0 if train else 2.0) * rows * M)
    K, N = case["K"], case["N"]
    if op in ("linear", "linear_train"):
        rows, weights, x = T, float(K * N), T * K
    else:
        fills = _fills(case)
        rows = T * case["k"]
        live = float((fills >= 0.5).sum()) if rows > 4 * case["E"] else case["E"] * (1.0 - (1.0 - case["k"] / case["E"]) ** T)
        weights, x = live * K * N, T * K
    bytes_ = es * (x + weights + rows * N * (2 if case.get("residual") else 1))
    if train:                                    # dy in, dx and the weights' gradient out
        bytes_ += es * (rows * N + rows * K + (weights if op == "linear_train" else float(case["E"] * K * N)))
    return dict(bytes=bytes_, flops=(6.0 if train else 2.0) * rows * K * N)


def _fills(case):
    """Expected kept choices of each expert, from a fixed sample of gate logits."""
    T, E, k = case["T"], case["E"], case["k"]
    n = min(max(T, 1024), 8192)
    logits = np.random.Generator(np.random.Philox(key=[13, E])).standard_normal((n, E), dtype=np.float32)
    if case.get("zipf"):
        logits -= 2.4 * np.log(np.arange(1, E + 1, dtype=np.float32))
    chosen = np.argpartition(-logits, k - 1, axis=1)[:, :k]
    fills = np.bincount(chosen.ravel(), minlength=E) * (T / n)
    return np.minimum(fills, _capacity(case)) if case.get("f") else fills


def _act_exact(v, act):
    """The activation and its derivative in float64."""
    if act == "none":
        return v, torch.ones_like(v)
    if act == "relu":
        return v.clamp(min=0), torch.where(v > 0, 1.0, 0.0).double()
    if act == "gelu":
        phi = torch.special.ndtr(v)
        return v * phi, phi + v * torch.exp(-v.square() / 2) / math.sqrt(2 * math.pi)
    e = torch.exp(-v)
    return v / (1 + e), (1 + e + v * e) / (1 + e).square()


def _project_exact(x, W, b, act, dy):
    v = x @ W.double() + (0 if b is None else b.double())
    y, slope = _act_exact(v, act)
    if dy is None:
        return y, None, None, None
    d = dy.double() * slope
    return y, d @ W.double().T, x.T @ d, d.sum(0)


def _multiplier_exact(seed, T, M, p):
    """What an element of [T, M] is multiplied by.  32-bit words as two halves of 16 bits, whose products stay below 2^63."""
    if p == 0.0:
        return 1.0
    s0, s1 = (int(v) & 0xFFFFFFFFFFFFFFFF for v in seed.tolist())

    def times(a, m):                             # high and low word of a * m
        low = (a & 0xFFFF) * (m & 0xFFFF)
        mid = (a >> 16) * (m & 0xFFFF) + (low >> 16)
        mid2 = (a & 0xFFFF) * (m >> 16) + (mid & 0xFFFF)
        return (a >> 16) * (m >> 16) + (mid >> 16) + (mid2 >> 16), ((mid2 & 0xFFFF) << 16) | (low & 0xFFFF)

    out = torch.empty((T * M // 8, 8), dtype=torch.float64, device="cuda")
    border = math.floor(p * 65536 + 0.5) if (p * 65536) % 1 != 0.5 else 2 * round(p * 32768)
    for lo in range(0, out.shape[0], 1 << 22):
        n = min(1 << 22, out.shape[0] - lo)
        at = torch.arange(lo, lo + n, dtype=torch.int64, device="cuda")
        c = [at % 2 ** 32, at // 2 ** 32, torch.full_like(at, s1 % 2 ** 32), torch.full_like(at, s1 // 2 ** 32)]
        for r in range(10):
            k0, k1 = (s0 % 2 ** 32 + r * 0x9E3779B9) % 2 ** 32, (s0 // 2 ** 32 + r * 0xBB67AE85) % 2 ** 32
            (h0, l0), (h1, l1) = times(c[0], 0xD2511F53), times(c[2], 0xCD9E8D57)
            c = [h1 ^ c[1] ^ k0, l1, h0 ^ c[3] ^ k1, l0]
        for j in range(8):
            out[lo:lo + n, j] = ((c[j // 2] >> 16 * (j % 2)) % 65536 >= border).double()
    return out.view(T, M) / (1.0 - border / 65536.0)


def exact(case, seed):
    """The operators' definitions in float64, expert by expert."""
    s, op = prepare(case, seed), case["op"]
    train = op.endswith("_train")
    if op in ("dropout", "dropout_train"):
        m = _multiplier_exact(s["seed"], case["T"], case["M"], case["p"])
        y = s["x"].double() * m + (0 if s["residual"] is None else s["residual"].double())
        return dict(y=y, dx=s["dy"].double() * m) if train else dict(y=y)
    if op in ("linear", "linear_train"):
        y, dx, dW, db = _project_exact(s["x"].double(), s["W"], s["bias"], case["act"], s["dy"])
        if s["residual"] is not None:
            y = y + s["residual"].double()
        return dict(y=y, dx=dx, dW=dW, db=db if case["bias"] else None) if train else dict(y=y)
    E, k, T = case["E"], case["k"], case["T"]
    if op in ("ragged", "ragged_train"):
        at = s["offsets"].tolist()
        y = torch.zeros((T * k, case["N"]), dtype=torch.float64, device="cuda")
        dx, dW, db = torch.zeros((T * k, case["K"]) if train else 0, dtype=torch.float64, device="cuda"), [], []
        for e in range(E):
            rows = slice(at[e], at[e + 1])
            y[rows], gx, gW, gb = _project_exact(s["x"][s["row_src"][rows].long()].double(), s["W"][e], None if s["bias"] is None else s["bias"][e],
                                                 case["act"], s["dy"][rows] if train else None)
            if train:
                dx[rows] = gx
                dW.append(gW)
                db.append(gb)
        return dict(y=y, dx=dx, dW=torch.stack(dW), db=torch.stack(db) if case["bias"] else None) if train else dict(y=y)
    m, C = _multiplier_exact(s["seed"], T, case["M"], case["p"]), s["C"] or T * k
    first, n = [], 0
    for c in s["counts"].tolist():
        first.append(n)
        n += min(c, C)
    first = torch.tensor(first, device="cuda")
    out = torch.zeros((T, case["M"]), dtype=torch.float64, device="cuda")
    dY, dw = torch.zeros(s["Y"].shape if train else 0, dtype=torch.float64, device="cuda"), torch.zeros((T, k), dtype=torch.float64, device="cuda")
    for j in range(k):
        t = torch.nonzero(s["loc"][:, j] < C).flatten()
        row = first[s["idx"][t, j].long()] + s["loc"][t, j]
        w = s["gate_w"][t, j].double()[:, None]
        out[t] += w * s["Y"][row].double()
        if train:
            d = s["dy"][t].double() * (m[t] if case["p"] > 0 else m)
            dY[row] = w * d
            dw[t, j] = (d * s["Y"][row].double()).sum(1)
    out = out * m + (0 if s["residual"] is None else s["residual"].double())
    r = dict(offsets=None, row_src=None, row_of=None, out=out)
    if train:
        r.update(dY=dY, dgate_w=dw)
    return r
