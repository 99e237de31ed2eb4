"""The operators around the experts' 8-bit and few-token paths, as cases that can be timed and checked: what each one stands for,
its inputs, one pass in plain torch and one through the public entry points, and the work that the pass cannot do without.

A case is a dict of plain values.  Every case has
  op       "norm"     h = x + residual, y = RMS norm of h, in the storage type and / or in 8 bits (rms_norm, dequantize8)
           "norm_bwd" the gradient of that norm (rms_norm_backward)
           "ffn8"     the experts' feed-forward layer on 8-bit tokens and weights, rows gathered by the router's slots, and the
                      weighted combine (expert_ffn8, decode)
           "train8"   one training pass of an expert projection in 8 bits: the operands are quantised, y = x W, dx and dW
                      (expert_linear8_train, expert_linear8_backward)
           "few"      a whole layer for a few tokens, gate included (FewTokenLayer.forward)
  dtype    "bf16" or "fp32" storage
and the sizes of its op: T tokens, M model dim, H hidden dim, E experts, k choices per token, f capacity factor; "train8": C rows of
each of E experts, K and N the projection's input and output widths.

8 bits: e4m3 values in blocks of 128 along the axis that a product sums over, with one power of two for each block, the smallest
under which the block's largest magnitude is at most 448 (and at least 2^-126); weights share one for 128 x 128.  Rows of 8-bit values
are zero-padded to whole blocks, rows of exponents (biased by 127, one byte each) to a multiple of four.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
_ES = {"bf16": 2, "fp32": 4}
_EPS = 1e-6
_PER = 128


def _norm(name, op, dtype, T, M, residual, y, q):
    return dict(name=name, op=op, dtype=dtype, T=T, M=M, residual=residual, y=y, q=q)


def _ffn8(name, T, M, H, E, k, f, act, zipf, bias):
    return dict(name=name, op="ffn8", dtype="bf16", T=T, M=M, H=H, E=E, k=k, f=f, act=act, zipf=zipf, bias=bias)


def _train8(name, dtype, E, C, K, N, ragged):
    return dict(name=name, op="train8", dtype=dtype, E=E, C=C, K=K, N=N, ragged=ragged)


def _few(name, dtype, T, M, H, E, k, f, act, bias, w8):
    return dict(name=name, op="few", dtype=dtype, T=T, M=M, H=H, E=E, k=k, f=f, act=act, bias=bias, w8=w8)


def listed():
    return [
        # before the experts of one decode step: a handful of rows, for the gate (storage type) and the experts (8 bits)
        _norm("norm_decode", "norm", "bf16", 16, 4096, True, True, True),
        # the repository's largest workload: its tokens and the residual stream, normalised for a training forward
        _norm("norm_large", "norm", "bf16", 131072, 4096, True, True, False),
        # a quarter of the same tokens, trained: gradient through the norm joined with the residual's
        _norm("norm_backward", "norm_bwd", "bf16", 32768, 4096, True, True, False),
        # sizes that are no multiple of anything but 8, fp32, both outputs, no residual
        _norm("norm_ragged_fp32", "norm", "fp32", 3001, 776, False, True, True),
        # serving, a prefill chunk: many experts, a few rows each
        _ffn8("ffn8_prefill", 512, 1024, 4096, 64, 2, 2.0, "gelu", False, False),
        # a quarter of the largest workload's tokens through its fine-grained experts
        _ffn8("ffn8_finegrained", 32768, 4096, 1024, 128, 8, 1.25, "silu", False, False),
        # the first projection of the middle workload's experts, trained
        _train8("train8_mid", "bf16", 8, 4096, 2048, 2048, False),
        # odd widths, odd numbers of experts and rows, experts that hold fewer rows than their slab or none
        _train8("train8_ragged", "bf16", 17, 453, 776, 1544, True),
        # one decode step of a small batch: every expert's weights are read for a handful of rows
        _few("few_decode", "bf16", 16, 2048, 2048, 8, 2, 2.0, "gelu", False, False),
        # one token through fine-grained experts in 8 bits: the lowest latency there is
        _few("few_one8", "bf16", 1, 4096, 1024, 128, 8, 2.0, "silu", False, True),
        # a larger batch: four rows of tokens for the fullest experts, expert biases
        _few("few_batch", "bf16", 64, 1024, 4096, 64, 2, 2.0, "gelu", True, False),
        # the repository's smallest layer, a few tokens of it
        _few("few_tiny_fp32", "fp32", 5, 256, 512, 4, 1, 2.0, "relu", True, False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, step):
    return max(256, _log_int(rng, 256, 4096) // step * step)


def draw(rng):
    """One more case of the same ranges: sizes spread over their logarithm, a third of the widths multiples of 8 only."""
    while True:
        op = rng.choice(["norm", "norm", "norm_bwd", "ffn8", "ffn8", "train8", "train8", "few", "few", "few"])
        step = rng.choice([8, 64, 256])
        dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
        M, H = _width(rng, step), _width(rng, step)
        E = rng.choice([4, 8, 16, 32, 64, 128, _log_int(rng, 3, 128)])
        k = min(E, rng.choice([1, 1, 2, 2, 4, 8]))
        act = rng.choice(["relu", "gelu", "silu"])
        f = rng.choice([1.0, 1.25, 2.0])
        bias = rng.random() < 0.5
        if op in ("norm", "norm_bwd"):
            T = _log_int(rng, 1, 131072 if op == "norm" else 32768)
            q = op == "norm" and rng.random() < 0.5
            c = _norm("", op, dtype, T, M, rng.random() < 0.7, not q or rng.random() < 0.7, q)
            if T * M * _ES[dtype] > (1.1e9 if op == "norm" and not q else 2.7e8):
                continue
        elif op == "ffn8":
            T = _log_int(rng, 16, 32768)
            c = _ffn8("", T, M, H, E, k, f, act, rng.random() < 0.3, bias)
            if 4.0 * T * k * f * M * H > 5.5e12 or E * M * H > 6e8 or T * k * f * (M + H) > 1.7e9:
                continue
        elif op == "train8":
            E = min(E, 32)
            c = _train8("", dtype, E, _log_int(rng, 16, 8192), M, H, rng.random() < 0.5)
            if E * c["C"] * M * H > 1.38e11 or E * M * H > 1.5e8:
                continue
        else:
            w8 = dtype == "bf16" and rng.random() < 0.4
            c = _few("", dtype, rng.choice([1, _log_int(rng, 1, 64), _log_int(rng, 1, 64)]), M, H, E, k, f, act, bias, w8)
            if E * M * H > 6e8:
                continue
        return {n: v for n, v in c.items() if n != "name"}


# ---- inputs ------------------------------------------------------------------------------------------------------------

def _exponents(amax):
    """e of the smallest 2^e with amax <= 448 * 2^e, at least -126."""
    m, p = torch.frexp(amax)
    return (p - 9 + (m > 0.875).to(p.dtype)).clamp(min=-126)


def _padded(v, rows, cols):
    return torch.nn.functional.pad(v, (0, -v.shape[-1] % cols, 0, -v.shape[-2] % rows))


def _quantized(v, rows):
    """The last two axes of fp32 `v` in 8 bits: e4m3 values [.., R, K up to 128s] and the exponents of groups of 128 along K,
    of one row each (rows = 1) or of 128 (rows = 128): [.., ceil(R / rows), groups]."""
    R = v.shape[-2]
    p = _padded(v, rows, _PER)
    g = p.reshape(*p.shape[:-2], p.shape[-2] // rows, rows, p.shape[-1] // _PER, _PER)
    e = _exponents(g.abs().amax(dim=(-3, -1)))
    q = torch.ldexp(g, -e[..., :, None, :, None]).to(torch.float8_e4m3fn)
    return q.reshape(p.shape)[..., :R, :], e


def _values(q, e, rows):
    """What _quantized holds, as fp32 [.., R, K up to 128s]."""
    p = _padded(q.float(), rows, _PER)
    g = p.reshape(*p.shape[:-2], p.shape[-2] // rows, rows, p.shape[-1] // _PER, _PER)
    return torch.ldexp(g, e[..., :, None, :, None]).reshape(p.shape)[..., :q.shape[-2], :]


def _bytes_of(e):
    """Exponents as they are stored: biased by 127, one byte each, rows padded to a multiple of four with 127."""
    return torch.nn.functional.pad((e + 127).to(torch.uint8), (0, -e.shape[-1] % 4), value=127).contiguous()


def _rounded(v, rows):
    """fp32 values as 8 bits hold them, in the layout of `v`."""
    return _values(*_quantized(v, rows), rows)[..., :v.shape[-1]]


def _routing(g, T, E, k, C, zipf):
    """A router's decisions: distinct experts, normalised weights, arrival positions in the order (choice, token), arrivals, slots."""
    logits = torch.randn((T, E), generator=g, device="cuda")
    if zipf:
        logits -= 2.4 * torch.log(torch.arange(1, E + 1, device="cuda", dtype=torch.float32))
    top = torch.topk(logits, k, dim=1)
    idx = top.indices.to(torch.int32)
    gate_w = torch.softmax(top.values, dim=1)
    flat = idx.t().reshape(-1).long()
    order = torch.argsort(flat, stable=True)
    counts = torch.bincount(flat, minlength=E)
    start = torch.cumsum(counts, 0) - counts
    place = torch.empty_like(flat)
    place[order] = torch.arange(T * k, device="cuda") - start[flat[order]]
    loc = place.view(k, T).t().contiguous().to(torch.int32)
    slot_src = torch.full((E, C), -1, dtype=torch.int32, device="cuda")
    kept = place < C
    token = torch.arange(T, device="cuda", dtype=torch.int32).repeat(k)
    slot_src[flat[kept], place[kept]] = token[kept]
    return dict(idx=idx, gate_w=gate_w.contiguous(), loc=loc, counts=counts.to(torch.int32), slot_src=slot_src)


def _capacity(case):
    return math.ceil(case["k"] * case["f"] * case["T"] / case["E"])


def prepare(case, seed):
    """Tokens, weights and routing on the GPU, as a program has them before the call; 8-bit tensors in their stored form."""
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    op, dt = case["op"], _DTYPES[case["dtype"]]

    def stored(*shape, std=1.0):                 # in pieces of the first dimension: no fp32 copy of a large tensor
        out = torch.empty(shape, dtype=dt, device="cuda")
        rows = max(1, min(shape[0], (1 << 26) // max(1, math.prod(shape[1:]))))
        for i in range(0, shape[0], rows):
            out[i:i + rows] = torch.randn(out[i:i + rows].shape, generator=g, device="cuda").mul_(std)
        return out

    def stored8(E, K, N):                        # a weight [K, N] for each expert, in 8 bits as [N, K up to 128s]
        q = torch.empty((E, N, K + -K % _PER), dtype=torch.float8_e4m3fn, device="cuda")
        s = []
        step = max(1, (1 << 26) // (K * N))
        for i in range(0, E, step):
            w = torch.randn((min(step, E - i), N, K), generator=g, device="cuda").mul_(1.0 / math.sqrt(K))
            q[i:i + step], e = _quantized(w, _PER)
            s.append(_bytes_of(e))
        return q, torch.cat(s)

    s = dict(case=case)
    if op in ("norm", "norm_bwd"):
        T, M = case["T"], case["M"]
        s["x"] = stored(T, M)                    # "norm_bwd": the residual stream h that the forward wrote
        s["weight"] = (1.0 + 0.1 * torch.randn((M,), generator=g, device="cuda")).to(dt)
        s["residual"] = stored(T, M, std=2.0) if case["residual"] else None
        s["dy"] = stored(T, M) if op == "norm_bwd" else None
        return s
    if op == "train8":
        E, C, K, N = case["E"], case["C"], case["K"], case["N"]
        s["x"], s["W"], s["dy"] = stored(E, C, K), stored(E, K, N, std=1.0 / math.sqrt(K)), stored(E, C, N)
        s["counts"] = None
        if case["ragged"]:                       # from empty to beyond the slab, as un-truncated arrivals are
            s["counts"] = torch.randint(0, C + C // 4 + 1, (E,), generator=g, device="cuda", dtype=torch.int32)
            s["counts"][0] = 0
        return s
    T, M, H, E, k = (case[n] for n in ("T", "M", "H", "E", "k"))
    C = _capacity(case)
    s.update(C=C, x=stored(T, M), b1=stored(E, H, std=0.1) if case["bias"] else None, b2=stored(E, M, std=0.1) if case["bias"] else None)
    if op == "ffn8" or case["w8"]:
        (s["W1"], s["s1"]), (s["W2"], s["s2"]) = stored8(E, M, H), stored8(E, H, M)
    else:
        s["W1"], s["W2"], s["s1"], s["s2"] = stored(E, M, H, std=1.0 / math.sqrt(M)), stored(E, H, M, std=1.0 / math.sqrt(H)), None, None
    if op == "ffn8":
        q, e = _quantized(s.pop("x").float(), 1)
        s["x8"], s["xs"] = q.contiguous(), _bytes_of(e)
        s.update(_routing(g, T, E, k, C, case["zipf"]))
    else:
        s["Wg"] = stored(M, E, std=1.0 / math.sqrt(M))
    return s


# ---- one pass in plain torch ---------------------------------------------------------------------------------------------

def _act(v, act):
    if act == "relu":
        return torch.relu(v)
    if act == "gelu":
        return 0.5 * v * (1.0 + torch.erf(v * math.sqrt(0.5)))
    return v * torch.sigmoid(v)


def _plain_norm(s, case):
    h = s["x"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
    y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + _EPS) * s["weight"].float()
    dt = s["x"].dtype
    return dict(h=h.to(dt) if s["residual"] is not None else None, y=y.to(dt) if case["y"] else None,
                y8=_rounded(y, 1).to(torch.bfloat16) if case["q"] else None)     # bf16 holds every value of the 8-bit format


def _plain_norm_bwd(s, case):
    h, dy, dt = s["x"].float(), s["dy"].float(), s["x"].dtype
    r = torch.rsqrt((h * h).mean(1, keepdim=True) + _EPS)
    g = dy * s["weight"].float()
    dx = r * (g - h * (r * r * (g * h).mean(1, keepdim=True)))
    if s["residual"] is not None:                # the gradient that reaches the residual stream past the norm
        dx = dx + s["residual"].float()
    return dict(dx=dx.to(dt), dweight=(dy * h * r).sum(0).to(dt))


def _weights8(q, s, K):
    """[E, N, K up to 128s] in 8 bits -> fp32 [E, K, N]."""
    e = s[..., :q.shape[-1] // _PER].to(torch.int32) - 127
    return _values(q, e, _PER)[..., :K].transpose(1, 2).contiguous()


def _bias(b):
    return 0.0 if b is None else b.float()[:, None, :]


def _combine(Y, idx, loc, gate_w, C):
    rows = Y[idx.long(), loc.long().clamp(max=C - 1)]
    return ((gate_w * (loc < C))[..., None] * rows).sum(1)


def _plain_ffn8(s, case):
    M, H, C = case["M"], case["H"], s["C"]
    x = _values(s["x8"], s["xs"][:, :s["x8"].shape[1] // _PER].to(torch.int32) - 127, 1)[:, :M]
    Z = x[s["slot_src"].clamp(min=0).long()]
    hidden = _act(torch.bmm(Z, _weights8(s["W1"], s["s1"], M)) + _bias(s["b1"]), case["act"])
    Y = torch.bmm(_rounded(hidden, 1), _weights8(s["W2"], s["s2"], H)) + _bias(s["b2"])
    return _combine(Y, s["idx"], s["loc"], s["gate_w"], C).to(torch.bfloat16)


def _plain_train8(s, case):
    x, W, dy, dt = s["x"].float(), s["W"].float(), s["dy"].float(), s["x"].dtype
    if s["counts"] is not None:
        live = (torch.arange(case["C"], device=x.device)[None, :] < s["counts"][:, None])[..., None]
        x, dy = torch.where(live, x, 0.0), torch.where(live, dy, 0.0)
    W = _rounded(W, _PER)
    y = torch.bmm(_rounded(x, 1), W)
    dx = torch.bmm(_rounded(dy, 1), W.transpose(1, 2).contiguous())
    dW = torch.bmm(_rounded(x.transpose(1, 2).contiguous(), 1), _rounded(dy.transpose(1, 2).contiguous(), 1).transpose(1, 2).contiguous())
    return dict(y=y.to(dt), dx=dx.to(dt), dW=dW.to(dt))


def _plain_few(s, case):
    M, H, T, E, k, C = case["M"], case["H"], case["T"], case["E"], case["k"], s["C"]
    x = s["x"].float()
    logits = x @ s["Wg"].float()
    order = torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :k]
    gate_w = torch.softmax(logits, 1).gather(1, order)
    if k > 1:
        gate_w = gate_w / gate_w.sum(1, keepdim=True)
    chosen = (order.t().reshape(-1, 1) == torch.arange(E, device=x.device)).int()            # in the order (choice, token)
    loc = ((torch.cumsum(chosen, 0) - chosen) * chosen).sum(1).view(k, T).t()
    pick = order.reshape(-1) if T * k <= E else None                                        # each pair's weights, or every expert's

    def picked(v):
        return v if v is None or pick is None else v[pick]

    def weights(q, e, K):
        return q.float() if e is None else _weights8(q, e, K)

    rows = x.repeat_interleave(k, 0)[:, None, :] if pick is not None else x.expand(E, T, M)
    hidden = _act(torch.bmm(rows, weights(picked(s["W1"]), picked(s["s1"]), M)) + _bias(picked(s["b1"])), case["act"])
    Y = torch.bmm(hidden, weights(picked(s["W2"]), picked(s["s2"]), H)) + _bias(picked(s["b2"]))
    Y = Y.view(T, k, M) if pick is not None else Y[order, torch.arange(T, device=x.device)[:, None]]
    out = ((gate_w * (loc < C))[..., None] * Y).sum(1).to(s["x"].dtype)
    return dict(out=out, idx=order.int(), loc=loc.int(), gate_w=gate_w)


_PLAIN = {"norm": _plain_norm, "norm_bwd": _plain_norm_bwd, "ffn8": _plain_ffn8, "train8": _plain_train8, "few": _plain_few}


# ---- one pass through the framework ---------------------------------------------------------------------------------------

def _own(s, case):
    from paper_2206_03382_amd import moe
    op = case["op"]
    if op == "norm":
        s["out"] = r = moe.rms_norm(s["x"], s["weight"], _EPS, residual=s["residual"], want_y=case["y"], want_8=case["q"], out=s.get("out"))
        y8 = moe.dequantize8(r["y8"], torch.bfloat16) if case["q"] else None
        return dict(h=r["h"] if s["residual"] is not None else None, y=r["y"], y8=y8)
    if op == "norm_bwd":
        s["out"] = moe.rms_norm_backward(s["dy"], s["x"], s["weight"], _EPS, dh=s["residual"], out=s.get("out"))
        return s["out"]
    if op == "train8":
        y, kept = moe.expert_linear8_train(s["x"], s["W"], counts=s["counts"])
        dx, dW = moe.expert_linear8_backward(s["dy"], kept)
        return dict(y=y, dx=dx, dW=dW)
    act = {"relu": moe.ACT_RELU, "gelu": moe.ACT_GELU, "silu": moe.ACT_SILU}[case["act"]]
    M, H = case["M"], case["H"]
    if s["s1"] is not None:
        W1, W2 = moe.Block8(s["W1"], s["s1"], M, True), moe.Block8(s["W2"], s["s2"], H, True)
    else:
        W1, W2 = s["W1"], s["W2"]
    if op == "ffn8":
        Y = moe.expert_ffn8(moe.Block8(s["x8"], s["xs"], M, False), W1, s["b1"], W2, s["b2"], act, torch.bfloat16,
                            counts=s["counts"], slot_src=s["slot_src"])
        return moe.decode(Y, s["idx"], s["loc"], s["gate_w"])
    if "layer" not in s:                         # owns the workspace and the outputs
        s["layer"] = moe.FewTokenLayer(s["Wg"], None, W1, s["b1"], W2, s["b2"], T=case["T"], k=case["k"], f=case["f"],
                                       normalize=int(case["k"] > 1), act=act, keep_routing=True)
    out, r = s["layer"].forward(s["x"]), s["layer"].routing
    return dict(out=out, idx=r["idx"], loc=r["loc"], gate_w=r["gate_w"])


def run(state):
    case = state["case"]
    return _own(state, case) if own else _PLAIN[case["op"]](state, case)


# ---- the work, and the result in 64 bits -----------------------------------------------------------------------------------

def work(case):
    op, es = case["op"], _ES[case["dtype"]]
    if op in ("norm", "norm_bwd"):
        n = float(case["T"] * case["M"])
        if op == "norm_bwd":                     # stream, gradient, residual's gradient in; gradient out
            return dict(bytes=n * es * (4 if case["residual"] else 3) + 2 * case["M"] * es, flops=10 * n)
        slabs = es * (3 if case["residual"] else 1) + (es if case["y"] else 0) + ((3 + 1.0 / _PER) if case["q"] else 0)
        return dict(bytes=n * slabs + case["M"] * es, flops=6 * n)
    if op == "train8":
        E, C, K, N = (float(case[n]) for n in ("E", "C", "K", "N"))
        rows = E * C * (0.6 * (E - 1) / E if case["ragged"] else 1.0)    # mean fill of uniform arrivals up to 1.25 C
        return dict(bytes=es * (2 * rows * K + 2 * rows * N + 2 * E * K * N), flops=6.0 * rows * K * N)
    T, M, H, E, k = (float(case[n]) for n in ("T", "M", "H", "E", "k"))
    fills = _fills(case)
    pairs, live = float(fills.sum()), float((fills >= 0.5).sum()) if case["T"] * case["k"] > 4 * case["E"] else E * (1.0 - (1.0 - k / E) ** T)
    weights = live * M * H * 2 * (1 + 1.0 / 16384 if op == "ffn8" or case.get("w8") else es)
    if op == "ffn8":
        return dict(bytes=T * M * (1 + 1.0 / _PER) + weights + T * M * 2 + 12 * T * k, flops=4.0 * pairs * M * H)
    return dict(bytes=2 * T * M * es + weights + M * E * es, flops=4.0 * pairs * M * H + 2.0 * T * M * E)


def _fills(case):
    """Expected kept choices of each expert, from a fixed sample of gate logits."""
    T, E, k = case["T"], case["E"], case["k"]
    n = min(max(T, 1024), 8192)
    logits = np.random.Generator(np.random.Philox(key=[11, E])).standard_normal((n, E), dtype=np.float32)
    if case.get("zipf"):
        logits -= 2.4 * np.log(np.arange(1, E + 1, dtype=np.float32))
    chosen = np.argpartition(-logits, k - 1, axis=1)[:, :k]
    return np.minimum(np.bincount(chosen.ravel(), minlength=E) * (T / n), _capacity(case))


def _round8(v, axes):
    """float64 `v`, whose last axis is the one that is summed over, rounded as the 8-bit format rounds it: blocks of 128 along the last
    axis, and along the one before it too where axes = 2."""
    shape = v.shape
    out = v.new_zeros((*shape[:-2], shape[-2] + (-shape[-2] % _PER if axes == 2 else 0), shape[-1] + -shape[-1] % _PER))
    out[..., :shape[-2], :shape[-1]] = v
    wide = out.shape
    b = out.view(*wide[:-2], -1, _PER if axes == 2 else 1, wide[-1] // _PER, _PER)
    top = b.abs().amax(-1).amax(-2)[..., :, None, :, None]
    scale = torch.exp2(torch.ceil(torch.log2(torch.where(top > 0, top, torch.ones_like(top)) / 448.0)).clamp(min=-126.0))
    scale = torch.where(top > 448.0 * scale, 2.0 * scale, scale)                # log2's own rounding, either way
    scale = torch.where((top <= 224.0 * scale) & (top > 0), 0.5 * scale, scale).clamp(min=2.0 ** -126)
    v = b / scale
    size = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6)))) / 8.0         # spacing of e4m3 numbers near v
    size = torch.where(v.abs() >= 16.0 * size, 2.0 * size, size)
    return (torch.round(v / size) * size * scale).view(wide)[..., :shape[-2], :shape[-1]]


def _stored8_exact(q, s, K):
    """[E, N, K up to 128s] -> float64 [E, N, K]."""
    n = torch.arange(q.shape[1], device=q.device) // _PER
    j = torch.arange(K, device=q.device) // _PER
    return q[:, :, :K].double() * torch.exp2(s.double() - 127.0)[:, n][:, :, j]


def _act_exact(v, act):
    if act == "relu":
        return v.clamp(min=0)
    if act == "gelu":
        return v * torch.special.ndtr(v)
    return v / (1.0 + torch.exp(-v))


def exact(case, seed):
    """The operators' definitions in float64, expert by expert."""
    s, op = prepare(case, seed), case["op"]
    if op == "norm":
        h = s["x"].double() + (0 if s["residual"] is None else s["residual"].double())
        y = h / torch.sqrt(h.square().sum(1, keepdim=True) / case["M"] + _EPS) * s["weight"].double()
        return dict(h=h if case["residual"] else None, y=y if case["y"] else None, y8=_round8(y, 1) if case["q"] else None)
    if op == "norm_bwd":
        h, dy = s["x"].double(), s["dy"].double()
        root = torch.sqrt(h.square().sum(1, keepdim=True) / case["M"] + _EPS)
        n, g = h / root, dy * s["weight"].double()
        dx = (g - n * (n * g).sum(1, keepdim=True) / case["M"]) / root
        return dict(dx=dx if s["residual"] is None else dx + s["residual"].double(), dweight=(dy * n).sum(0))
    if op == "train8":
        E, C = case["E"], case["C"]
        fills = [C] * E if s["counts"] is None else [min(C, c) for c in s["counts"].tolist()]
        y = torch.zeros((E, C, case["N"]), dtype=torch.float64, device="cuda")
        dx = torch.zeros((E, C, case["K"]), dtype=torch.float64, device="cuda")
        dW = torch.zeros(s["W"].shape, dtype=torch.float64, device="cuda")
        for e, n in enumerate(fills):
            if n:
                x, dy, W = s["x"][e, :n].double(), s["dy"][e, :n].double(), _round8(s["W"][e].double(), 2)
                y[e, :n] = _round8(x, 1) @ W
                dx[e, :n] = _round8(dy, 1) @ W.T
                dW[e] = _round8(x.T.contiguous(), 1) @ _round8(dy.T.contiguous(), 1).T
        return dict(y=y, dx=dx, dW=dW)
    T, M, H, E, k, C = *(case[n] for n in ("T", "M", "H", "E", "k")), s["C"]
    bias = [torch.zeros((E, 1), dtype=torch.float64, device="cuda") if b is None else b.double() for b in (s["b1"], s["b2"])]
    if op == "ffn8":
        x = s["x8"].double()[:, :M] * torch.exp2(s["xs"].double() - 127.0).repeat_interleave(_PER, 1)[:, :M]
        idx, loc, gate_w = s["idx"].long(), s["loc"].long(), s["gate_w"].double()
    else:
        x = s["x"].double()
        logits = (x @ s["Wg"].double()).float().double()
        idx = torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :k]
        gate_w = torch.exp(logits - torch.logsumexp(logits, 1, keepdim=True)).gather(1, idx)
        gate_w = gate_w / gate_w.sum(1, keepdim=True) if k > 1 else gate_w
        loc, seen = torch.zeros((T, k), dtype=torch.long), [0] * E
        for j in range(k):
            for t, e in enumerate(idx[:, j].tolist()):
                loc[t, j], seen[e] = seen[e], seen[e] + 1
        loc = loc.cuda()
    out = torch.zeros((T, M), dtype=torch.float64, device="cuda")
    for e in range(E):
        t, j = torch.nonzero((idx == e) & (loc < C), as_tuple=True)
        if not t.numel():
            continue
        W1 = s["W1"][e].double() if s["s1"] is None else _stored8_exact(s["W1"][e:e + 1], s["s1"][e:e + 1], M)[0].T
        W2 = s["W2"][e].double() if s["s2"] is None else _stored8_exact(s["W2"][e:e + 1], s["s2"][e:e + 1], H)[0].T
        hidden = _act_exact(x[t] @ W1 + bias[0][e], case["act"])
        if op == "ffn8":
            hidden = _round8(hidden, 1)
        out.index_add_(0, t, gate_w[t, j][:, None] * (hidden @ W2 + bias[1][e]))
    return out if op == "ffn8" else dict(out=out, idx=None, loc=None, gate_w=gate_w)
