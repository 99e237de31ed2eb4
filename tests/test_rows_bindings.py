"""What the bindings of the operators on experts' rows, of dense projections and of dropout hand to the library and refuse, with the library replaced by one that records its calls: no GPU needed.  And
the reference generator's published known answers."""
import pytest
import torch

from oracle import rows_oracle as O
from paper_2206_03382_amd import moe

BF = torch.bfloat16


class Recorder:
    """The library: every entry point succeeds, every size is 4096, and the last call of each is kept."""

    def __init__(self):
        self.calls = {}

    def __getattr__(self, name):
        def call(*args):
            self.calls[name] = args
            return 4096 if name.endswith("_bytes") else moe.OK
        return call


@pytest.fixture()
def library(monkeypatch):
    r = Recorder()
    monkeypatch.setattr(moe, "lib", lambda: r)
    monkeypatch.setattr(moe, "_stream", lambda: 0)
    monkeypatch.setattr(moe, "_here", lambda *t: [None if x is None else x.data_ptr() for x in t])
    return r


def z(*shape, dtype=BF):
    return torch.zeros(shape, dtype=dtype)


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def test_tensors_of_another_device_are_refused(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    with pytest.raises(ValueError):
        moe._here(z(8))
    moe._here(None)


def test_ragged_rows(library):
    r = moe.ragged_rows(i32(6, 2), i32(6, 2), i32(5), C=3)
    assert r.offsets.shape == (6,) and r.row_src.shape == (12,) and r.row_of.shape == (6, 2) and library.calls["moe_ragged_rows"][3:7] == (6, 5, 2, 3)
    for bad in ((z(6, 2), i32(6, 2), i32(5)), (i32(6), i32(6), i32(5)), (i32(6, 2), i32(2, 6), i32(5)), (i32(6, 2), i32(6, 2), z(5))):
        with pytest.raises(ValueError):
            moe.ragged_rows(*bad)


def test_ragged_matmul(library):
    A, W, off = z(10, 16), z(3, 16, 24), i32(4)
    out, pre = moe.ragged_matmul(A, W, off, z(3, 24), moe.ACT_SILU, gather=i32(30), keep_pre=True)
    assert out.shape == pre.shape == (30, 24) and library.calls["moe_ragged_matmul"][8:12] == (30, 3, 16, 24) and library.calls["moe_ragged_matmul"][2] == 10
    assert moe.ragged_matmul(A, W, off, keep_pre=True)[1] is None and library.calls["moe_ragged_matmul"][12] is None
    mine = z(10, 24)
    assert moe.ragged_matmul(A, W, off, out=mine) is mine
    for bad in (dict(A=z(10, 24)), dict(A=z(10, 16, dtype=torch.float32)), dict(offsets=i32(3)), dict(offsets=z(4)), dict(bias=z(24)), dict(bias=z(3, 24, dtype=torch.float32)),
                dict(gather=z(30)), dict(gather=i32(5, 6)), dict(out=z(9, 24)), dict(out=z(10, 24, dtype=torch.float32))):
        with pytest.raises(ValueError):
            moe.ragged_matmul(**{**dict(A=A, W=W, offsets=off), **bad})
    with pytest.raises(TypeError):
        moe.ragged_matmul(z(10, 16, dtype=torch.float16), z(3, 16, 24, dtype=torch.float16), off)


def test_ragged_matmul_backward(library):
    base = dict(dy=z(10, 24), x=z(10, 16), W=z(3, 16, 24), offsets=i32(4))
    g = moe.ragged_matmul_backward(**base)
    assert g["dx"].shape == (10, 16) and g["dW"].shape == (3, 16, 24) and g["db"].shape == (3, 24)
    g = moe.ragged_matmul_backward(**{**base, "dy": z(7, 24)}, gather=i32(7), want_dW=False, want_db=False)
    assert g["dx"].shape == (7, 16) and g["dW"] is None and g["db"] is None and library.calls["moe_ragged_matmul_backward"][-3:-1] == (None, None)
    for bad in (dict(dy=z(9, 24)), dict(dy=z(10, 16)), dict(x=z(10, 24)), dict(pre=z(10, 16)), dict(x_pre=z(10, 24)), dict(gather=i32(9)), dict(offsets=i32(5)),
                dict(dy=z(10, 24, dtype=torch.float32)), dict(pre=z(10, 24, dtype=torch.float32))):
        with pytest.raises(ValueError):
            moe.ragged_matmul_backward(**{**base, **bad})


def test_linear(library):
    x, W, res = z(5, 16), z(16, 24), z(5, 24)
    assert moe.linear(x, W, z(24), moe.ACT_RELU, residual=res, out=res) is res
    assert moe.linear(x, W, None, moe.ACT_GELU, keep_pre=True)[1].shape == (5, 24) and library.calls["moe_linear"][10] == 4096
    assert moe.linear(x, W, keep_pre=True)[1] is None and library.calls["moe_linear"][11] is None
    for bad in (dict(x=z(5, 24)), dict(bias=z(16)), dict(residual=z(4, 24)), dict(residual=z(5, 24, dtype=torch.float32)), dict(out=z(5, 16))):
        with pytest.raises(ValueError):
            moe.linear(**{**dict(x=x, W=W), **bad})
    g = moe.linear_backward(res, x, W, moe.ACT_RELU, z(5, 24), want_dx=False)
    assert g["dx"] is None and g["dW"].shape == (16, 24) and g["db"].shape == (24,)
    for bad in (dict(dy=x), dict(x=res), dict(pre=x)):
        with pytest.raises(ValueError):
            moe.linear_backward(**{**dict(dy=res, x=x, W=W), **bad})


def test_dropout_and_combine(library):
    x, seed = z(4, 16), torch.zeros(2, dtype=torch.int64)
    assert moe.dropout(x, 0.1, seed, residual=x, out=x) is x and library.calls["moe_dropout"][5] == 64
    library.calls.clear()
    assert moe.dropout(x, 0.0, seed) is x and not library.calls
    assert moe.dropout(x, 0.0, seed, residual=x) is not x and library.calls.pop("moe_dropout") and moe.dropout(x, 0.0, seed, out=z(4, 16)) is not x and library.calls
    for bad in (dict(seed=seed[:1]), dict(seed=seed.int()), dict(residual=z(4, 8)), dict(residual=z(4, 16, dtype=torch.float32)), dict(out=z(8, 8))):
        with pytest.raises(ValueError):
            moe.dropout(**{**dict(x=x, p=0.1, seed=seed), **bad})
    Y, of, w = z(9, 16), i32(4, 2), z(4, 2, dtype=torch.float32)
    assert moe.ragged_combine(Y, of, w, residual=x, dropout=(0.1, seed), out=x) is x
    assert library.calls["moe_ragged_combine"][5] == 0.1 and moe.ragged_combine(Y, of, None).shape == (4, 16) and library.calls["moe_ragged_combine"][5] == 0.0
    for bad in (dict(gate_w=z(4, 2)), dict(gate_w=w[:3]), dict(row_of=z(4, 2)), dict(row_of=i32(8)), dict(residual=z(4, 8)), dict(out=z(9, 16)), dict(dropout=(0.1, seed[:1]))):
        with pytest.raises(ValueError):
            moe.ragged_combine(**{**dict(Y=Y, row_of=of, gate_w=w), **bad})
    dY, dw = moe.ragged_combine_backward(x, Y, of, w)
    assert dY.shape == (9, 16) and dw.shape == (4, 2) and dw.dtype == torch.float32
    for bad in (dict(d_out=Y), dict(dY=x), dict(d_out=z(4, 16, dtype=torch.float32))):
        with pytest.raises(ValueError):
            moe.ragged_combine_backward(**{**dict(d_out=x, Y=Y, row_of=of, gate_w=w), **bad})


def test_reference_generator():
    """The known answers that were published with the generator."""
    full = 0xFFFFFFFF
    assert O.philox((0, 0), (0, 0, 0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert O.philox((full, full), (full, full, full, full)) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    m = O.multiplier(8, 0.5, 0, 0)                                  # halves of the first answer, the lower one first, against 0x8000
    assert m.tolist() == [2.0 * (h >= 0x8000) for h in (0xE8D5, 0x6627, 0xC58D, 0xE169, 0xAC4C, 0xBC57, 0xDBD8, 0x9B00)]
