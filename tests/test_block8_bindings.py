"""What the bindings of the norm, the 8-bit matrices and the few-token layer hand to the library and give back, with the library replaced by one that records its
calls: no GPU needed, and a call with wrong sizes reads nothing."""
import pytest
import torch

from paper_2206_03382_amd import moe


class Recorder:
    """The library: every entry point succeeds, every size is 4096, and the last call of each is kept."""

    def __init__(self):
        self.calls = {}

    def __getattr__(self, name):
        def call(*args):
            self.calls[name] = args
            return b"recorded" if name == "moe_status_string" else 4096 if name.endswith("_bytes") else 8 if name == "moe_capacity" else moe.OK
        return call


@pytest.fixture()
def library(monkeypatch):
    r = Recorder()
    monkeypatch.setattr(moe, "lib", lambda: r)
    monkeypatch.setattr(moe, "_p", lambda t: None if t is None else t.data_ptr())
    monkeypatch.setattr(moe, "_stream", lambda: 0)
    return r


# ---- rms_norm's results, used again as `out` ------------------------------------------------------------------------

def test_rms_norm_without_a_residual_gives_this_call_s_x(library):
    a, b = torch.ones((4, 64)), torch.full((4, 64), 2.0)
    first = moe.rms_norm(a, None, 1e-6)
    assert first["h"] is a
    again = moe.rms_norm(b, None, 1e-6, out=first)
    assert again["h"] is b and library.calls["moe_rms_norm"][7] is None


def test_rms_norm_with_a_residual_never_writes_into_an_earlier_x(library):
    a, b, res = torch.ones((4, 64)), torch.full((4, 64), 2.0), torch.zeros((4, 64))
    out = moe.rms_norm(a, None, 1e-6)
    got = moe.rms_norm(b, None, 1e-6, residual=res, out=out)
    to = library.calls["moe_rms_norm"][7]
    assert to == got["h"].data_ptr() and to not in (a.data_ptr(), b.data_ptr(), res.data_ptr())
    # from then on the same memory, calls without a residual in between or not
    moe.rms_norm(a, None, 1e-6, out=got)
    assert got["h"] is a
    last = moe.rms_norm(a, None, 1e-6, residual=res, out=got)
    assert library.calls["moe_rms_norm"][7] == to == last["h"].data_ptr()


def test_rms_norm_writes_h_where_the_caller_says(library):
    x, res, y = torch.ones((4, 64)), torch.zeros((4, 64)), torch.empty((4, 64))
    mine = torch.empty((4, 64))
    moe.rms_norm(x, None, 1e-6, residual=res, out={**moe.rms_norm(x, None, 1e-6), "h": mine})
    assert library.calls["moe_rms_norm"][7] == mine.data_ptr()
    plain = moe.rms_norm(x, None, 1e-6)
    with pytest.raises(ValueError):
        moe.rms_norm(x, None, 1e-6, residual=res, out={**plain, "y": y[:2]})
    assert plain["h"] is x                                          # a refused call changes nothing
    out = dict(h=res, y=y, y8=None)                                # the sum replaces the residual
    got = moe.rms_norm(x, None, 1e-6, residual=res, out=out)
    assert library.calls["moe_rms_norm"][7] == res.data_ptr() and got["h"] is res and got["y"] is y


def test_norm_layer_without_a_residual(library):
    """The first block of a model: h is x, and the next forward, with a residual, has its own h again."""
    bf = torch.bfloat16
    W1, W2 = moe._alloc8((4,), 128, 64, True, "cpu"), moe._alloc8((4,), 64, 128, True, "cpu")
    for T in (8, 100):
        layer = moe.NormMoELayer8(None, 1e-6, torch.zeros((64, 4), dtype=bf), None, W1, None, W2, None, T, 2, 1.0, 1, 0)
        x, res = torch.ones((T, 64), dtype=bf), torch.zeros((T, 64), dtype=bf)
        out, h = layer.forward(x, None)
        assert h is x and out is layer.out
        _, h = layer.forward(x, res)
        own = library.calls["moe_rms_norm"][7]
        assert h.data_ptr() == own and own not in (x.data_ptr(), res.data_ptr())
        _, h = layer.forward(x, None)
        assert h is x


# ---- shapes of 8-bit matrices: a product reads what they say ------------------------------------------------------------

def matrix8(*shape, blocks=False):
    *lead, R, K = shape
    return moe._alloc8(tuple(lead), R, K, blocks, "cpu")


def test_matmul8_refuses_plain_matrices(library):
    """Two [256, 512] operands pass for 256 experts of [512, 512] if rows are taken for experts."""
    plain, stack = matrix8(256, 512), matrix8(2, 16, 128)
    four = moe.Block8(stack.q[None], stack.s[None], 128, False)
    rows = torch.zeros((2, 16), dtype=torch.int32)
    for A, B, gather in [(plain, plain, None), (plain, matrix8(256, 512, blocks=True), None), (stack, matrix8(16, 128), None), (four, four, None), (stack, four, None),
                         (four, stack, None), (stack, stack, rows), (four, stack, rows), (matrix8(2, 128), matrix8(2, 128), rows)]:
        with pytest.raises(ValueError):
            moe.matmul8(A, B, gather=gather)
    assert "moe_matmul8" not in library.calls
    assert moe.matmul8(stack, stack).shape == (2, 16, 16) and moe.matmul8(matrix8(9, 128), stack, gather=rows).shape == (2, 16, 16)
    assert library.calls["moe_matmul8"][12:16] == (2, 16, 128, 16)


def test_expert_ffn8_refuses_plain_matrices(library):
    W1, W2 = matrix8(4, 256, 128, blocks=True), matrix8(4, 128, 256, blocks=True)
    slots = torch.zeros((4, 16), dtype=torch.int32)
    for x8, a, b, s in [(matrix8(4, 128), W1, W2, None), (matrix8(1, 9, 128), W1, W2, slots), (matrix8(1, 4, 16, 128), W1, W2, None),
                        (matrix8(4, 16, 128), matrix8(128, 128, blocks=True), matrix8(128, 128, blocks=True), None)]:
        with pytest.raises(ValueError):
            moe.expert_ffn8(x8, a, None, b, None, moe.ACT_RELU, slot_src=s)
    with pytest.raises(ValueError):
        moe.FewTokenLayer(torch.zeros((128, 128), dtype=torch.bfloat16), None, matrix8(128, 128, blocks=True), None, matrix8(128, 128, blocks=True), None, 4, 1, 1.0, 0, 0)
    assert not any(name.startswith(("moe_expert", "moe_layer")) for name in library.calls)
    assert moe.expert_ffn8(matrix8(4, 16, 128), W1, None, W2, None, moe.ACT_RELU).shape == (4, 16, 128)


def test_matmul8_checks_the_bias(library):
    A, B = matrix8(2, 16, 128), matrix8(2, 24, 128)
    for bad in (torch.zeros(24, dtype=torch.bfloat16), torch.zeros((2, 16), dtype=torch.bfloat16), torch.zeros((1, 24), dtype=torch.bfloat16), torch.zeros((2, 24))):
        with pytest.raises(ValueError):
            moe.matmul8(A, B, bias=bad)
    assert "moe_matmul8" not in library.calls
    moe.matmul8(A, B, bias=torch.zeros((2, 24), dtype=torch.bfloat16))


def few_layer(gate_bias=None, b1=None, b2=None, w8=False):
    bf = torch.bfloat16
    W1, W2 = (matrix8(4, 128, 64, blocks=True), matrix8(4, 64, 128, blocks=True)) if w8 else (torch.zeros((4, 64, 128), dtype=bf), torch.zeros((4, 128, 64), dtype=bf))
    return moe.FewTokenLayer(torch.zeros((64, 4), dtype=bf), gate_bias, W1, b1, W2, b2, 8, 2, 1.0, 1, 0)


@pytest.mark.parametrize("w8", [False, True])
def test_few_token_layer_checks_the_experts_biases(library, w8):
    bf = dict(dtype=torch.bfloat16)
    for b1, b2 in [(torch.zeros(128, **bf), None), (torch.zeros((4, 64), **bf), None), (torch.zeros((4, 128)), None), (None, torch.zeros(64, **bf)),
                   (None, torch.zeros((4, 128), **bf)), (None, torch.zeros((1, 64), **bf))]:
        with pytest.raises(ValueError):
            few_layer(None, b1, b2, w8)
    few_layer(None, torch.zeros((4, 128), **bf), torch.zeros((4, 64), **bf), w8)


def test_layers_check_the_gate_bias(library):
    bf = torch.bfloat16
    W1, W2 = matrix8(4, 128, 64, blocks=True), matrix8(4, 64, 128, blocks=True)

    def norm_layer(bias, T):
        return moe.NormMoELayer8(None, 1e-6, torch.zeros((64, 4), dtype=bf), bias, W1, None, W2, None, T, 2, 1.0, 1, 0)
    for bad in (torch.zeros(4, dtype=bf), torch.zeros(3), torch.zeros(4, dtype=torch.float64), torch.zeros((4, 4))):
        for make in (few_layer, lambda b: norm_layer(b, 8), lambda b: norm_layer(b, 100)):
            with pytest.raises(ValueError):
                make(bad)
    for make in (few_layer, lambda b: norm_layer(b, 8), lambda b: norm_layer(b, 100)):
        make(torch.zeros(4))


def test_more_leading_dimensions_are_refused(library):
    """The library takes one leading dimension; of more, all but the first matrices were left unwritten."""
    with pytest.raises(ValueError):
        moe.quantize8(torch.zeros((2, 3, 16, 128)))
    with pytest.raises(ValueError):
        moe.dequantize8(matrix8(2, 3, 16, 128))
    assert not library.calls
    for shape in ((16, 128), (2, 16, 128)):
        q, _ = moe.quantize8(torch.zeros(shape))
        assert tuple(moe.dequantize8(q).shape) == shape


def test_rms_norm_refuses_outputs_that_out_has_no_memory_for(library):
    x = torch.ones((4, 128))
    only_8, only_y = moe.rms_norm(x, None, 1e-6, want_y=False, want_8=True), moe.rms_norm(x, None, 1e-6)
    for kept, asked in [(only_8, dict(want_y=True)), (only_y, dict(want_8=True)), (only_8, dict(want_y=True, want_8=True))]:
        library.calls.clear()
        with pytest.raises(ValueError):
            moe.rms_norm(x, None, 1e-6, out=kept, **asked)
        assert not library.calls
    for kept, y, y8 in [(only_8, False, True), (only_y, True, False)]:          # without a word: what `out` has
        got = moe.rms_norm(x, None, 1e-6, out=kept)
        assert (got["y"] is not None, got["y8"] is not None) == (y, y8)
        moe.rms_norm(x, None, 1e-6, out=kept, want_y=y, want_8=y8)
    both = moe.rms_norm(x, None, 1e-6, want_8=True)
    moe.rms_norm(x, None, 1e-6, want_y=False, out=both)                         # all of them are this call's
    assert library.calls["moe_rms_norm"][8] == both["y"].data_ptr()
