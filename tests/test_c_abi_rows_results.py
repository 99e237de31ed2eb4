"""Results of the operators on experts' rows that would go onto what they are made of, or onto each other, are refused on the host: nothing is launched, no GPU is needed."""
import itertools
import os

import pytest


@pytest.fixture(scope="module")
def moe():
    from paper_2206_03382_amd import moe as m
    if not os.path.exists(m.LIB_PATH):
        from paper_2206_03382_amd.build import build_library
        build_library(verbose=False)
    m.lib()
    return m


# every pointer an address of its own, aligned and never dereferenced
AT = {n: (i + 1) << 20 for i, n in enumerate(
    "idx loc counts offsets row_src row_of A gather W bias pre out dy x x_pre ws dx dW db residual seed Y gate_w d_out dY dgate_w".split())}

# entry point -> (arguments by name, pointers among them), results, pairs that may share memory
CALLS = {
    "moe_ragged_rows": (("idx", "loc", "counts", 8, 4, 2, 0, "offsets", "row_src", "row_of"), ("offsets", "row_src", "row_of"), ()),
    "moe_ragged_matmul": (("A", "gather", 16, "W", "bias", 1, 1, "offsets", 8, 2, 64, 64, "pre", "out"), ("pre", "out"), ()),
    "moe_ragged_matmul_backward": (("dy", "x", "gather", 16, "W", "pre", 1, "x_pre", 1, 1, "offsets", 8, 2, 64, 64, "ws", 1 << 40, "dx", "dW", "db"), ("dx", "dW", "db", "ws"), ()),
    "moe_linear": (("x", "W", "bias", 1, "residual", 1, 1, 4096, 64, "ws", 1 << 40, "pre", "out"), ("pre", "out", "ws"), (("out", "residual"),)),
    "moe_linear_backward": (("dy", "x", "W", "pre", 1, 1, 8, 64, 64, "ws", 1 << 40, "dx", "dW", "db"), ("dx", "dW", "db", "ws"), ()),
    "moe_dropout": (("x", "residual", 0.5, "seed", 1, 64, "out"), ("out",), (("out", "x"), ("out", "residual"))),
    "moe_ragged_combine": (("Y", 8, "row_of", "gate_w", "residual", 0.5, "seed", 1, 4, 64, 2, "out"), ("out",), (("out", "residual"),)),
    "moe_ragged_combine_backward": (("d_out", "Y", 8, "row_of", "gate_w", 0.5, "seed", 1, 4, 64, 2, "dY", "dgate_w"), ("dY", "dgate_w"), ()),
}


def pairs():
    for name, (args, results, may) in CALLS.items():
        pointers = [a for a in args if isinstance(a, str)]
        for result, other in itertools.product(results, pointers):
            if result != other and (result, other) not in may:
                yield name, result, other


@pytest.mark.parametrize("name,result,onto", list(pairs()))
def test_result_onto_another_pointer(moe, name, result, onto):
    at = {**AT, result: AT[onto]}
    args = [at[a] if isinstance(a, str) else a for a in CALLS[name][0]]
    assert getattr(moe.lib(), name)(*args, None) == moe.INVALID_ARG
