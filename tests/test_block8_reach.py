"""The GPU cases of the 8-bit products reach the tiles that they are there for (csrc/matmul8_rules.h, compiled on its own).  No GPU needed."""
from test_block8_forms_gpu import STREAMED, TO_8BITS
from test_block8_rules import takes_large                            # noqa: F401


def test_streamed_cases_take_the_large_tile(takes_large):            # noqa: F811
    E, C, K, N = STREAMED
    row8 = -(-K // 128) * 128
    assert takes_large(E, C, K, N)
    for result in (1, 2):                                            # bytes of a value; 96 MB from where results are streamed
        assert E * (C * row8 + N * row8 + C * N * result) >= 96 << 20


def test_results_in_8bits_take_both_tiles(takes_large):              # noqa: F811
    assert [takes_large(*c) for c in TO_8BITS] == [True, False]
