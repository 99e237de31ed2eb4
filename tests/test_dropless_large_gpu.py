"""The layer without a capacity at widths whose products go to the 256 x 256 tile in every layout (test_rows_rules.py), against the 64-bit reference of test_dropless_gpu.py with its bounds."""
import pytest

import test_dropless_gpu
from test_rows_gpu import BF, F32, moe   # noqa: F401

pytestmark = pytest.mark.gpu

LAYERS = [(4700, 16, 2, 1024, 1024)]                               # tokens, experts, choices, widths


@pytest.mark.parametrize("T,E,k,M,H", LAYERS)
@pytest.mark.parametrize("dtype,act", [(BF, "gelu"), (BF, "silu"), (F32, "gelu")])
def test_layer(moe, T, E, k, M, H, act, dtype):   # noqa: F811
    test_dropless_gpu.test_layer(moe, T, E, k, M, H, act, 1, 0.0, True, True, dtype)
