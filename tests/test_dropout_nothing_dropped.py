"""dropout with p = 0, without residual and memory for the result, gives x itself; what it refuses is what it refuses with any other p.  The library is not called: no GPU needed."""
import pytest
import torch

from paper_2206_03382_amd import moe
from test_rows_bindings import BF, library, z   # noqa: F401


@pytest.mark.parametrize("x,code", [(z(0, 16), moe.INVALID_ARG), (z(3, 4), moe.UNSUPPORTED), (z(33)[1:], moe.UNSUPPORTED), (z(40)[4:36], moe.UNSUPPORTED), (z(17, dtype=torch.float32)[1:], moe.UNSUPPORTED)])
def test_refusals(library, x, code):   # noqa: F811
    library.moe_status_string = lambda status: b"refused"
    with pytest.raises(moe.MoEError) as e:
        moe.dropout(x, 0.0, torch.zeros(2, dtype=torch.int64))
    assert e.value.status == code and not library.calls


def test_x_itself(library):   # noqa: F811
    for x in (z(4, 16), z(8), z(2, 3, 4, dtype=torch.float32), z(48)[8:]):
        assert moe.dropout(x, 0.0, torch.zeros(2, dtype=torch.int64)) is x and not library.calls
    with pytest.raises(TypeError):
        moe.dropout(z(4, 16, dtype=torch.float16), 0.0, torch.zeros(2, dtype=torch.int64))
