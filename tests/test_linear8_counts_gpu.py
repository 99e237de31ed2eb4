"""The training pass of a projection goes by the counts that its forward saw, whatever the caller's buffer holds when the backward runs."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def moe():
    assert torch.cuda.is_available(), "these tests need a GPU"
    from paper_2206_03382_amd import moe as m
    m.lib()
    return m


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("E,C,K,N", [(5, 300, 200, 328), (17, 453, 776, 1544)])
def test_counts_overwritten_between_forward_and_backward(moe, E, C, K, N, dtype):
    g = torch.Generator(device="cuda").manual_seed(C)
    x, W, dy = (torch.randn(s, generator=g, device="cuda").to(dtype) for s in ((E, C, K), (E, K, N), (E, C, N)))
    fills = torch.randint(-3, C + C // 4, (E,), generator=g, device="cuda", dtype=torch.int32)
    fills[0], fills[1] = 0, 130
    _, kept = moe.expert_linear8_train(x, W, counts=fills.clone())
    want = moe.expert_linear8_backward(dy, kept)
    for later in (torch.full_like(fills, C), torch.zeros_like(fills), fills.flip(0)):
        counts = fills.clone()
        y, kept = moe.expert_linear8_train(x, W, counts=counts)
        counts.copy_(later)                                        # the next micro-batch's routing
        for a, b in zip(moe.expert_linear8_backward(dy, kept), want):
            assert torch.equal(a, b)
    live = torch.arange(C, device="cuda")[None, :] < fills[:, None]
    assert (want[0][~live] == 0).all() and (y[~live] == 0).all() and torch.isfinite(want[1]).all()


def test_backward_of_a_forward_without_counts(moe):
    E, C, K, N = 3, 200, 136, 264
    x, W, dy = torch.randn((E, C, K), device="cuda"), torch.randn((E, K, N), device="cuda"), torch.randn((E, C, N), device="cuda")
    full = torch.full((E,), C, dtype=torch.int32, device="cuda")
    (ya, a), (yb, b) = moe.expert_linear8_train(x, W), moe.expert_linear8_train(x, W, counts=full)
    assert torch.equal(ya, yb)
    for p, q in zip(moe.expert_linear8_backward(dy, a), moe.expert_linear8_backward(dy, b)):
        assert torch.equal(p, q)
