"""Groups chosen by the sum of their two largest where large biases of both signs cancel in it: fp32 has lost there what the sum is made of, and the
choice is still that of 64 bits."""
import pytest
import torch

from test_gpu_topk import check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ms():
    from paper_2508_12801_b200 import binding
    return binding


# a warp a token, and eight lanes a token; groups that are whole lanes and groups that are not
@pytest.mark.parametrize("T", [300, 2601])
@pytest.mark.parametrize("E, k, groups, keep", [(64, 8, 8, 4), (128, 8, 8, 4), (64, 8, 32, 8), (60, 4, 5, 3), (128, 6, 4, 1)])
@pytest.mark.parametrize("large", [1000.0, 2.0 ** 17, 1e30])
@pytest.mark.parametrize("sigmoid", [False, True])
def test_biases_that_cancel(ms, T, E, k, groups, keep, large, sigmoid):
    g = torch.Generator().manual_seed(E + T)
    l = torch.randn(T, E, generator=g)
    bias = torch.full((E,), -large)
    bias[::E // groups] = large                                # one expert of each group
    check(ms, l, bias, k, sigmoid, groups=groups, keep=keep, pairs=True)
    bias += torch.randn(E, generator=g) * 0.05
    check(ms, l, bias, k, sigmoid, groups=groups, keep=keep, pairs=True)


@pytest.mark.parametrize("T", [300, 2601])
def test_experts_that_a_bias_takes_out(ms, T):
    """Biases of -inf and of -1e9 beside ordinary ones, some groups with one expert left or none."""
    g = torch.Generator().manual_seed(T)
    l = torch.randn(T, 64, generator=g)
    for out in (-float("inf"), -1e9):
        bias = torch.randn(64, generator=g) * 0.05
        bias[8:16] = out
        bias[17:24] = out
        bias[::5] = out
        for pairs in (False, True):
            check(ms, l, bias, 6, True, groups=8, keep=4, pairs=pairs)
