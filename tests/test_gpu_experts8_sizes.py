"""Sizes at which the 8-bit forms change kernels: both sides of each rule, and the ends of the shared memory."""
import pytest

import test_gpu_experts8 as base

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ms():
    from paper_2508_12801_b200 import binding
    return binding


# integers: up to 80 rows an expert the weights are the product's M side
@pytest.mark.parametrize("E, C, K, N", [(5, 41, 400, 136), (5, 64, 400, 136), (4, 80, 1040, 264), (4, 81, 1040, 264), (3, 79, 272, 200), (3, 65, 16, 8)])
def test_integer_products(ms, E, C, K, N):
    base.test_product(ms, E, C, K, N)
    base.test_gated_product(ms, E, C, K, N)


# kept activations: few rows up to 64 an expert, and up to 128 from a contraction of 2048 on; two column tiles at a time (256 x 512)
# from a contraction of 4096 on and four tiles a pair (8 * 2 * 21 tiles here, the last column tile alone and narrow)
@pytest.mark.parametrize("E, C, K, f", [(2, 64, 520, 136), (2, 65, 520, 136), (2, 128, 2056, 136), (3, 100, 2048, 72), (3, 65, 2048, 8), (3, 81, 2040, 72),
                                        (2, 129, 2056, 136), (8, 300, 4096, 2568)])
@pytest.mark.parametrize("layout", [0, 1])
def test_kept_activations(ms, E, C, K, f, layout):
    base.test_keeping_forward(ms, E, C, K, f, layout)
    if E < 8:
        base.test_backward_from_what_was_kept(ms, E, C, K, f, layout)
