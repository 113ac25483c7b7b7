"""Products of 8-bit integers whose scales lie far from 1: the product of two scales may leave fp32's range where the result does not."""
import pytest
import torch

from test_gpu_experts8 import BF16, DEV, F64, HALF, context, ints

pytestmark = pytest.mark.gpu

MAX = 3.4028234663852886e38


@pytest.fixture(scope="module")
def ms():
    from paper_2508_12801_b200 import binding
    return binding


def spread(n, lo, hi, gen):
    """fp32 values m 2^e, m in [1, 2), e from lo to hi."""
    return torch.ldexp(1 + torch.rand(n, generator=gen), torch.randint(lo, hi + 1, (n,), generator=gen).float())


# exponents of the rows' and of the columns' scales; quantised bf16 rows have 2^-125 to 2^121
RANGES = [((-80, -66), (-80, -66)), ((-125, -100), (-20, 20)), ((60, 121), (60, 121)), ((-125, 121), (-125, 121)), ((-125, -90), (100, 121)),
          ((-64, 64), (-64, 64)), ((-1, 1), (-1, 1)), ((-140, -120), (30, 121))]


# few rows and many, a row or a column that stands alone, sums that are zero
@pytest.mark.parametrize("E, C, K, N", [(1, 1, 16, 8), (2, 20, 80, 136), (2, 300, 144, 264)])
@pytest.mark.parametrize("rows, cols", RANGES)
def test_product(ms, E, C, K, N, rows, cols):
    g = torch.Generator().manual_seed(C + rows[0] + cols[1])
    xq, wq = ints(g, E, C, K), ints(g, E, N, K)
    xq[0, C // 2] = 0
    wq[E - 1, 3] = 0
    xs, ws = spread(E * C, *rows, g).view(E, C), spread(E * N, *cols, g).view(E, N)
    xs[E - 1, C // 3] = 0
    load = torch.full((E,), C, dtype=torch.int32, device=DEV)
    ctx, y = context(ms, E, C), torch.full((E, C, N), 7.0, dtype=BF16, device=DEV)
    ms.expert_gemm_q8(ctx, xq.to(DEV), xs.to(DEV), wq.to(DEV), ws.to(DEV), load, y, K, N)
    assert ms.check_internal(ctx) == 0
    ref = torch.bmm(xq.to(F64), wq.to(F64).transpose(1, 2)) * xs.to(F64)[:, :, None] * ws.to(F64)[:, None, :]
    got = y.cpu().to(F64)
    over = ref.abs() >= MAX * (1 - 2.0 ** -9)                       # may or must round to infinity
    # one rounding to bf16 behind three to fp32; below 2^-126 half a step is 2^-134, and 2^-150 for each that fp32 took there
    bar = (HALF + 2.0 ** -21) * ref.abs() + 2.0 ** -134 + 2.0 ** -147
    assert ((got - ref).abs() <= bar)[~over].all()
    assert ((got.abs() >= MAX * (1 - 2.0 ** -7)) & (got.sign() == ref.sign()))[over].all()


@pytest.mark.parametrize("E, C, K, N", [(1, 1, 16, 8), (2, 20, 80, 136), (2, 300, 144, 264)])
def test_gated_product(ms, E, C, K, N):
    """g tiny, where silu(g) is g / 2, and u large: h is an ordinary number."""
    g = torch.Generator().manual_seed(C)
    xq, wq = ints(g, E, C, K), ints(g, E, 2 * N, K)
    xq[0, C // 2] = 0
    xs = spread(E * C, -75, -68, g).view(E, C)
    ws = torch.cat([spread(E * N, -75, -62, g).view(E, N), spread(E * N, 100, 119, g).view(E, N)], 1)
    load = torch.full((E,), C, dtype=torch.int32, device=DEV)
    ctx, h = context(ms, E, C), torch.full((E, C, N), 7.0, dtype=BF16, device=DEV)
    ms.expert_glu_q8(ctx, xq.to(DEV), xs.to(DEV), wq.to(DEV), ws.to(DEV), load, h, K, N)
    assert ms.check_internal(ctx) == 0
    pre = torch.bmm(xq.to(F64), wq.to(F64).transpose(1, 2)) * xs.to(F64)[:, :, None] * ws.to(F64)[:, None, :]
    gt, u = pre[..., :N], pre[..., N:]
    ref = torch.nn.functional.silu(gt) * u
    # steps of 2^-24 as for scales near 1 (18); g below 2^-126 is off by 2^-150 and so is half of it, each times u
    bar = (HALF * (1 + HALF) + 2.0 ** -24 * 18) * ref.abs() + 2.0 ** -149 * u.abs() + 2.0 ** -134
    assert ((h.cpu().to(F64) - ref).abs() <= bar).all()


def test_a_value_does_not_depend_on_its_neighbours_scales(ms):
    """A row and a column of usual scales give the same bits whether or not far ones share their tile."""
    for E, C, K, N in ((1, 20, 80, 136), (1, 300, 144, 264)):
        g = torch.Generator().manual_seed(C)
        xq, wq = ints(g, E, C, K).to(DEV), ints(g, E, N, K).to(DEV)
        xs, ws = spread(C, -9, 0, g).view(E, C), spread(N, -12, -3, g).view(E, N)
        load = torch.full((E,), C, dtype=torch.int32, device=DEV)
        ctx, y, z = context(ms, E, C), torch.empty(E, C, N, dtype=BF16, device=DEV), torch.empty(E, C, N, dtype=BF16, device=DEV)
        ms.expert_gemm_q8(ctx, xq, xs.to(DEV), wq, ws.to(DEV), load, y, K, N)
        xs[0, ::7] = 2.0 ** -90
        ws[0, ::5] = 2.0 ** 100
        ms.expert_gemm_q8(ctx, xq, xs.to(DEV), wq, ws.to(DEV), load, z, K, N)
        same = torch.ones(E, C, N, dtype=torch.bool)
        same[0, ::7] = False
        same[0, :, ::5] = False
        assert torch.equal(y.cpu()[same], z.cpu()[same])
