"""dW over few rows: every slice of every tile ends inside the depth of an MMA, so the two CTAs of a pair hand over a masked slice
each time, and either may run ahead of the other by the whole ring.

Tolerance.  Products of bf16 numbers are exact in fp32; at most 64 of them are summed, each sum off by a step of 2^-23 of the
magnitudes at most: 64 * 2^-23 = 8e-6.  Adding the same again doubles every entry, which is exact."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("E,C,d_in,d_out,fixed", [(128, 40, 512, 512, 40), (128, 40, 512, 512, None), (64, 63, 1024, 776, None), (128, 9, 2048, 512, 9),
                                                  (48, 100, 512, 1024, 100), (100, 200, 256, 512, None)])
def test_masked_slices_one_after_the_other(E, C, d_in, d_out, fixed):
    from paper_2508_12801_b200 import binding as ms
    g = torch.Generator().manual_seed(41)
    rows = torch.full((E,), fixed) if fixed else torch.randint(1, C + 1, (E,), generator=g)
    load = rows.to(torch.int32).to(DEV)
    used = (torch.arange(C)[None, :] < rows[:, None])[:, :, None].to(DEV)
    x, dy = (torch.randn(E, C, w, generator=g).to(torch.bfloat16).to(DEV) for w in (d_in, d_out))
    X, DY = x.double() * used, dy.double() * used
    ref, bar = X.transpose(1, 2) @ DY, 64 * 2.0 ** -23 * -(-C // 64) * (X.abs().transpose(1, 2) @ DY.abs())
    ctx = ms.create(ms.make_params(C, 64, E, 1, capacity=C, io_dtype=ms.BF16), DEV)
    dw = torch.empty(E, d_in, d_out, device=DEV)
    first = None
    for _ in range(30):
        dw.fill_(float("nan"))
        ms.expert_gemm_dw(ctx, x, dy, load, dw, d_in, d_out, 0)
        once = dw.clone()
        ms.expert_gemm_dw(ctx, x, dy, load, dw, d_in, d_out, 0, accumulate=1)
        assert ms.check_internal(ctx) == 0, "a bounded wait gave up"
        if first is None:
            first = once
            assert ((first.double() - ref).abs() <= bar).all()
        assert torch.equal(once, first) and torch.equal(dw, 2 * first)
