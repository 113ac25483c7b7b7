"""How exact dW is over many rows: fp32 sums, whatever the number of rows.

Tolerance, for rows of one sign (every partial sum is below the result).  Sums over 256 rows are formed 16 rows at a time, and each
time the sum is cut off below its 24th bit, by up to one step of 2^-23 of the partial sum, which is 17/32 of the whole on average:
16 * 17/32 * 2^-23 = 1.0e-6.  (The products, 16 bits each, are cut two bits further down: 2^-25 of a sum of at most 256 of them is below
half of their last bit, so they come in whole but for the smallest ones.)
The n partial sums are then added with rounding, half a step of 2^-24 of the sum so far each: (n + 1) / 2 * 2^-24 at worst, and as a
root mean square, the roundings being independent, sqrt(n / 3) * 2^-24 / sqrt(3).  fp32 inputs are summed row by row with rounding:
sqrt(rows / 3) * 2^-24 as a root mean square."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def inputs(E, C, d_in, d_out, dtype, sign):
    from paper_2508_12801_b200 import binding as ms
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator(device=DEV).manual_seed(C)
    x, dy = (torch.empty(E, C, w, device=DEV, dtype=dt).normal_(generator=g) for w in (d_in, d_out))
    if sign:
        x, dy = x.abs(), dy.abs()
    load = torch.tensor([C, C - 3, C // 2 + 1, 0][:E], dtype=torch.int32, device=DEV)
    ref = torch.stack([x[e, :n].double().T @ dy[e, :n].double() for e, n in enumerate(load.tolist())])
    ctx = ms.create(ms.make_params(C, 64, E, 1, capacity=C, io_dtype=ms.BF16 if dtype == "bf16" else ms.F32), DEV)
    return ms, ctx, x, dy, load, ref


def bar(n, dtype):
    if dtype == "f32":
        return math.sqrt(n / 3) * 2 ** -24
    return min(16, -(-n // 16)) * 17 / 32 * 2 ** -23 + math.sqrt(-(-n // 256)) / 3 * 2 ** -24


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("C,d_in,d_out", [(256, 264, 520), (257, 256, 512), (512, 136, 264), (1023, 256, 256), (2560, 512, 256), (4096, 64, 776),
                                          (5000, 256, 512), (20000, 128, 256)])
def test_sums_of_one_sign_keep_fp32(C, d_in, d_out, layout, dtype):
    ms, ctx, x, dy, load, ref = inputs(4, C, d_in, d_out, dtype, sign=True)
    dw = torch.full((4, d_in, d_out) if layout == 0 else (4, d_out, d_in), float("nan"), device=DEV)
    ms.expert_gemm_dw(ctx, x, dy, load, dw, d_in, d_out, layout)
    got = dw.double() if layout == 0 else dw.double().transpose(1, 2)
    for e, n in enumerate(load.tolist()):
        if n == 0:
            assert (got[e] == 0).all()
            continue
        rel = float(((got[e] - ref[e]) / ref[e]).square().mean().sqrt())
        assert rel <= bar(n, dtype), f"expert {e}, {n} rows: {rel:.2e}, bar {bar(n, dtype):.2e}"
    assert ms.check_internal(ctx) == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C,d_in,d_out", [(40, 256, 512), (256, 72, 520), (300, 256, 264), (4500, 264, 256)])
def test_adding_rounds_once(C, d_in, d_out, dtype):
    """accumulate adds the call's own sum to what is there, with one rounding."""
    ms, ctx, x, dy, load, _ = inputs(4, C, d_in, d_out, dtype, sign=False)
    once = torch.empty(4, d_in, d_out, device=DEV)
    ms.expert_gemm_dw(ctx, x, dy, load, once, d_in, d_out, 0)
    old = torch.randn(4, d_in, d_out, device=DEV) * 30
    flat = torch.full((once.numel() + 64,), 7.0, device=DEV)
    dw = flat[:once.numel()].view_as(once)
    dw.copy_(old)
    ms.expert_gemm_dw(ctx, x, dy, load, dw, d_in, d_out, 0, accumulate=1)
    assert torch.equal(dw, old + once) and (flat[once.numel():] == 7.0).all()
    assert ms.check_internal(ctx) == 0
