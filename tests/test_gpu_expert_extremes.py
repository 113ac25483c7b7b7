"""Expert products at the ends of their range: gates far out in the backward of the activation, infinities, very long contractions,
very wide weights.

Tolerances.  bf16 outputs are rounded by 2^-8 of the value at most.  The tensor cores add 16 products to a sum at a time and cut what they
add off instead of rounding it, each of the 17 numbers below a quarter of a step of the sum: 17 / 4 * 2^-23 of the partial sum at worst.
Over K terms of one sign that is K / 16 such steps at half of the result on average, K / 32 * 17 / 4 * 2^-23: 4.1e-3 at K = 2^18, the longest
contraction that is taken (the average is half of it, half a step of bf16).  fp32 sums are rounded term by term: sqrt(K / 3) * 2^-24
as a root mean square, 1.8e-5 at 2^18; five times that bounds single entries."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def context(E, C, dtype):
    from paper_2508_12801_b200 import binding as ms
    return ms, ms.create(ms.make_params(C, 64, E, 1, capacity=C, io_dtype=ms.BF16 if dtype == "bf16" else ms.F32), DEV)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C", [4, 200])
def test_backward_of_gates_far_out(C, dtype):
    ms, ctx = context(1, C, dtype)
    d, f, dt = 64, 64, DT[dtype]
    g = torch.tensor([-1e30, -500.0, -100.0, -88.5, -87.0, -20.0, -1.28, 0.0, 1e-30, 20.0, 88.5, 100.0, 1e4, 1e30, 3.0, -3.0] * 4, dtype=dt, device=DEV)
    pre = torch.empty(1, C, 2 * f, dtype=dt, device=DEV)
    pre[..., :f], pre[..., f:] = g, 2.0
    dy = torch.zeros(1, C, d, dtype=dt, device=DEV)
    dy[..., 0] = 1.0
    w = torch.zeros(1, f, d, dtype=dt, device=DEV)
    w[..., 0] = 0.5                                               # dh = 0.5 everywhere
    out = torch.empty_like(pre)
    ms.expert_glu_bwd(ctx, dy, w, pre, torch.tensor([C], dtype=torch.int32, device=DEV), out, d, f, 0)
    G = g.double()
    s = torch.sigmoid(G)
    slope = torch.where(G.abs() > 1e3, (G > 0).double(), s + G * s * (1 - s))
    silu = torch.where(G < -1e3, torch.zeros_like(G), G * s)
    half, acc = (2.0 ** -8, 1e-5) if dtype == "bf16" else (0.0, 1e-5)
    for got, ref, mag in ((out[0, :, :f], slope, 1 + (G * s).abs().clamp(max=1e3) * (1 - s)), (out[0, :, f:], 0.5 * silu, 0.5 * silu.abs())):
        assert torch.isfinite(got).all()
        assert ((got.double() - ref).abs() <= half * ref.abs() + acc * mag + 1e-30).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C", [5, 140])
def test_infinities_and_nan_stay_in_their_rows_and_columns(C, dtype):
    ms, ctx = context(2, C, dtype)
    dt, g = DT[dtype], torch.Generator().manual_seed(3)
    x, w = (torch.randn(2, *s, generator=g).to(dt).to(DEV) for s in ((C, 72), (72, 136)))
    x[0, 1, 7], x[1, 3, 70], w[1, 5, 100] = float("inf"), float("nan"), float("-inf")
    y, dw = torch.empty(2, C, 136, dtype=dt, device=DEV), torch.empty(2, 72, 136, device=DEV)
    load = torch.full((2,), C, dtype=torch.int32, device=DEV)
    ms.expert_gemm(ctx, x, w, load, y, 72, 136)
    want = x.double() @ w.double()
    assert torch.equal(torch.isfinite(y), torch.isfinite(want)) and torch.equal(torch.isnan(y), torch.isnan(want))
    dy = torch.randn(2, C, 136, generator=g).to(dt).to(DEV)
    ms.expert_gemm_dw(ctx, x, dy, load, dw, 72, 136)
    want = x.double().transpose(1, 2) @ dy.double()
    assert torch.equal(torch.isfinite(dw), torch.isfinite(want)) and torch.equal(torch.isnan(dw), torch.isnan(want))
    assert ms.check_internal(ctx) == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C", [3, 130])
def test_long_contractions_and_wide_weights(C, dtype):
    ms, ctx = context(1, C, dtype)
    dt, K = DT[dtype], 1 << 18
    g = torch.Generator(device=DEV).manual_seed(4)
    x, w = (torch.empty(1, *s, dtype=dt, device=DEV).uniform_(0.1, 1.0, generator=g) for s in ((C, K), (K, 72)))
    load = torch.tensor([C - 1], dtype=torch.int32, device=DEV)
    y = torch.empty(1, C, 72, dtype=dt, device=DEV)
    ms.expert_gemm(ctx, x, w, load, y, K, 72)
    ref = x[0, :C - 1].double() @ w[0].double()
    bar = 2.0 ** -8 + K / 32 * 17 / 4 * 2.0 ** -23 if dtype == "bf16" else 5 * (K / 3) ** 0.5 * 2.0 ** -24
    assert ((y[0, :C - 1].double() - ref).abs() <= bar * ref).all() and (y[0, C - 1] == 0).all()
    # the same weight as 72 -> 2^18: every column of a short contraction
    xs, yw = x[:, :, :72].contiguous(), torch.empty(1, C, K, dtype=dt, device=DEV)
    ms.expert_gemm(ctx, xs, w, load, yw, 72, K, 1)
    ref = xs[0, :C - 1].double() @ w[0].double().T
    assert ((yw[0, :C - 1].double() - ref).abs() <= (2.0 ** -8 if dtype == "bf16" else 0) * ref + 1e-5 * ref).all() and (yw[0, C - 1] == 0).all()
    dw = torch.empty(1, K, 72, device=DEV)
    ms.expert_gemm_dw(ctx, x, y, load, dw, K, 72)
    ref = x[0, :C - 1].double().T @ y[0, :C - 1].double()
    assert ((dw[0].double() - ref).abs() <= 1e-5 * ref).all()
    assert ms.check_internal(ctx) == 0


def test_contractions_that_lose_bf16_are_refused():
    """Beyond 2^18 terms the cut-off sums are further off than the output's own rounding; fp32 I/O has no such limit."""
    for dtype, refused in (("bf16", True), ("f32", False)):
        ms, ctx = context(1, 2, dtype)
        dt, K = DT[dtype], (1 << 18) + 8
        z = lambda *s: torch.zeros(*s, dtype=dt, device=DEV)  # noqa: E731
        load = torch.tensor([2], dtype=torch.int32, device=DEV)
        calls = [lambda: ms.expert_gemm(ctx, z(1, 2, K), z(1, K, 8), load, z(1, 2, 8), K, 8),
                 lambda: ms.expert_glu(ctx, z(1, 2, K), z(1, K, 16), load, None, z(1, 2, 8), K, 8),
                 lambda: ms.expert_glu_bwd(ctx, z(1, 2, K), z(1, 8, K), z(1, 2, 16), load, z(1, 2, 16), K, 8)]
        for call in calls:
            if refused:
                with pytest.raises(ms.MaxScoreError) as e:
                    call()
                assert e.value.status == 6
            else:
                call()
        ms.expert_gemm(ctx, z(1, 2, 8), z(1, 8, K), load, z(1, 2, K), 8, K)                    # as many columns are fine
        ms.expert_gemm_dw(ctx, z(1, 2, K), z(1, 2, 8), load, torch.zeros(1, K, 8, device=DEV), K, 8)
        assert ms.check_internal(ctx) == 0
