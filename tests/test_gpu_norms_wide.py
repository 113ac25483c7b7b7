"""Norms on the widest rows (up to 16384 in bf16, 8192 in fp32; behind combine too) and column sums over many tokens, against 64 bits.

Tolerances as for the ordinary sizes: one rounding of a stored output, and 1e-5 of the magnitudes that enter for fp32 arithmetic.  A
column sum over T tokens is formed by at most 592 CTAs in a row of at most T / 148 additions each, then over 592 parts by 32 warps:
(T / 148 + 19 + 32) * 2^-24 / 2 of the magnitudes if every rounding went one way, 2e-5 at T 100 000; as roundings are independent
the square root of their number counts, (26 + 8) * 2^-24 = 2e-6, and the 1e-5 holds."""
import pytest
import torch

from test_gpu_norms import ACC, DEV, Case, assignment, backward64, run_backward

pytestmark = pytest.mark.gpu
WIDE = [("bf16", 4104), ("bf16", 8184), ("bf16", 8192), ("bf16", 8200), ("bf16", 12288), ("bf16", 16376), ("bf16", 16384),
        ("f32", 4092), ("f32", 4100), ("f32", 4104), ("f32", 6000), ("f32", 8188), ("f32", 8192)]


@pytest.fixture(scope="module")
def ms():
    from paper_2508_12801_b200 import binding
    assert torch.cuda.is_available()
    return binding


@pytest.mark.parametrize("dtype,d", WIDE)
@pytest.mark.parametrize("T,E,k,gates,post", [(1, 4, 2, 0, True), (400, 8, 8, 3, True), (37, 5, 3, 1, False)])
def test_combine_norm(ms, T, E, k, gates, post, dtype, d):
    c = Case(ms, T, d, dtype, gates=min(gates, T), post=post, E=E, k=k, seed=21, res_scale=0.75)
    idx, slot = (t.to(DEV) for t in assignment(T, E, k, c.C, 22))
    gw = torch.rand(T, k, generator=c.g).to(DEV)
    src, res = c.rand(E, c.C, d), c.rand(T, d)
    y, r_out, h = c.empty(T, d), c.empty(T, d), c.empty(T, d)
    want = torch.empty(T, d, dtype=c.dt, device=DEV)
    ms.combine(c.ctx, src, idx, slot, gw, want)
    ms.combine_norm(c.ctx, src, idx, slot, gw, res, c.norm, y, r_out, h)
    assert torch.equal(y, want)
    ok = ((idx >= 0) & (slot < c.C)).double()
    rows = src.double()[idx.long().clamp(min=0), slot.long().clamp(max=c.C - 1)]
    wt = (ok * gw.double())[:, :, None]
    c.check_forward((rows * wt).sum(1), res, r_out, h, y_mag=(rows * wt).abs().sum(1))
    ms.combine_norm(c.ctx, src, idx, slot, gw, res, c.norm, None, res, want)             # in the residual's own buffer, y not wanted
    assert torch.equal(res, r_out) and torch.equal(want, h)
    assert ms.check_internal(c.ctx) == 0


@pytest.mark.parametrize("dtype,d", WIDE)
@pytest.mark.parametrize("T,opt", [(1, dict(gates=1)), (350, dict(gates=3, res_scale=0.5)), (40, dict(post=False, gates=2)), (333, dict(w_offset=1.0)),
                                   (200, dict(post=False, pre=False)), (170, dict(pre=False, gates=170))], ids=str)
def test_block_norm_and_backward(ms, T, opt, dtype, d):
    c = Case(ms, T, d, dtype, seed=23, **opt)
    y, res = c.rand(T, d), c.rand(T, d)
    r_out, h = c.empty(T, d), c.empty(T, d) if c.w_pre is not None else None
    ms.block_norm(c.ctx, y, res, c.norm, r_out, h)
    c.check_forward(y, res, r_out, h)
    dro, dh = c.rand(T, d), c.rand(T, d) if c.w_pre is not None else None
    for up in (dro, None):
        got = run_backward(ms, c, up, dh, y, r_out)
        ref, mag = backward64(c, up, dh, y, r_out)
        for name, g in got.items():
            assert (g is None) == (name not in ref)
            if g is not None and name in ("dy", "dr"):
                c.close(g, ref[name], mag[name], name)
            elif g is not None:
                assert ((g.double() - ref[name]).abs() <= ACC * mag[name]).all(), name
        again = run_backward(ms, c, up, dh, y, r_out)
        assert all(g is None or torch.equal(g, again[n]) for n, g in got.items())
    assert ms.check_internal(c.ctx) == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gates", [0, 1, 75, 149, 5000])
def test_column_sums_over_many_tokens(ms, gates, dtype):
    T, d = 100003, 264
    c = Case(ms, T, d, dtype, gates=gates, seed=24)
    g = torch.Generator(device=DEV).manual_seed(25)
    y, r_out, dro, dh = (torch.empty(T, d, dtype=c.dt, device=DEV).normal_(generator=g) for _ in range(4))
    dh += 0.5 * r_out                                       # sums that do not cancel
    got = run_backward(ms, c, dro, dh, y, r_out)
    ref, mag = backward64(c, dro, dh, y, r_out)
    for name in ("dw_post", "dw_pre") + (("dgate",) if gates else ()):
        assert ((got[name].double() - ref[name]).abs() <= ACC * mag[name]).all(), name
    assert ms.check_internal(c.ctx) == 0


def test_column_sums_behind_32_bit_offsets(ms):
    """dw_pre over rows of more than 2^31 elements, block by block in 64 bits."""
    T, d = 140000, 16384
    c = Case(ms, T, d, "bf16", post=False, seed=26, E=2, k=1)
    g = torch.Generator(device=DEV).manual_seed(27)
    rows = torch.empty(T, d, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    dr, dw = torch.empty_like(rows), torch.empty(d, device=DEV)
    ms.block_norm_bwd(c.ctx, None, rows, None, rows, c.norm, None, dr, None, None, dw)
    ref = torch.zeros(d, dtype=torch.float64, device=DEV)
    for i in range(0, T, 4000):
        r = rows[i:i + 4000].double()
        ref += (r * r / c.rms(r)).sum(0)                    # every term is positive: the sum is its own magnitude
    assert ((dw.double() - ref).abs() <= ACC * ref).all()
    assert ms.check_internal(c.ctx) == 0
