"""Experts in 8-bit integers and expert activations kept in 8 bits against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF16, F64 = torch.bfloat16, torch.float64
HALF = 2.0 ** -8                      # half a step of bf16, relative


@pytest.fixture(scope="module")
def ms():
    from paper_2508_12801_b200 import binding
    return binding


def context(ms, E, C, d=64, T=None, k=1):
    """A context whose buffers are [E, C]: the calls take everything else from their arguments."""
    return ms.create(ms.make_params(T or C, d, E, k, capacity=C, io_dtype=ms.BF16), DEV)


def quant64(x):
    """Integers and scale of rows x [..., n] by the definition: fp32 quotients, the product rounded once."""
    x = x.to(F64).numpy()
    amax = np.abs(x).max(axis=-1, keepdims=True)
    with np.errstate(all="ignore"):
        fine = (amax >= 2.0 ** -118) & np.isfinite(amax)
        inv = np.where(fine, (np.float32(127) / amax.astype(np.float32)), np.float32(0)).astype(np.float32)
        scale = np.where(fine, amax.astype(np.float32) / np.float32(127), np.float32(0)).astype(np.float32)
        q = np.where(fine, np.rint(x * inv.astype(np.float64)), 0.0)
    scale = np.where(np.isfinite(amax), scale, np.float32(np.nan))
    return torch.from_numpy(q).to(torch.int8), torch.from_numpy(scale[..., 0].astype(np.float32))


def same(a, b):
    return torch.equal(a.cpu().nan_to_num(-9.0), b.nan_to_num(-9.0))


def rows_in_use(load, E, C):
    return torch.arange(C)[None, :] < load.clamp(0, C)[:, None]


def some_load(E, C, gen):
    load = torch.randint(0, C + 1, (E,), generator=gen, dtype=torch.int32)
    load[0] = C
    if E > 1:
        load[1] = 0
    if E > 2:
        load[2] = C + 3                # more than fits
    if E > 3:
        load[3] = -1
    return load


@pytest.mark.parametrize("E, C, width", [(1, 1, 16), (4, 7, 48), (3, 33, 512), (5, 9, 1040), (2, 5, 2064), (2, 3, 4096), (2, 2, 4112), (1, 2, 20000)])
def test_quantised_rows(ms, E, C, width):
    g = torch.Generator().manual_seed(width)
    x = (torch.randn(E, C, width, generator=g) * torch.exp(torch.randn(E, C, 1, generator=g) * 4)).to(BF16)
    x[0, 0, width // 2] = x[0, 0].abs().max() * 1.5                        # an outlier
    load = some_load(E, C, g)
    if C > 4:
        x[0, 1] = 0
        x[0, 2] = 2.0 ** -119                                              # too small to divide by
        x[0, 3, 5] = float("inf")
        x[0, 4, 3] = float("nan")
    ctx = context(ms, E, C)
    q, s = torch.full((E, C, width), 77, dtype=torch.int8, device=DEV), torch.full((E, C), 7.0, device=DEV)
    ms.expert_quant(ctx, x.to(DEV), load.to(DEV), q, s, width)
    used = rows_in_use(load, E, C)
    wq, wsc = quant64(torch.where(used[..., None], x, torch.zeros_like(x)))
    assert same(q, wq) and same(s, wsc)


def test_halves_go_to_the_even_number(ms):
    """amax 127 makes inv and scale 1: the values are their own integers, halves round to even."""
    x = torch.tensor([127.0, 0.5, 1.5, 2.5, -0.5, -1.5, -126.5, 63.5, -0.0, 0.25, 126.5, -127.0, 3.5, 4.5, -3.5, 1e-30]).to(BF16)[None, None]
    ctx = context(ms, 1, 1)
    q, s = torch.empty(1, 1, 16, dtype=torch.int8, device=DEV), torch.empty(1, 1, device=DEV)
    ms.expert_quant(ctx, x.to(DEV), torch.ones(1, dtype=torch.int32, device=DEV), q, s, 16)
    assert q.flatten().tolist() == [127, 0, 2, 2, 0, -2, -126, 64, 0, 0, 126, -127, 4, 4, -4, 0] and s.item() == 1.0


@pytest.mark.parametrize("T, d, E, k, C", [(1, 16, 4, 2, 1), (50, 64, 8, 3, 20), (300, 1040, 5, 2, 100), (33, 4112, 33, 5, 9)])
def test_dispatch(ms, T, d, E, k, C):
    g = torch.Generator().manual_seed(T)
    x = torch.randn(T, d, generator=g).to(BF16)
    if T > 3:
        x[1] = 0
        x[2, 0] = float("nan")
    idx = torch.rand(T, E, generator=g).topk(k, 1).indices.sort(1).values.to(torch.int32)
    if T > 5:
        idx[5, k - 1] = -1                                                 # an empty pair
    ctx = ms.create(ms.make_params(T, d, E, k, capacity=max(C, -(-T * k // E)), io_dtype=ms.BF16), DEV)
    C = ctx.capacity
    i = idx.to(DEV)
    slot, tok, load = torch.full_like(i, -1), torch.empty(E, C, dtype=torch.int32, device=DEV), torch.empty(E, dtype=torch.int32, device=DEV)
    ms.index_build(ctx, i, slot, tok, load)
    q, s = torch.full((E, C, d), 77, dtype=torch.int8, device=DEV), torch.full((E, C), 7.0, device=DEV)
    ms.dispatch_q8(ctx, x.to(DEV), i, slot, tok, q, s)
    wq, wsc = quant64(x)
    t = tok.cpu().long()
    there = t >= 0
    t = t.clamp(min=0)
    assert same(q, torch.where(there[..., None], wq[t], torch.zeros_like(wq[t])))
    assert same(s, torch.where(there, wsc[t], torch.zeros_like(wsc[t])))


@pytest.mark.parametrize("E, d_in, d_out", [(1, 16, 8), (3, 48, 72), (2, 144, 200), (2, 1040, 64), (4, 512, 136)])
@pytest.mark.parametrize("layout", [0, 1])
def test_quantised_weights(ms, E, d_in, d_out, layout):
    g = torch.Generator().manual_seed(d_in)
    w = (torch.randn(E, d_out, d_in, generator=g) * torch.exp(torch.randn(E, d_out, 1, generator=g))).to(BF16)
    w[0, 3] = 0
    w[0, 5, 1] = float("inf")
    ctx = context(ms, E, 4)
    q, s = torch.full((E, d_out, d_in), 77, dtype=torch.int8, device=DEV), torch.full((E, d_out), 7.0, device=DEV)
    src = w if layout == 1 else w.transpose(1, 2)
    ms.expert_quant_weight(ctx, src.contiguous().to(DEV), q, s, d_in, d_out, layout)
    wq, wsc = quant64(w)
    assert same(q, wq) and same(s, wsc)


def ints(gen, *shape):
    return torch.randint(-128, 128, shape, generator=gen, dtype=torch.int8)


# E, C, d_in, d_out: rows up to 128 take one kernel, more the other; tiles of 128 and 256 columns, slices of 128
PRODUCTS = [(1, 1, 16, 8), (4, 3, 48, 24), (3, 16, 128, 128), (5, 40, 400, 136), (2, 128, 1040, 264), (33, 9, 256, 72), (2, 129, 128, 256), (3, 300, 272, 520),
            (2, 513, 1040, 264), (1, 257, 64, 8), (9, 600, 512, 1024), (2, 700, 8192, 1032)]


@pytest.mark.parametrize("E, C, K, N", PRODUCTS)
def test_product(ms, E, C, K, N):
    g = torch.Generator().manual_seed(K + N)
    xq, wq = ints(g, E, C, K), ints(g, E, N, K)
    xs, ws = torch.rand(E, C, generator=g) + 0.01, torch.rand(E, N, generator=g) * 0.01 + 1e-5
    load = some_load(E, C, g)
    used = rows_in_use(load, E, C)
    dirty = torch.where(used, xs, torch.full_like(xs, float("nan")))       # what lies behind the load is never used
    ctx = context(ms, E, C)
    y = torch.full((E, C, N), 7.0, dtype=BF16, device=DEV)
    ms.expert_gemm_q8(ctx, xq.to(DEV), dirty.to(DEV), wq.to(DEV), ws.to(DEV), load.to(DEV), y, K, N)
    assert ms.check_internal(ctx) == 0
    ref = torch.bmm(xq.to(DEV).to(F64), wq.to(DEV).to(F64).transpose(1, 2)).cpu() * (xs.to(F64)[:, :, None] * ws.to(F64)[:, None, :]) * used[..., None]
    # one rounding to bf16 of a product of three fp32 values: the integer sum, and the two scales, each rounded once
    assert ((y.cpu().to(F64) - ref).abs() <= (HALF + 2.0 ** -21) * ref.abs()).all()
    assert (y.cpu()[~used] == 0).all()
    again = torch.empty_like(y)
    ms.expert_gemm_q8(ctx, xq.to(DEV), dirty.to(DEV), wq.to(DEV), ws.to(DEV), load.to(DEV), again, K, N)
    assert torch.equal(y, again)


@pytest.mark.parametrize("E, C, K, N", PRODUCTS)
def test_gated_product(ms, E, C, K, N):
    g = torch.Generator().manual_seed(K + N + 1)
    xq, wq = ints(g, E, C, K), ints(g, E, 2 * N, K)
    xs, ws = torch.rand(E, C, generator=g) * 0.02 + 0.001, (torch.rand(E, 2 * N, generator=g) + 0.1) * 0.02 / K ** 0.5
    load = some_load(E, C, g)
    used = rows_in_use(load, E, C)
    ctx = context(ms, E, C)
    h = torch.full((E, C, N), 7.0, dtype=BF16, device=DEV)
    ms.expert_glu_q8(ctx, xq.to(DEV), xs.to(DEV), wq.to(DEV), ws.to(DEV), load.to(DEV), h, K, N)
    assert ms.check_internal(ctx) == 0
    pre = torch.bmm(xq.to(DEV).to(F64), wq.to(DEV).to(F64).transpose(1, 2)).cpu() * (xs.to(F64)[:, :, None] * ws.to(F64)[:, None, :])
    gt, u = pre[..., :N], pre[..., N:]
    ref = torch.nn.functional.silu(gt) * u * used[..., None]
    # g and u are off by three steps of 2^-24; silu's relative slope is at most 1 + |g|; its exponential by 2 + 1.2 |g| steps of 2^-23 and
    # the quotient by 2: below 2^-24 (3 + 3 (1 + |g|) + 4 + 2.4 |g| + 4 + 4)
    tol = HALF * (1 + HALF) + 2.0 ** -24 * (18 + 6 * gt.abs())
    assert ((h.cpu().to(F64) - ref).abs() <= tol * ref.abs() + 1e-37).all()


@pytest.mark.parametrize("C", [2, 130])
@pytest.mark.parametrize("a, b", [(-128, -128), (127, -128), (127, 127)])
def test_longest_sums(ms, C, a, b):
    K, N = (1 << 17) - 16, 16
    xq = torch.full((1, C, K), a, dtype=torch.int8, device=DEV)
    wq = torch.full((1, N, K), b, dtype=torch.int8, device=DEV)
    wq[0, 1::2, ::2] = 0
    one = torch.ones(1, max(C, N), device=DEV)
    y = torch.empty(1, C, N, dtype=BF16, device=DEV)
    ctx = context(ms, 1, C)
    ms.expert_gemm_q8(ctx, xq, one[:, :C].contiguous(), wq, one[:, :N].contiguous(), torch.full((1,), C, dtype=torch.int32, device=DEV), y, K, N)
    full = torch.tensor([a * b * K, a * b * K // 2], dtype=F64).repeat(N // 2)
    assert torch.equal(y.cpu(), full.to(torch.float32).to(BF16).expand(1, C, N))


def test_not_finite_scales_reach_their_rows_and_columns_only(ms):
    for C in (4, 140):
        g = torch.Generator().manual_seed(C)
        xq, wq = ints(g, 2, C, 32), ints(g, 2, 24, 32)
        xs, ws = torch.ones(2, C), torch.ones(2, 24)
        xs[0, 1] = float("nan")
        ws[1, 5] = float("nan")
        y = torch.empty(2, C, 24, dtype=BF16, device=DEV)
        ctx = context(ms, 2, C)
        ms.expert_gemm_q8(ctx, xq.to(DEV), xs.to(DEV), wq.to(DEV), ws.to(DEV), torch.full((2,), C, dtype=torch.int32, device=DEV), y, 32, 24)
        want = torch.zeros(2, C, 24, dtype=torch.bool)
        want[0, 1] = True
        want[1, :, 5] = True
        assert torch.equal(y.cpu().isnan(), want)


# ---- activations kept in 8 bits ------------------------------------------------------------------------------------------

def keep_views(keep, E, C, f):
    w = -(-f // 32) * 32
    at = -(-E * C * 2 * w // 256) * 256
    return keep[:E * C * 2 * w].view(torch.int8).view(E, C, 2, w), keep[at:].view(torch.float32).view(E, 2, w // 32, C).permute(0, 3, 1, 2)


def kept_values(keep, E, C, f):
    q, s = keep_views(keep.cpu(), E, C, f)
    return (q.to(F64) * s.to(F64).repeat_interleave(32, 3))[..., :f]


# E, C, d_in, d_ff
KEPT = [(1, 1, 8, 8), (4, 3, 64, 40), (3, 16, 136, 64), (5, 40, 256, 104), (2, 128, 520, 136), (2, 129, 64, 64), (3, 300, 136, 168), (2, 513, 520, 264),
        (1, 257, 64, 8), (9, 600, 256, 512), (2, 300, 4096, 136)]


@pytest.mark.parametrize("E, C, K, f", KEPT)
@pytest.mark.parametrize("layout", [0, 1])
def test_keeping_forward(ms, E, C, K, f, layout):
    g = torch.Generator().manual_seed(K + f)
    x, w = torch.randn(E, C, K, generator=g).to(BF16), (torch.randn(E, K, 2 * f, generator=g) * K ** -0.5).to(BF16)
    load = some_load(E, C, g)
    used = rows_in_use(load, E, C)
    x[~used] = float("nan")                                                # never used
    x[0, 0] = 0
    ctx = context(ms, E, C)
    keep = torch.full((ms.keep8_bytes(ctx, f),), 77, dtype=torch.uint8, device=DEV)
    h = torch.full((E, C, f), 7.0, dtype=BF16, device=DEV)
    wd = (w if layout == 0 else w.transpose(1, 2)).contiguous().to(DEV)
    ms.expert_glu_keep8(ctx, x.to(DEV), wd, load.to(DEV), keep, h, K, f, layout)
    assert ms.check_internal(ctx) == 0
    plain, h2 = torch.empty(E, C, 2 * f, dtype=BF16, device=DEV), torch.empty_like(h)
    ms.expert_glu(ctx, x.to(DEV), wd, load.to(DEV), plain, h2, K, f, layout)
    assert torch.equal(h, h2)                                              # h is expert_glu's, bit for bit
    x0 = torch.where(used[..., None], x, torch.zeros_like(x)).to(DEV).to(F64)
    pre = torch.bmm(x0, w.to(DEV).to(F64)).cpu().view(E, C, 2, f)
    mag = torch.bmm(x0.abs(), w.to(DEV).to(F64).abs()).cpu().view(E, C, 2, f)
    off = 1e-5 * mag                                                       # fp32 sums on the tensor cores
    q, s = keep_views(keep.cpu(), E, C, f)
    blocks = torch.nn.functional.pad(pre, (0, q.shape[3] - f)).unflatten(3, (-1, 32))
    boff = torch.nn.functional.pad(off, (0, q.shape[3] - f)).unflatten(3, (-1, 32)).amax(4)
    amax = blocks.abs().amax(4)
    assert ((s.to(F64) * 127 - amax).abs() <= boff + 2.0 ** -22 * amax)[used].all()
    # half a step, the sum's error, and the steps of inv, scale and their product
    val = kept_values(keep, E, C, f)
    half = (s.to(F64) * (0.5 + 2.0 ** -15)).repeat_interleave(32, 3)[..., :f]
    assert ((val - pre).abs() <= half + off)[used].all()
    assert (q[0, 0] == 0).all() and (s[0, 0] == 0).all()
    top = q.unflatten(3, (-1, 32)).abs().amax(4)
    assert (top[used] == torch.where(s[used] > 0, 127, 0)).all()           # the largest of a block is 127 steps
    assert (q[~used] == 77).all()                                          # rows that are not in use are not written
    assert (s.contiguous().view(torch.int32)[~used] == 0x4d4d4d4d).all()


@pytest.mark.parametrize("E, C, K, f", KEPT)
@pytest.mark.parametrize("layout", [0, 1])
def test_backward_from_what_was_kept(ms, E, C, K, f, layout):
    g = torch.Generator().manual_seed(K + f + 1)
    dy, w = torch.randn(E, C, K, generator=g).to(BF16), (torch.randn(E, f, K, generator=g) * K ** -0.5).to(BF16)
    load = some_load(E, C, g)
    used = rows_in_use(load, E, C)
    dy[~used] = float("nan")
    ctx = context(ms, E, C)
    keep = torch.full((ms.keep8_bytes(ctx, f),), 0xff, dtype=torch.uint8)  # scales that are NaN
    q, s = keep_views(keep, E, C, f)
    q[used] = torch.randint(-127, 128, q.shape, generator=g, dtype=torch.int8)[used]
    rand = torch.rand(s.shape, generator=g) * 0.05
    s.copy_(torch.where(used[:, :, None, None], rand, s))
    gt, u = kept_values(keep, E, C, f).unbind(2)
    dpre, h = torch.full((E, C, 2 * f), 7.0, dtype=BF16, device=DEV), torch.full((E, C, f), 7.0, dtype=BF16, device=DEV)
    wd = (w if layout == 0 else w.transpose(1, 2)).contiguous().to(DEV)
    ms.expert_glu_bwd_keep8(ctx, dy.to(DEV), wd, keep.to(DEV), load.to(DEV), dpre, h, K, f, layout)
    assert ms.check_internal(ctx) == 0
    gt, u = (torch.where(used[..., None], t, torch.zeros_like(t)) for t in (gt, u))
    d0 = torch.where(used[..., None], dy, torch.zeros_like(dy)).to(DEV).to(F64)
    dh, mag = (torch.bmm(a, b.transpose(1, 2)).cpu() for a, b in ((d0, w.to(DEV).to(F64)), (d0.abs(), w.to(DEV).to(F64).abs())))
    sg = torch.sigmoid(gt)
    tol = HALF * (1 + HALF) + 2.0 ** -24 * (24 + 8 * gt.abs())             # as in the gated product; 1 + g (1 - s) adds a sum and a product
    a = u * sg * (1 + gt * (1 - sg))
    # where 1 + g (1 - s) cancels (g near -1.28) its terms count
    a_mag = u.abs() * sg * (1 + gt.abs() * (1 - sg))
    for got, factor, fmag in ((dpre[..., :f], a, a_mag), (dpre[..., f:], gt * sg, (gt * sg).abs())):
        ref = dh * factor
        bar = HALF * (1 + HALF) * ref.abs() + (1e-5 * mag + 2.0 ** -24 * (24 + 8 * gt.abs()) * dh.abs()) * fmag + 1e-37
        assert ((got.cpu().to(F64) - ref).abs() <= bar).all()
    ref = gt * sg * u
    assert ((h.cpu().to(F64) - ref).abs() <= tol * ref.abs() + 1e-37).all()
    assert (dpre.cpu()[~used] == 0).all() and (h.cpu()[~used] == 0).all()
    alone = torch.full_like(dpre, 7.0)
    ms.expert_glu_bwd_keep8(ctx, dy.to(DEV), wd, keep.to(DEV), load.to(DEV), alone, None, K, f, layout)
    assert torch.equal(alone, dpre)


def test_not_finite_activations_spoil_their_block_only(ms):
    for C in (4, 140):
        E, K, f = 2, 64, 72
        g = torch.Generator().manual_seed(C)
        x, w = torch.randn(E, C, K, generator=g).to(BF16), torch.randn(E, K, 2 * f, generator=g).to(BF16)
        w[0, 3, 40] = float("inf")                                         # g, second block of expert 0
        w[1, 2, f + 70] = float("nan")                                     # u, third block of expert 1
        ctx = context(ms, E, C)
        load = torch.full((E,), C, dtype=torch.int32, device=DEV)
        keep, h = torch.empty(ms.keep8_bytes(ctx, f), dtype=torch.uint8, device=DEV), torch.empty(E, C, f, dtype=BF16, device=DEV)
        ms.expert_glu_keep8(ctx, x.to(DEV), w.to(DEV), load, keep, h, K, f)
        q, s = keep_views(keep.cpu(), E, C, f)
        want = torch.zeros(E, C, 2, 3, dtype=torch.bool)
        want[0, :, 0, 1] = x[0, :, 3] != 0
        want[1, :, 1, 2] = True
        assert torch.equal(s.isnan(), want) and (q.unflatten(3, (3, 32))[want] == 0).all()


def test_sizes_beyond_32_bits(ms):
    """A kept buffer of more than 2^32 bytes and integer rows of more than 2^31: the last rows are where they belong."""
    E, C, K, f = 2, 1100000, 64, 1024
    ctx = context(ms, E, C)
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.zeros(E, C, K, dtype=BF16, device=DEV)
    x[:, -300:] = torch.randn(E, 300, K, generator=g, device=DEV).to(BF16)
    w = (torch.randn(E, K, 2 * f, generator=g, device=DEV) * K ** -0.5).to(BF16)
    load = torch.full((E,), C, dtype=torch.int32, device=DEV)
    keep, h = torch.empty(ms.keep8_bytes(ctx, f), dtype=torch.uint8, device=DEV), torch.empty(E, C, f, dtype=BF16, device=DEV)
    ms.expert_glu_keep8(ctx, x, w, load, keep, h, K, f)
    q, s = keep_views(keep, E, C, f)
    val = q[:, -300:].to(F64) * s[:, -300:].to(F64).repeat_interleave(32, 3)
    pre = torch.bmm(x[:, -300:].to(F64), w.to(F64)).view(E, 300, 2, f)
    assert ((val - pre).abs() <= 0.51 * s[:, -300:].to(F64).repeat_interleave(32, 3) + 1e-4).all()
    assert (q[:, :-300:1000] == 0).all()
    xq, xs = torch.empty(E, C, f, dtype=torch.int8, device=DEV), torch.empty(E, C, device=DEV)
    ms.expert_quant(ctx, h, load, xq, xs, f)
    want, scale = quant64(h[1, -300:].cpu())
    assert torch.equal(xq[1, -300:].cpu(), want) and torch.equal(xs[1, -300:].cpu(), scale)
    dy = torch.zeros(E, C, K, dtype=BF16, device=DEV)
    dy[:, -300:] = 1.0
    wd = (torch.randn(E, f, K, generator=g, device=DEV) * f ** -0.5).to(BF16)
    dpre, h2 = torch.empty(E, C, 2 * f, dtype=BF16, device=DEV), torch.empty(E, C, f, dtype=BF16, device=DEV)
    ms.expert_glu_bwd_keep8(ctx, dy, wd, keep, load, dpre, h2, K, f)
    assert ms.check_internal(ctx) == 0
    gt, u = val.unbind(2)
    ref = torch.nn.functional.silu(gt) * u
    assert ((h2[:, -300:].to(F64) - ref).abs() <= 2 * HALF * ref.abs() + 1e-6).all()
    dh = torch.bmm(dy[:, -300:].to(F64), wd.to(F64).transpose(1, 2))
    ref = dh * torch.nn.functional.silu(gt)
    assert ((dpre[:, -300:, f:].to(F64) - ref).abs() <= 2 * HALF * ref.abs() + 1e-4).all()
    assert (dpre[:, :-300:1000] == 0).all()


def test_graph_streams_and_two_contexts(ms):
    """A captured int8 block and training step replayed with new inputs; two contexts at once on two streams."""
    T, d, E, k, f = 600, 128, 8, 2, 96
    g = torch.Generator().manual_seed(2)
    r = lambda *s: torch.randn(*s, generator=g).to(BF16).to(DEV)  # noqa: E731
    ctxs = [ms.create(ms.make_params(T, d, E, k, capacity=T, io_dtype=ms.BF16), DEV) for _ in range(2)]
    C = T
    idx = torch.rand(T, E, generator=g).topk(k, 1).indices.sort(1).values.to(torch.int32).to(DEV)
    slot, tok, load = torch.empty_like(idx), torch.empty(E, C, dtype=torch.int32, device=DEV), torch.empty(E, dtype=torch.int32, device=DEV)
    ms.index_build(ctxs[0], idx, slot, tok, load)
    w_up, w_down = r(E, d, 2 * f), r(E, f, d)
    i8 = lambda *s: torch.empty(*s, dtype=torch.int8, device=DEV)  # noqa: E731
    uq, us, dq, ds = i8(E, 2 * f, d), torch.empty(E, 2 * f, device=DEV), i8(E, d, f), torch.empty(E, d, device=DEV)
    ms.expert_quant_weight(ctxs[0], w_up, uq, us, d, 2 * f)
    ms.expert_quant_weight(ctxs[0], w_down, dq, ds, f, d)

    class Bufs:
        def __init__(self):
            self.xq, self.xs, self.h, self.hq, self.hs = i8(E, C, d), torch.empty(E, C, device=DEV), r(E, C, f), i8(E, C, f), torch.empty(E, C, device=DEV)
            self.y, self.x, self.dpre, self.h2 = r(E, C, d), r(E, C, d), r(E, C, 2 * f), r(E, C, f)
            self.keep = torch.empty(ms.keep8_bytes(ctxs[0], f), dtype=torch.uint8, device=DEV)

    def step(ctx, x, b, stream=None):
        ms.dispatch_q8(ctx, x, idx, slot, tok, b.xq, b.xs, stream=stream)
        ms.expert_glu_q8(ctx, b.xq, b.xs, uq, us, load, b.h, d, f, stream=stream)
        ms.expert_quant(ctx, b.h, load, b.hq, b.hs, f, stream=stream)
        ms.expert_gemm_q8(ctx, b.hq, b.hs, dq, ds, load, b.y, f, d, stream=stream)
        ms.dispatch(ctx, x, idx, slot, tok, b.x, stream=stream)
        ms.expert_glu_keep8(ctx, b.x, w_up, load, b.keep, b.h, d, f, stream=stream)
        ms.expert_glu_bwd_keep8(ctx, b.x, w_down, b.keep, load, b.dpre, b.h2, d, f, stream=stream)

    xs = [r(T, d), r(T, d)]
    eager = [Bufs(), Bufs()]
    for x, b in zip(xs, eager):
        step(ctxs[0], x, b)
    torch.cuda.synchronize()
    live, b, graph = xs[0].clone(), Bufs(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(ctxs[0], live, b)
    for x, e in zip(xs, eager):
        live.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        for n in ("y", "dpre", "h2"):
            assert torch.equal(getattr(b, n), getattr(e, n)), n
    both = [Bufs(), Bufs()]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for c, x, b, st in zip(ctxs, xs, both, streams):
        step(c, x, b, stream=st)
    torch.cuda.synchronize()
    for b, e in zip(both, eager):
        for n in ("y", "dpre", "h2"):
            assert torch.equal(getattr(b, n), getattr(e, n)), n


def test_int8_experts_approach_the_bf16_experts(ms):
    """The whole serving block against the bf16 experts: off by what 8 bits lose, 2 ** -8 of amax a value, averaged over the sums."""
    T, d, E, k, f = 512, 256, 8, 2, 128
    g = torch.Generator().manual_seed(3)
    x = torch.randn(T, d, generator=g).to(BF16).to(DEV)
    w_up, w_down = ((torch.randn(E, *s, generator=g) * s[0] ** -0.5).to(BF16).to(DEV) for s in ((d, 2 * f), (f, d)))
    ctx = ms.create(ms.make_params(T, d, E, k, capacity=T, io_dtype=ms.BF16), DEV)
    idx = torch.rand(T, E, generator=g).topk(k, 1).indices.sort(1).values.to(torch.int32).to(DEV)
    new = lambda *s, dtype=BF16: torch.empty(*s, dtype=dtype, device=DEV)  # noqa: E731
    i8, f32 = torch.int8, torch.float32
    slot, tok, load = torch.empty_like(idx), new(E, T, dtype=torch.int32), new(E, dtype=torch.int32)
    ms.index_build(ctx, idx, slot, tok, load)
    uq, us, dq, ds = new(E, 2 * f, d, dtype=i8), new(E, 2 * f, dtype=f32), new(E, d, f, dtype=i8), new(E, d, dtype=f32)
    ms.expert_quant_weight(ctx, w_up, uq, us, d, 2 * f)
    ms.expert_quant_weight(ctx, w_down, dq, ds, f, d)
    xq, xs, h, hq, hs, y = new(E, T, d, dtype=i8), new(E, T, dtype=f32), new(E, T, f), new(E, T, f, dtype=i8), new(E, T, dtype=f32), new(E, T, d)
    ms.dispatch_q8(ctx, x, idx, slot, tok, xq, xs)
    ms.expert_glu_q8(ctx, xq, xs, uq, us, load, h, d, f)
    ms.expert_quant(ctx, h, load, hq, hs, f)
    ms.expert_gemm_q8(ctx, hq, hs, dq, ds, load, y, f, d)
    xe, h16, y16 = new(E, T, d), new(E, T, f), new(E, T, d)
    ms.dispatch(ctx, x, idx, slot, tok, xe)
    ms.expert_glu(ctx, xe, w_up, load, None, h16, d, f)
    ms.expert_gemm(ctx, h16, w_down, load, y16, f, d)
    # A value's rounding is uniform within half a step, amax / 254: an rms of amax / 440.  Rows and columns of 256 normal values have amax
    # of 3 to 4 rms, of 128 gated values up to 9: at most 1 %, 1 %, 2 % and 1 % of the rms of x, w_up, h and w_down; x and w_up reach h
    # twice (g and u, each with a slope below 1.1).  Independent: the root of the squares' sum is below 3.5 %.
    assert (y.float() - y16.float()).norm() <= 0.035 * y16.float().norm()


@pytest.mark.parametrize("C", [5, 300])
@pytest.mark.parametrize("load", [0, -2])
def test_no_rows_at_all(ms, C, load):
    """Every expert without a row: zeros out, nothing of the kept buffer touched."""
    E, K, f = 3, 64, 40
    ctx = context(ms, E, C)
    n = torch.full((E,), load, dtype=torch.int32, device=DEV)
    nan = lambda *s, dtype=BF16: torch.full(s, float("nan"), dtype=dtype, device=DEV)  # noqa: E731
    q = lambda *s: torch.full(s, 5, dtype=torch.int8, device=DEV)  # noqa: E731
    w = torch.ones(E, K, 2 * f, dtype=BF16, device=DEV)
    y, h, dpre, h2 = nan(E, C, f), nan(E, C, f), nan(E, C, 2 * f), nan(E, C, f)
    keep = torch.full((ms.keep8_bytes(ctx, f),), 77, dtype=torch.uint8, device=DEV)
    ms.expert_gemm_q8(ctx, q(E, C, K), nan(E, C, dtype=torch.float32), q(E, f, K), nan(E, f, dtype=torch.float32), n, y, K, f)
    assert (y == 0).all()
    ms.expert_glu_q8(ctx, q(E, C, K), nan(E, C, dtype=torch.float32), q(E, 2 * f, K), nan(E, 2 * f, dtype=torch.float32), n, h, K, f)
    assert (h == 0).all()
    h.fill_(float("nan"))
    ms.expert_glu_keep8(ctx, nan(E, C, K), w, n, keep, h, K, f)
    ms.expert_glu_bwd_keep8(ctx, nan(E, C, K), torch.ones(E, f, K, dtype=BF16, device=DEV), keep, n, dpre, h2, K, f)
    assert (h == 0).all() and (dpre == 0).all() and (h2 == 0).all() and (keep == 77).all()
    out, s = q(E, C, K), nan(E, C, dtype=torch.float32)
    ms.expert_quant(ctx, nan(E, C, K), n, out, s, K)
    assert (out == 0).all() and (s == 0).all() and ms.check_internal(ctx) == 0


def test_one_call_after_another_on_dirty_shared_memory(ms):
    """The same products again and again, between products of other sizes and forms: bit for bit the same."""
    E, C, K, f = 4, 300, 272, 104
    g = torch.Generator().manual_seed(8)
    ctx = context(ms, E, C)
    few = context(ms, E, 20)
    load, few_load = torch.tensor([300, 129, 0, 77], dtype=torch.int32, device=DEV), torch.tensor([20, 1, 0, 17], dtype=torch.int32, device=DEV)
    x, w, wd = (torch.randn(*s, generator=g).to(BF16).to(DEV) for s in ((E, C, K), (E, K, 2 * f), (E, f, K)))
    xq, wq = ints(g, E, C, K).to(DEV), ints(g, E, 2 * f, K).to(DEV)
    xs, ws = torch.rand(E, C, generator=g).to(DEV), (torch.rand(E, 2 * f, generator=g) * 1e-3).to(DEV)

    def once(c, n, ld):
        new = lambda *s: torch.full(s, float("nan"), dtype=BF16, device=DEV)  # noqa: E731
        rows = lambda t: t[:, :n].contiguous()  # noqa: E731
        keep = torch.zeros(ms.keep8_bytes(c, f), dtype=torch.uint8, device=DEV)
        h, dpre, h2, hq = new(E, n, f), new(E, n, 2 * f), new(E, n, f), new(E, n, f)
        ms.expert_glu_keep8(c, rows(x), w, ld, keep, h, K, f)
        ms.expert_glu_q8(c, rows(xq), rows(xs), wq, ws, ld, hq, K, f)
        ms.expert_glu_bwd_keep8(c, rows(x), wd, keep, ld, dpre, h2, K, f)
        return h, hq, dpre, h2, keep

    want, few_want = once(ctx, C, load), once(few, 20, few_load)
    for _ in range(20):
        for c, n, ld, ref in ((few, 20, few_load, few_want), (ctx, C, load, want)):
            assert all(torch.equal(a, b) for a, b in zip(once(c, n, ld), ref))
    assert ms.check_internal(ctx) == 0 and ms.check_internal(few) == 0
