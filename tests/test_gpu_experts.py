"""Expert products (grouped by expert, ragged loads) against a plain implementation in 64 bits.

Tolerances.  A product of bf16 numbers is exact in fp32 and so is the product of two fp32 numbers to half a step; the sum of
up to a few thousand of them in fp32 is off by a random walk of roundings, well below 1e-5 of the sum of their magnitudes
(sqrt(4096) * 2^-24 = 4e-6).  A bf16 output is rounded once: 2^-8 of the value.  The gated forms pass those errors on through
the derivative of silu (at most 1.1) and add an exponential and a quotient (below 1e-5 of the factors).
What lies behind an expert's load holds NaN on input, and has to be zero on output."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ACC = 1e-5
ROUND = {"bf16": 2.0 ** -8, "f32": 0.0}
INVALID, UNSUPPORTED = 1, 6


@pytest.fixture(scope="module")
def ms():
    from paper_2508_12801_b200 import binding
    assert torch.cuda.is_available()
    return binding


def make_ctx(ms, E, C, dtype, d=64):
    return ms.create(ms.make_params(C, d, E, 1, capacity=C, io_dtype=ms.BF16 if dtype == "bf16" else ms.F32), DEV)


def loads(E, C, kind, seed):
    g = torch.Generator().manual_seed(seed)
    l = torch.randint(0, C + 1, (E,), generator=g)
    if kind == "full":
        l[:] = C
    elif kind == "odd":        # every special value: none, one, full, beyond the capacity, negative
        for i, v in enumerate([0, 1, C, C + 7, -3][:E]):
            l[i] = v
    elif kind == "empty":
        l[:] = 0
    elif kind == "one":        # a single row in the last expert
        l[:] = 0
        l[-1] = 1
    return l.to(torch.int32)


class Data:
    """Host-made inputs: NaN behind the loads; float64 images with zero rows there."""

    def __init__(self, dtype, E, C, load, seed):
        self.dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.E, self.C = E, C
        self.rows = load.clamp(0, C).tolist()
        self.g = torch.Generator().manual_seed(seed)

    def buffer(self, width):
        x = torch.randn(self.E, self.C, width, generator=self.g).to(self.dt)
        ref = x.double()
        for e, n in enumerate(self.rows):
            x[e, n:] = float("nan")
            ref[e, n:] = 0
        return x.to(DEV), ref.to(DEV)

    def weight(self, d_in, d_out, layout):
        w = (torch.randn(self.E, d_in, d_out, generator=self.g) * d_in ** -0.5).to(self.dt)
        dev = (w if layout == 0 else w.transpose(1, 2).contiguous()).to(DEV)
        return dev, w.double().to(DEV)


def guarded(shape, dt):
    """An output full of NaN with a guard row behind it; the guard has to stay as it is."""
    n = int(np.prod(shape))
    flat = torch.full((n + 256,), float("nan"), dtype=dt, device=DEV)
    flat[n:] = 7.0
    return flat, flat[:n].view(shape)


def assert_guard(flat, shape):
    assert (flat[int(np.prod(shape)):] == 7.0).all(), "written behind the buffer"


def assert_within(got, ref, bar, rows, what):
    got = got.double()
    for e, n in enumerate(rows):
        assert (got[e, n:] == 0).all(), f"{what}: rows behind the load of expert {e} are not zero"
    d = (got - ref).abs()
    bad = ~(d <= bar)
    assert not bad.any(), f"{what}: {int(bad.sum())} entries off, worst {float((d / (bar + 1e-300)).nan_to_num(1e30).max()):.3g} x the bar"


SHAPES = [
    # E, C, d_in, d_out, kind
    (1, 1, 8, 8, "full"), (5, 1, 64, 64, "odd"), (5, 5, 72, 200, "odd"), (8, 16, 256, 512, "rand"), (3, 17, 136, 264, "rand"),
    (8, 64, 512, 256, "odd"), (6, 65, 200, 128, "odd"), (5, 100, 128, 72, "odd"), (4, 130, 264, 1000, "rand"), (7, 257, 320, 320, "odd"),
    (3, 300, 72, 136, "full"), (2, 520, 1024, 256, "rand"), (128, 9, 64, 128, "rand"), (64, 130, 64, 64, "rand"), (4, 33, 64, 64, "empty"),
    (33, 4, 128, 264, "one"), (5, 700, 136, 776, "odd"),
    (5, 128, 192, 392, "odd"), (4, 127, 1032, 128, "rand"), (3, 129, 192, 64, "full"), (2, 4300, 72, 264, "full"),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("E,C,d_in,d_out,kind", SHAPES)
def test_expert_gemm(ms, E, C, d_in, d_out, kind, layout, dtype):
    load = loads(E, C, kind, 1)
    d = Data(dtype, E, C, load, 2)
    x, X = d.buffer(d_in)
    w, W = d.weight(d_in, d_out, layout)
    ctx = make_ctx(ms, E, C, dtype)
    flat, y = guarded((E, C, d_out), d.dt)
    ms.expert_gemm(ctx, x, w, load.to(DEV), y, d_in, d_out, layout)
    ref, mag = X @ W, X.abs() @ W.abs()
    assert_within(y, ref, ROUND[dtype] * ref.abs() + ACC * mag, d.rows, "expert_gemm")
    assert_guard(flat, y.shape)
    assert ms.check_internal(ctx) == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("E,C,d_in,d_out,kind", SHAPES)
def test_expert_gemm_dw(ms, E, C, d_in, d_out, kind, layout, dtype):
    load = loads(E, C, kind, 3)
    d = Data(dtype, E, C, load, 4)
    x, X = d.buffer(d_in)
    dy, DY = d.buffer(d_out)
    ctx = make_ctx(ms, E, C, dtype)
    shape = (E, d_in, d_out) if layout == 0 else (E, d_out, d_in)
    flat, dw = guarded(shape, torch.float32)
    ms.expert_gemm_dw(ctx, x, dy, load.to(DEV), dw, d_in, d_out, layout)
    ref, mag = X.transpose(1, 2) @ DY, X.abs().transpose(1, 2) @ DY.abs()
    if layout:
        ref, mag = ref.transpose(1, 2), mag.transpose(1, 2)
    assert_within(dw, ref, ACC * mag, [shape[1]] * E, "expert_gemm_dw")
    assert_guard(flat, shape)
    # accumulate: once more on top; the sum of two equal numbers is exact, and the call repeats bit for bit (over more rows than
    # one sum takes, 4096, the parts are added one after the other and round on the way)
    first = dw.clone()
    ms.expert_gemm_dw(ctx, x, dy, load.to(DEV), dw, d_in, d_out, layout, accumulate=1)
    if C <= 4096:
        assert torch.equal(dw, 2 * first)
    assert_within(dw, 2 * ref, ACC * 2 * mag, [shape[1]] * E, "expert_gemm_dw, added")
    assert_guard(flat, shape)
    assert ms.check_internal(ctx) == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("keep", [True, False])
@pytest.mark.parametrize("E,C,d_in,d_ff,kind", SHAPES)
def test_expert_glu(ms, E, C, d_in, d_ff, kind, keep, layout, dtype):
    load = loads(E, C, kind, 5)
    d = Data(dtype, E, C, load, 6)
    x, X = d.buffer(d_in)
    w, W = d.weight(d_in, 2 * d_ff, layout)
    W = W.clone()
    ctx = make_ctx(ms, E, C, dtype)
    flat, h = guarded((E, C, d_ff), d.dt)
    pflat, pre = guarded((E, C, 2 * d_ff), d.dt)
    ms.expert_glu(ctx, x, w, load.to(DEV), pre if keep else None, h, d_in, d_ff, layout)
    P, mag = X @ W, X.abs() @ W.abs()
    g, u = P[..., :d_ff], P[..., d_ff:]
    silu = g * torch.sigmoid(g)
    ref = silu * u
    bar = (ROUND[dtype] + ACC) * ref.abs() + ACC * (1.1 * u.abs() * mag[..., :d_ff] + silu.abs() * mag[..., d_ff:])
    assert_within(h, ref, bar, d.rows, "expert_glu h")
    assert_guard(flat, h.shape)
    if keep:
        assert_within(pre, P, ROUND[dtype] * P.abs() + ACC * mag, d.rows, "expert_glu pre")
        assert_guard(pflat, pre.shape)
    assert ms.check_internal(ctx) == 0


def dact64(dh, g, u):
    s = torch.sigmoid(g)
    return torch.cat([dh * u * (s + g * s * (1 - s)), dh * g * s], dim=2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("E,C,d_out,d_ff,kind", SHAPES)
def test_expert_glu_bwd(ms, E, C, d_out, d_ff, kind, layout, dtype):
    load = loads(E, C, kind, 7)
    d = Data(dtype, E, C, load, 8)
    dy, DY = d.buffer(d_out)
    pre, PRE = d.buffer(2 * d_ff)
    w, W = d.weight(d_ff, d_out, layout)
    ctx = make_ctx(ms, E, C, dtype)
    flat, dpre = guarded((E, C, 2 * d_ff), d.dt)
    ms.expert_glu_bwd(ctx, dy, w, pre, load.to(DEV), dpre, d_out, d_ff, layout)
    dh, mag = DY @ W.transpose(1, 2), DY.abs() @ W.abs().transpose(1, 2)
    g, u = PRE[..., :d_ff], PRE[..., d_ff:]
    ref = dact64(dh, g, u)
    one = torch.ones_like(g)
    # 1 + g (1 - s) cancels near g = -1.28: its error scales with 1 + |g|, not with its value
    bar = ROUND[dtype] * ref.abs() + ACC * torch.cat([(mag + dh.abs()) * u.abs() * (one + g.abs()), (mag + dh.abs()) * g.abs()], dim=2)
    assert_within(dpre, ref, bar, d.rows, "expert_glu_bwd")
    assert_guard(flat, dpre.shape)
    assert ms.check_internal(ctx) == 0


def test_glu_bwd_is_the_derivative(ms):
    """Against central differences of the forward formula in 64 bits."""
    E, C, d_out, d_ff = 3, 6, 24, 16
    load = torch.tensor([6, 2, 4], dtype=torch.int32)
    d = Data("f32", E, C, load, 9)
    dy, DY = d.buffer(d_out)
    pre, PRE = d.buffer(2 * d_ff)
    w, W = d.weight(d_ff, d_out, 0)
    ctx = make_ctx(ms, E, C, "f32")
    dpre = torch.empty_like(pre)
    ms.expert_glu_bwd(ctx, dy, w, pre, load.to(DEV), dpre, d_out, d_ff, 0)

    def loss(p):
        h = p[..., :d_ff] * torch.sigmoid(p[..., :d_ff]) * p[..., d_ff:]
        return ((h @ W) * DY).sum()
    eps = 1e-5
    num = torch.zeros_like(PRE)
    for idx in np.ndindex(*PRE.shape):
        p = PRE.clone(); p[idx] += eps
        m = PRE.clone(); m[idx] -= eps
        num[idx] = (loss(p) - loss(m)) / (2 * eps)
    # the differences are good to about eps^2 = 1e-10, the fp32 kernel to 1e-5 of terms of order 1 to 10
    assert (dpre.double() - num).abs().max() < 2e-4
    assert (num.abs().max() > 0.5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_extreme_gate_values(ms, dtype):
    """Gates far out: silu(g) -> 0 or g without NaN; an infinite weight stays in its column, a NaN row in its row."""
    E, C, d_in, d_ff = 2, 4, 64, 64
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = torch.zeros(E, C, d_in, dtype=dt, device=DEV)
    x[:, :, 0] = 1.0
    x[1, 2, 5] = float("nan")
    w = torch.zeros(E, d_in, 2 * d_ff, dtype=dt, device=DEV)
    w[:, 0, :d_ff] = torch.tensor([-1e30, -500.0, -100.0, -20.0, 0.0, 20.0, 100.0, 1e4] * 8, dtype=dt, device=DEV)
    w[:, 0, d_ff:] = 2.0
    w[0, 0, d_ff + 9] = float("inf")
    load = torch.full((E,), C, dtype=torch.int32, device=DEV)
    ctx = make_ctx(ms, E, C, dtype)
    h = torch.empty(E, C, d_ff, dtype=dt, device=DEV)
    ms.expert_glu(ctx, x, w, load, None, h, d_in, d_ff, 0)
    g = w[0, 0, :d_ff].double()
    ref = g * torch.sigmoid(g) * 2.0
    got = h[0].double()
    ok = torch.arange(d_ff, device=DEV) != 9
    assert ((got[:, ok] - ref[ok]).abs() <= (ROUND[dtype] + ACC) * ref[ok].abs() + 1e-30).all()
    assert torch.isinf(got[:, 9]).all() or torch.isnan(got[:, 9]).all()
    assert torch.isnan(h[1, 2]).all() and not torch.isnan(h[1, [0, 1, 3]]).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_repeats_bit_for_bit_and_on_another_stream(ms, dtype):
    E, C, d_in, d_out = 9, 70, 256, 264
    load = loads(E, C, "odd", 11)
    d = Data(dtype, E, C, load, 12)
    x, _ = d.buffer(d_in)
    dy, _ = d.buffer(d_out)
    w, _ = d.weight(d_in, d_out, 0)
    l = load.to(DEV)
    ctx = make_ctx(ms, E, C, dtype)
    y = [torch.empty(E, C, d_out, dtype=d.dt, device=DEV) for _ in range(2)]
    dw = [torch.empty(E, d_in, d_out, device=DEV) for _ in range(2)]
    s = torch.cuda.Stream()
    for i in range(2):
        torch.cuda.synchronize()
        with torch.cuda.stream(s if i else torch.cuda.current_stream()):
            ms.expert_gemm(ctx, x, w, l, y[i], d_in, d_out, 0)
            ms.expert_gemm_dw(ctx, x, dy, l, dw[i], d_in, d_out, 0)
    torch.cuda.synchronize()
    assert torch.equal(y[0], y[1]) and torch.equal(dw[0], dw[1])


@pytest.mark.parametrize("dtype,C", [("f32", 40), ("bf16", 40), ("bf16", 300)])
def test_captured_and_replayed_with_other_loads(ms, dtype, C):
    """The loads are read on the device: one captured graph serves every load."""
    E, d_in, d_ff, d_out = 6, 128, 72, 64
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    ctx = make_ctx(ms, E, C, dtype)
    g = torch.Generator().manual_seed(3)
    x = torch.randn(E, C, d_in, generator=g).to(dt).to(DEV)
    wu = (torch.randn(E, d_in, 2 * d_ff, generator=g) * 0.1).to(dt).to(DEV)
    wd = (torch.randn(E, d_ff, d_out, generator=g) * 0.1).to(dt).to(DEV)
    load = loads(E, C, "full", 0).to(DEV)
    h = torch.empty(E, C, d_ff, dtype=dt, device=DEV)
    y = torch.empty(E, C, d_out, dtype=dt, device=DEV)

    def step():
        ms.expert_glu(ctx, x, wu, load, None, h, d_in, d_ff, 0)
        ms.expert_gemm(ctx, h, wd, load, y, d_ff, d_out, 0)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for kind in ["odd", "rand", "empty", "full"]:
        load.copy_(loads(E, C, kind, 5))
        y.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        y.fill_(float("nan"))
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, y) and not torch.isnan(y).any()


def test_refusals(ms):
    E, C, d_in, d_out = 4, 8, 64, 32
    ctx = make_ctx(ms, E, C, "bf16")
    bf = dict(dtype=torch.bfloat16, device=DEV)
    x, w, y = torch.zeros(E, C, d_in, **bf), torch.zeros(E, d_in, d_out, **bf), torch.full((E, C, d_out), 3.0, **bf)
    load = torch.zeros(E, dtype=torch.int32, device=DEV)
    for bad in [dict(x=x.float()), dict(x=x[:, :4]), dict(x=x.cpu()), dict(w=w.transpose(1, 2)), dict(w=w[:3]), dict(load=load.long()),
                dict(load=load[:2]), dict(y=y.float()), dict(x=None), dict(y=None)]:
        a = dict(x=x, w=w, load=load, y=y)
        a.update(bad)
        with pytest.raises(ValueError):
            ms.expert_gemm(ctx, a["x"], a["w"], a["load"], a["y"], d_in, d_out, 0)
    lib, st = ms._lib, 0
    p = lambda t: t.data_ptr()  # noqa: E731
    gemm = lib.maxscore_expert_gemm
    assert gemm(ctx.handle, p(x), p(w), p(load), p(y), d_in, d_out, 2, st) == INVALID
    assert gemm(ctx.handle, p(x), p(w), p(load), p(y), 0, d_out, 0, st) == INVALID
    assert gemm(ctx.handle, p(x), p(w), p(load), p(y), d_in, -8, 0, st) == INVALID
    assert gemm(ctx.handle, p(x), p(w), p(load), p(y), d_in, 28, 0, st) == UNSUPPORTED
    assert gemm(ctx.handle, p(x), p(w), p(load), p(x), d_in, d_out, 0, st) == INVALID
    assert gemm(ctx.handle, p(x) + 2, p(w), p(load), p(y), d_in, d_out, 0, st) == INVALID
    assert gemm(ctx.handle, p(x), p(w), None, p(y), d_in, d_out, 0, st) == INVALID
    assert lib.maxscore_expert_gemm_dw(ctx.handle, p(x), p(y), p(load), None, d_in, d_out, 0, 0, st) == INVALID
    assert lib.maxscore_expert_glu(ctx.handle, p(x), p(w), p(load), p(x), p(y), d_in, d_out // 2, 0, st) == INVALID
    assert lib.maxscore_expert_glu_bwd(ctx.handle, p(x), p(w), None, p(load), p(y), d_in, d_out, 0, st) == INVALID
    torch.cuda.synchronize()
    assert (y == 3.0).all()                     # nothing ran


def test_offsets_beyond_32_bits(ms):
    """An output of more than 2^31 elements: rows at both ends are right and the padding between is zero."""
    E, C, d_in, d_out = 2, 66000, 64, 16384
    dt = torch.bfloat16
    ctx = make_ctx(ms, E, C, "bf16")
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.empty(E, C, d_in, dtype=dt, device=DEV).normal_(generator=g)
    w = torch.empty(E, d_in, d_out, dtype=dt, device=DEV).normal_(generator=g)
    load = torch.tensor([C - 300, C], dtype=torch.int32, device=DEV)
    y = torch.full((E, C, d_out), float("nan"), dtype=dt, device=DEV)
    ms.expert_gemm(ctx, x, w, load, y, d_in, d_out, 0)
    for e, rows in ((0, [0, 1, C - 301]), (1, [0, C // 2, C - 257, C - 1])):
        X, W = x[e, rows].double(), w[e].double()
        ref, mag = X @ W, X.abs() @ W.abs()
        assert ((y[e, rows].double() - ref).abs() <= ROUND["bf16"] * ref.abs() + ACC * mag).all()
    assert (y[0, C - 300:] == 0).all() and not torch.isnan(y[1, ::997]).any()
    dw = torch.empty(E, d_in, d_out, device=DEV)
    ms.expert_gemm_dw(ctx, x, y, load, dw, d_in, d_out, 0)
    ref = torch.einsum("si,sj->ij", x[1].double(), y[1, :, :64].double())
    mag = torch.einsum("si,sj->ij", x[1].double().abs(), y[1, :, :64].double().abs())
    assert ((dw[1, :, :64].double() - ref).abs() <= 1e-5 * mag).all()
    assert ms.check_internal(ctx) == 0


@pytest.mark.parametrize("C", [40, 300])
def test_two_contexts_on_two_streams(ms, C):
    """Calls of two contexts that may overlap on the GPU give what they give one after the other."""
    E, d_in, d_out = 12, 512, 520
    sets = []
    for i in range(2):
        load = loads(E, C, "rand", 20 + i)
        d = Data("bf16", E, C, load, 30 + i)
        x, _ = d.buffer(d_in)
        dy, _ = d.buffer(d_out)
        w, _ = d.weight(d_in, d_out, i)
        sets.append((make_ctx(ms, E, C, "bf16"), x, dy, w, load.to(DEV), i))

    def go(s, stream=None):
        ctx, x, dy, w, load, layout = s
        y = torch.empty(E, C, d_out, dtype=torch.bfloat16, device=DEV)
        dw = torch.empty(w.shape, device=DEV)
        torch.cuda.synchronize()
        return y, dw, lambda: (ms.expert_gemm(ctx, x, w, load, y, d_in, d_out, layout, stream=stream),
                               ms.expert_gemm_dw(ctx, x, dy, load, dw, d_in, d_out, layout, stream=stream))
    alone = []
    for s in sets:
        y, dw, call = go(s)
        call()
        torch.cuda.synchronize()
        alone.append((y, dw))
    both = [go(s, torch.cuda.Stream()) for s in sets]
    for _ in range(5):
        for _, _, call in both:
            call()
    torch.cuda.synchronize()
    for (y, dw), (y2, dw2, _) in zip(alone, both):
        assert torch.equal(y, y2) and torch.equal(dw, dw2)


def test_launches_are_counted(ms):
    ctx = make_ctx(ms, 4, 8, "bf16")
    bf = dict(dtype=torch.bfloat16, device=DEV)
    x, w, y = torch.zeros(4, 8, 64, **bf), torch.zeros(4, 64, 32, **bf), torch.zeros(4, 8, 32, **bf)
    n = ms.launch_count(ctx)
    ms.expert_gemm(ctx, x, w, torch.ones(4, dtype=torch.int32, device=DEV), y, 64, 32, 0)
    assert ms.launch_count(ctx) == n + 1
