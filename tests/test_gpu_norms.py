"""Norms before and after a block (after-norm, gate, scaled residual, before-norm, optionally behind combine) against a plain
implementation in 64 bits.

A row passes through the forward steps without rounding, so the reference does too and every output is rounded once; the
backward takes the stored rows, and so does its reference.  Tolerances: one rounding of the output (2^-8 of the value in bf16; nothing in fp32) plus fp32 arithmetic:
sums over a row of at most 16384 terms and a handful of products, below 1e-5 of the magnitudes that enter; sums over tokens
below 1e-5 of the sum of their magnitudes."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ACC = 1e-5
ROUND = {"bf16": 2.0 ** -8, "f32": 0.0}
EPS = 1e-5
INVALID, UNSUPPORTED = 1, 6


@pytest.fixture(scope="module")
def ms():
    from paper_2508_12801_b200 import binding
    assert torch.cuda.is_available()
    return binding


def make_ctx(ms, T, d, E, k, C, dtype):
    return ms.create(ms.make_params(T, d, E, k, capacity=C, io_dtype=ms.BF16 if dtype == "bf16" else ms.F32), DEV)


def assignment(T, E, k, C, seed, drop=0.1):
    """Ascending experts, slots in token order, some pairs empty (-1) and some beyond the capacity."""
    g = torch.Generator().manual_seed(seed)
    idx = torch.rand(T, E, generator=g).topk(k, dim=1).indices.sort(dim=1).values
    slot = torch.zeros_like(idx)
    used = [0] * E
    for i in range(T):
        for c in range(k):
            e = int(idx[i, c])
            slot[i, c] = used[e]
            used[e] += 1
    idx[torch.rand(T, k, generator=g) < drop] = -1
    return idx.to(torch.int32), slot.to(torch.int32)


class Case:
    def __init__(self, ms, T, d, dtype, gates=0, post=True, pre=True, w_offset=0.0, res_scale=1.0, E=6, k=2, seed=0):
        self.T, self.d, self.dtype, self.k, self.E = T, d, dtype, k, E
        self.C = max(1, -(-T * k // E) + 1)
        if E * min(self.C, T) < T * k:
            self.C = T
        self.dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.ctx = make_ctx(ms, T, d, E, k, self.C, dtype)
        self.g = torch.Generator().manual_seed(seed)
        self.rpg = -(-T // gates) if gates else 0
        self.n_gates = -(-T // self.rpg) if gates else 0
        self.w_post = self.rand(d, scale=0.2, shift=1 - w_offset) if post else None
        self.w_pre = self.rand(d, scale=0.2, shift=1 - w_offset) if pre else None
        self.gate = self.rand(self.n_gates, d) if gates else None
        self.off, self.scale = w_offset, res_scale
        self.norm = ms.make_norm(self.w_post, self.gate, self.w_pre, self.rpg, EPS, w_offset, res_scale)

    def rand(self, *shape, scale=1.0, shift=0.0):
        return (torch.randn(*shape, generator=self.g) * scale + shift).to(self.dt).to(DEV)

    def empty(self, *shape):
        n = int(np.prod(shape))
        flat = torch.full((n + 64,), float("nan"), dtype=self.dt, device=DEV)
        flat[n:] = 7.0
        out = flat[:n].view(*shape)
        out.guard = flat[n:]
        return out

    def gate64(self):
        if self.gate is None:
            return torch.ones(1, self.d, dtype=torch.float64, device=DEV)
        return self.gate.double()[torch.arange(self.T, device=DEV) // self.rpg]

    def rms(self, v):
        return (v.square().mean(dim=1, keepdim=True) + EPS).sqrt()

    def close(self, got, ref, mag, what):
        bar = ROUND[self.dtype] * ref.abs() + ACC * mag
        d = (got.double() - ref).abs()
        bad = ~(d <= bar)
        assert not bad.any(), f"{what}: {int(bad.sum())} off, worst {float((d / (bar + 1e-300)).nan_to_num(1e30).max()):.3g} x the bar"
        if hasattr(got, "guard"):
            assert (got.guard == 7.0).all(), what + ": written behind the buffer"

    def check_forward(self, y, res, r_out, h, y_mag=None):
        """y: the block's output in 64 bits or as given; y_mag: magnitudes that entered it, where it was summed in fp32."""
        r = self.scale * res.double()
        mag = r.abs()
        if y is not None:
            Y = y.double()
            n, m = Y, Y.abs() if y_mag is None else y_mag
            if self.w_post is not None:
                w = (self.off + self.w_post.double()) / self.rms(Y)
                n, m = Y * w, m * w.abs()
            n, m = n * self.gate64(), m * self.gate64().abs()
            r, mag = r + n, mag + m
        if r_out is not None:
            self.close(r_out, r, mag, "r_out")
        if self.w_pre is not None:
            w = (self.off + self.w_pre.double()) / self.rms(r)
            self.close(h, r * w, mag * w.abs(), "h")


SHAPES = [(1, 8), (1, 2048), (3, 64), (7, 136), (64, 512), (65, 520), (129, 1000), (33, 1032), (200, 2048), (50, 4096), (9, 4104), (5, 8192)]
OPTIONS = [dict(), dict(gates=1), dict(gates=3, res_scale=0.5), dict(post=False, gates=1), dict(post=False, pre=False),
           dict(pre=False, gates=2), dict(w_offset=1.0, res_scale=-2.0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("opt", OPTIONS, ids=str)
@pytest.mark.parametrize("T,d", SHAPES)
def test_block_norm(ms, T, d, opt, dtype):
    opt = dict(opt)
    if "gates" in opt:
        opt["gates"] = min(opt["gates"], T)
    c = Case(ms, T, d, dtype, seed=1, **opt)
    y, res = c.rand(T, d), c.rand(T, d)
    r_out, h = c.empty(T, d), c.empty(T, d) if c.w_pre is not None else None
    ms.block_norm(c.ctx, y, res, c.norm, r_out, h)
    c.check_forward(y, res, r_out, h)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,d,E,k,gates,post", [(1, 256, 4, 2, 0, True), (1, 2048, 64, 8, 1, True), (16, 2048, 64, 8, 0, True),
                                                (77, 520, 5, 5, 3, True), (300, 1032, 8, 2, 1, False), (130, 4096, 12, 8, 1, True),
                                                (64, 64, 3, 1, 0, False)])
def test_combine_norm(ms, T, d, E, k, gates, post, dtype):
    c = Case(ms, T, d, dtype, gates=gates, post=post, E=E, k=k, seed=2, res_scale=0.75)
    idx, slot = assignment(T, E, k, c.C, 3)
    idx, slot = idx.to(DEV), slot.to(DEV)
    gw = torch.rand(T, k, generator=c.g).to(DEV)
    src, res = c.rand(E, c.C, d), c.rand(T, d)
    y, r_out, h = c.empty(T, d), c.empty(T, d), c.empty(T, d)
    for w in (gw, None):
        want = torch.empty(T, d, dtype=c.dt, device=DEV)
        ms.combine(c.ctx, src, idx, slot, w, want)
        ms.combine_norm(c.ctx, src, idx, slot, w, res, c.norm, y, r_out, h)
        assert torch.equal(y, want)                      # what combine alone writes, bit for bit
        ok = ((idx >= 0) & (slot < c.C)).double()
        rows = src.double()[idx.long().clamp(min=0), slot.long().clamp(max=c.C - 1)]
        wt = (ok if w is None else ok * w.double())[:, :, None]
        c.check_forward((rows * wt).sum(1), res, r_out, h, y_mag=(rows * wt).abs().sum(1))
        r2, h2 = c.empty(T, d), c.empty(T, d)
        ms.combine_norm(c.ctx, src, idx, slot, w, res, c.norm, None, r2, h2)      # y not wanted
        assert torch.equal(r2, r_out) and torch.equal(h2, h)
        if dtype == "f32":                                                        # no rounding of y between the two calls
            r3, h3 = c.empty(T, d), c.empty(T, d)
            ms.block_norm(c.ctx, y, res, c.norm, r3, h3)
            assert torch.equal(r3, r_out) and torch.equal(h3, h)


def test_combine_norm_reads_no_empty_pair(ms):
    """A token without any expert gets y = 0; NaN in rows that no pair names reaches nothing."""
    c = Case(ms, 10, 128, "bf16", gates=1, seed=4)
    idx = torch.full((10, 2), -1, dtype=torch.int32)
    slot = torch.zeros(10, 2, dtype=torch.int32)
    idx[3] = torch.tensor([0, 5]); slot[3] = torch.tensor([1, c.C])          # the second one is beyond the capacity
    idx[4, 0] = 6                                                            # no such expert
    src = torch.full((c.E, c.C, 128), float("nan"), dtype=c.dt, device=DEV)
    src[0, 1] = 2.0
    res = c.rand(10, 128)
    y, r_out, h = c.empty(10, 128), c.empty(10, 128), c.empty(10, 128)
    ms.combine_norm(c.ctx, src, idx.to(DEV), slot.to(DEV), None, res, c.norm, y, r_out, h)
    assert (y[3] == 2.0).all() and (y[[0, 1, 2, 4, 5, 6, 7, 8, 9]] == 0).all()
    c.check_forward(y, res, r_out, h)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_alone_and_in_place(ms, dtype):
    c = Case(ms, 37, 520, dtype, post=False, seed=5)
    res = c.rand(37, 520)
    h = c.empty(37, 520)
    ms.block_norm(c.ctx, None, res, c.norm, None, h)          # the norm in front of a first block
    c.check_forward(None, res, None, h)
    c = Case(ms, 37, 520, dtype, gates=2, seed=6)
    y, res = c.rand(37, 520), c.rand(37, 520)
    r_out, h, h2 = c.empty(37, 520), c.empty(37, 520), c.empty(37, 520)
    ms.block_norm(c.ctx, y, res, c.norm, r_out, h)
    ms.block_norm(c.ctx, y, res, c.norm, res, h2)             # r_out in the residual's own buffer
    assert torch.equal(res, r_out) and torch.equal(h, h2)


def test_a_row_of_zeros_and_a_row_of_nan(ms):
    c = Case(ms, 4, 256, "bf16", gates=1, seed=7)
    y, res = c.rand(4, 256), c.rand(4, 256)
    y[1], res[1] = 0, 0
    y[2, 5] = float("nan")
    r_out, h = c.empty(4, 256), c.empty(4, 256)
    ms.block_norm(c.ctx, y, res, c.norm, r_out, h)
    assert (r_out[1] == 0).all() and (h[1] == 0).all()
    assert torch.isnan(r_out[2]).all() and torch.isfinite(h[[0, 1, 3]]).all()


def backward64(c, dro, dh, y, r_out):
    """Gradients in 64 bits by the formula, and the magnitudes that their roundings scale with."""
    D, gate = c.d, c.gate64()
    out, mag = {}, {}
    dr = dro.double() if dro is not None else torch.zeros(c.T, D, dtype=torch.float64, device=DEV)
    m = dr.abs()
    if c.w_pre is not None:
        R, H, w = r_out.double(), dh.double(), c.off + c.w_pre.double()
        rms = c.rms(R)
        v, u = H * w / rms, R / rms
        out["dw_pre"], mag["dw_pre"] = (H * u).sum(0), (H * u).abs().sum(0)
        dr = dr + v - u * (v * u).mean(1, keepdim=True)
        m = m + v.abs() + u.abs() * (v * u).abs().mean(1, keepdim=True)
    out["dr"], mag["dr"] = c.scale * dr, abs(c.scale) * m
    if y is None:
        return out, mag
    Y = y.double()
    dn, mn = gate * dr, gate.abs() * m
    n = Y
    if c.w_post is not None:
        rms, w = c.rms(Y), c.off + c.w_post.double()
        u = Y / rms
        n = u * w
        out["dw_post"], mag["dw_post"] = (dn * u).sum(0), (mn * u.abs()).sum(0)
        v = dn * w / rms
        out["dy"] = v - u * (v * u).mean(1, keepdim=True)
        mv = mn * w.abs() / rms
        mag["dy"] = mv + u.abs() * (mv * u.abs()).mean(1, keepdim=True)
    else:
        out["dy"], mag["dy"] = dn, mn
    if c.gate is not None:
        at = torch.arange(c.T, device=DEV) // c.rpg
        z = lambda: torch.zeros(c.n_gates, D, dtype=torch.float64, device=DEV)  # noqa: E731
        out["dgate"], mag["dgate"] = z().index_add_(0, at, dr * n), z().index_add_(0, at, m * n.abs())
    return out, mag


def run_backward(ms, c, dro, dh, y, r_out):
    f = lambda *s: torch.full(s, float("nan"), device=DEV)  # noqa: E731
    got = dict(dy=c.empty(c.T, c.d) if y is not None else None, dr=c.empty(c.T, c.d), dw_post=f(c.d) if c.w_post is not None else None,
               dgate=f(c.n_gates, c.d) if c.gate is not None else None, dw_pre=f(c.d) if c.w_pre is not None else None)
    ms.block_norm_bwd(c.ctx, dro, dh, y, r_out, c.norm, got["dy"], got["dr"], got["dw_post"], got["dgate"], got["dw_pre"])
    return got


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("opt", OPTIONS + [dict(gates=64), dict(gates=10 ** 6)], ids=str)
@pytest.mark.parametrize("T,d", SHAPES + [(1500, 256), (700, 16)])
def test_block_norm_bwd(ms, T, d, opt, dtype):
    opt = dict(opt)
    if "gates" in opt:
        opt["gates"] = min(opt["gates"], T)
    c = Case(ms, T, d, dtype, seed=8, **opt)
    y, r_out, dro = c.rand(T, d), c.rand(T, d), c.rand(T, d)
    dh = c.rand(T, d) if c.w_pre is not None else None
    got = run_backward(ms, c, dro, dh, y, r_out)
    ref, mag = backward64(c, dro, dh, y, r_out)
    for name, g in got.items():
        assert (g is None) == (name not in ref)
        if g is not None and name in ("dy", "dr"):
            c.close(g, ref[name], mag[name], name)
        elif g is not None:
            assert ((g.double() - ref[name]).abs() <= ACC * mag[name]).all(), name
    again = run_backward(ms, c, dro, dh, y, r_out)
    for name, g in got.items():
        assert g is None or torch.equal(g, again[name]), name + " does not repeat"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_bwd_without_block_without_upstream_and_in_place(ms, dtype):
    T, d = 45, 264
    c = Case(ms, T, d, dtype, post=False, seed=9, res_scale=0.5)
    r_out, dh, dro = c.rand(T, d), c.rand(T, d), c.rand(T, d)
    for up in (dro, None):
        got = run_backward(ms, c, up, dh, None, r_out)
        ref, mag = backward64(c, up, dh, None, r_out)
        c.close(got["dr"], ref["dr"], mag["dr"], "dr")
        assert ((got["dw_pre"].double() - ref["dw_pre"]).abs() <= ACC * mag["dw_pre"]).all()
    first = run_backward(ms, c, dro, dh, None, r_out)["dr"]
    dw = torch.empty(d, device=DEV)
    ms.block_norm_bwd(c.ctx, dro, dh, None, r_out, c.norm, None, dro, None, None, dw)      # dr in dr_out's buffer
    assert torch.equal(dro, first)


def test_backward_is_the_derivative(ms):
    """Against central differences of the forward formula in 64 bits."""
    T, d = 5, 24
    c = Case(ms, T, d, "f32", gates=2, seed=10, res_scale=0.7)
    y, res, dro, dh = c.rand(T, d), c.rand(T, d), c.rand(T, d), c.rand(T, d)
    r_out, h = c.empty(T, d), c.empty(T, d)
    ms.block_norm(c.ctx, y, res, c.norm, r_out, h)
    got = run_backward(ms, c, dro, dh, y, r_out)

    def loss(y, res, wp, gate, wr):
        n = y / c.rms(y) * wp
        r = c.scale * res + gate[torch.arange(T, device=DEV) // c.rpg] * n
        return (r * dro.double()).sum() + (r / c.rms(r) * wr * dh.double()).sum()
    args = [t.double() for t in (y, res, c.w_post, c.gate, c.w_pre)]
    for pos, name in enumerate(["dy", "dr", "dw_post", "dgate", "dw_pre"]):
        num = torch.zeros_like(args[pos])
        for idx in np.ndindex(*num.shape):
            v = []
            for sign in (1, -1):
                a = [t.clone() for t in args]
                a[pos][idx] += sign * 1e-5
                v.append(loss(*a))
            num[idx] = (v[0] - v[1]) / 2e-5
        # differences: about 1e-9; the kernel worked from the fp32-rounded r_out: 1e-6 of terms of order 10
        assert (got[name].double() - num).abs().max() < 1e-4, name


def test_refusals(ms):
    c = Case(ms, 8, 64, "bf16", gates=2, seed=11)
    y, res, r, h = (c.rand(8, 64) for _ in range(4))
    keep = r.clone()
    for bad in [dict(y=y.float()), dict(res=res[:4]), dict(h=h.t()), dict(r=r.cpu())]:
        a = dict(y=y, res=res, r=r, h=h)
        a.update(bad)
        with pytest.raises(ValueError):
            ms.block_norm(c.ctx, a["y"], a["res"], c.norm, a["r"], a["h"])
    with pytest.raises(ValueError):
        ms.block_norm(c.ctx, y, res, ms.make_norm(w_post=c.w_post.float(), w_pre=c.w_pre), r, h)
    with pytest.raises(ValueError):
        ms.block_norm(c.ctx, y, res, ms.make_norm(gate=c.gate, w_pre=c.w_pre, rows_per_gate=1), r, h)

    def status(fn, *a):
        with pytest.raises(ms.MaxScoreError) as e:
            fn(c.ctx, *a)
        return e.value.status
    n = ms.make_norm
    assert status(ms.block_norm, y, res, n(w_pre=c.w_pre, eps=0.0), r, h) == INVALID
    assert status(ms.block_norm, y, res, n(w_pre=c.w_pre, eps=float("nan")), r, h) == INVALID
    assert status(ms.block_norm, y, res, n(w_pre=c.w_pre, res_scale=float("inf")), r, h) == INVALID
    assert status(ms.block_norm, y, res, n(gate=c.gate, w_pre=c.w_pre), r, h) == INVALID        # rows_per_gate missing
    assert status(ms.block_norm, y, res, n(w_pre=c.w_pre), r, None) == INVALID
    assert status(ms.block_norm, y, res, n(), r, h) == INVALID
    assert status(ms.block_norm, None, res, n(w_post=c.w_post, w_pre=c.w_pre), r, h) == INVALID
    assert status(ms.block_norm, y, res, n(w_pre=c.w_pre), y, h) == INVALID
    assert status(ms.block_norm, y, res, n(w_pre=c.w_pre), r, r) == INVALID
    assert status(ms.block_norm, y, res, n(), None, None) == INVALID
    src = torch.zeros(c.E, c.C, 64, dtype=torch.bfloat16, device=DEV)
    idx, slot = torch.zeros(8, 2, dtype=torch.int32, device=DEV), torch.zeros(8, 2, dtype=torch.int32, device=DEV)
    if src.numel() == 8 * 64:
        assert status(ms.combine_norm, src, idx, slot, None, res, n(w_pre=c.w_pre), None, r, src) == INVALID
    assert status(ms.combine_norm, src, idx, slot, None, res, n(w_pre=c.w_pre), r, r, h) == INVALID
    assert status(ms.combine_norm, src, idx, slot, None, res, n(w_pre=c.w_pre), res, r, h) == INVALID
    assert status(ms.combine_norm, src, idx, slot, None, res, n(w_pre=c.w_pre), None, r, None) == INVALID
    f = torch.empty(64, device=DEV)
    assert status(ms.block_norm_bwd, res, h, y, r, n(w_pre=c.w_pre), None, torch.empty_like(r), None, None, f) == INVALID
    assert status(ms.block_norm_bwd, res, h, y, r, n(w_pre=c.w_pre), torch.empty_like(r), y, None, None, f) == INVALID
    assert status(ms.block_norm_bwd, res, h, y, r, n(w_pre=c.w_pre), torch.empty_like(r), torch.empty_like(r), None, None, None) == INVALID
    torch.cuda.synchronize()
    assert torch.equal(r, keep)
    wide = make_ctx(ms, 2, 16392, 2, 1, 2, "bf16")
    t = torch.zeros(2, 16392, dtype=torch.bfloat16, device=DEV)
    w = torch.zeros(16392, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(ms.MaxScoreError) as e:
        ms.block_norm(wide, None, t, n(w_pre=w), None, torch.empty_like(t))
    assert e.value.status == UNSUPPORTED


def test_offsets_beyond_32_bits(ms):
    """Rows behind 2^31 elements."""
    T, d = 140000, 16384
    c = Case(ms, T, d, "bf16", post=False, seed=12, E=2, k=1)
    g = torch.Generator(device=DEV).manual_seed(1)
    res = torch.empty(T, d, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    h = torch.empty_like(res)
    ms.block_norm(c.ctx, None, res, c.norm, None, h)
    for rows in ([0, 1, 2], [T - 3, T - 1], [131071, 131072, 131073]):
        R = res[rows].double()
        ref = R / c.rms(R) * c.w_pre.double()
        c.close(h[rows], ref, ref.abs(), "h")
    dh, dr, dw = res, torch.empty_like(res), torch.empty(d, device=DEV)
    ms.block_norm_bwd(c.ctx, None, dh, None, h, c.norm, None, dr, None, None, dw)
    R, H, w = h[T - 2:].double(), dh[T - 2:].double(), c.w_pre.double()
    rms = c.rms(R)
    v, u = H * w / rms, R / rms
    c.close(dr[T - 2:], v - u * (v * u).mean(1, keepdim=True), v.abs() + u.abs() * (v * u).abs().mean(1, keepdim=True), "dr")


def test_gate_rows_wider_than_the_batch_and_streams(ms):
    c = Case(ms, 20, 264, "bf16", gates=1, seed=13)
    y, res = c.rand(20, 264), c.rand(20, 264)
    r1, h1, r2, h2 = (c.empty(20, 264) for _ in range(4))
    ms.block_norm(c.ctx, y, res, c.norm, r1, h1)
    wide = ms.make_norm(c.w_post, c.gate, c.w_pre, 10 ** 9, EPS, 0.0, 1.0)        # one gate row for many more tokens than there are
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    ms.block_norm(c.ctx, y, res, wide, r2, h2, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(r1, r2) and torch.equal(h1, h2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_captured_backward_replays(ms, dtype):
    c = Case(ms, 300, 520, dtype, gates=3, seed=14)
    y, r_out, dro, dh = (c.rand(300, 520) for _ in range(4))
    want = run_backward(ms, c, dro, dh, y, r_out)
    got = {k: torch.empty_like(v) for k, v in want.items()}
    call = lambda: ms.block_norm_bwd(c.ctx, dro, dh, y, r_out, c.norm, *(got[k] for k in ("dy", "dr", "dw_post", "dgate", "dw_pre")))  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for t in got.values():
        t.fill_(float("nan"))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(got[k], want[k]) for k in want)
