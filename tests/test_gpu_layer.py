"""A whole MoE layer (route, dispatch, experts, combine with the norms around it; forward and backward) against the same layer
in 64 bits, with the assignment that the library chose held constant.

fp32 is held tightly: every step is good to 1e-5 of what enters it and a handful of steps follow one another, so gradients are
held to 1e-4 of the largest entry of their tensor.  bf16 rounds every stored tensor (2^-8 each, about ten of them in a row, partly
cancelling): 2^-8 * 10 = 4e-2 of the root mean square over a tensor is the bar for the root mean square of the error."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-5


@pytest.fixture(scope="module")
def ms():
    from paper_2508_12801_b200 import binding
    assert torch.cuda.is_available()
    return binding


class Setup:
    def __init__(self, ms, T, d, E, k, f, cf, dtype, w_layout, gates, seed=0):
        from paper_2508_12801_b200.layer import MoELayer
        self.ms, self.T, self.d, self.E, self.k, self.f = ms, T, d, E, k, f
        self.dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        g = torch.Generator().manual_seed(seed)
        r = lambda *s, scale=1.0, shift=0.0: (torch.randn(*s, generator=g) * scale + shift).to(self.dt).to(DEV)  # noqa: E731
        p = ms.make_params(T, d, E, k, cf, io_dtype=ms.BF16 if dtype == "bf16" else ms.F32)
        self.layer = MoELayer(p, f, w_layout)
        self.L = w_layout
        self.h, self.res, self.wg = r(T, d), r(T, d), r(d, E, scale=d ** -0.5)
        self.wu = r(*((E, d, 2 * f) if w_layout == 0 else (E, 2 * f, d)), scale=d ** -0.5)
        self.wd = r(*((E, f, d) if w_layout == 0 else (E, d, f)), scale=f ** -0.5)
        self.w_post, self.w_pre = r(d, scale=0.1, shift=1.0), r(d, scale=0.1, shift=1.0)
        self.rpg = -(-T // gates)
        self.gate = r(gates, d, scale=0.5)
        self.norm = ms.make_norm(self.w_post, self.gate, self.w_pre, self.rpg, EPS, 0.0, 0.8)
        self.dro, self.dho = r(T, d), r(T, d)
        e = lambda *s, dtype=torch.float32: torch.full(s, float("nan"), dtype=dtype, device=DEV)  # noqa: E731
        self.r_out, self.h_out = e(T, d, dtype=self.dt), e(T, d, dtype=self.dt)
        self.out = dict(dh=e(T, d, dtype=self.dt), dr=e(T, d, dtype=self.dt), dw_gate=e(d, E), dw_up=e(*self.wu.shape), dw_down=e(*self.wd.shape),
                        dw_post=e(d), dgate=e(gates, d), dw_pre=e(d))

    def forward(self):
        self.layer.forward(self.h, self.res, self.wg, self.wu, self.wd, self.norm, self.r_out, self.h_out)

    def backward(self, **kw):
        self.layer.backward(self.dro, self.dho, self.h, self.r_out, self.wg, self.wu, self.wd, self.norm, **self.out, **kw)

    def reference(self):
        """torch autograd in 64 bits with the experts chosen by the library."""
        leaf = lambda t: t.double().requires_grad_(True)  # noqa: E731
        h, res, wg, wu, wd, wp, wr, gate = map(leaf, (self.h, self.res, self.wg, self.wu, self.wd, self.w_post, self.w_pre, self.gate))
        idx = self.layer.route.expert_idx.long()
        L = h @ wg
        # SoftTopk (Eq. 6, temperature 1): k softmaxes, level j over all but the j largest entries
        A, taken = torch.zeros_like(L), torch.zeros_like(L, dtype=torch.bool)
        order = L.detach().sort(dim=1, descending=True, stable=True).indices
        for j in range(self.k):
            A = A + L.masked_fill(taken, float("-inf")).softmax(dim=1)
            taken = taken.scatter(1, order[:, j:j + 1], True)
        wuT = wu if self.L == 0 else wu.transpose(1, 2)
        wdT = wd if self.L == 0 else wd.transpose(1, 2)
        y = torch.zeros_like(h)
        for e in range(self.E):
            tok = (idx == e).any(dim=1).nonzero()[:, 0]
            pre = h[tok] @ wuT[e]
            g, u = pre[:, :self.f], pre[:, self.f:]
            y = y.index_add(0, tok, A[tok, e][:, None] * ((g * g.sigmoid() * u) @ wdT[e]))
        rms = lambda v: (v.square().mean(1, keepdim=True) + EPS).sqrt()  # noqa: E731
        r = 0.8 * res + gate[torch.arange(self.T, device=DEV) // self.rpg] * (y / rms(y) * wp)
        ho = r / rms(r) * wr
        ((r * self.dro.double()).sum() + (ho * self.dho.double()).sum()).backward()
        return r.detach(), ho.detach(), dict(dh=h.grad, dr=res.grad, dw_gate=wg.grad, dw_up=wu.grad, dw_down=wd.grad, dw_post=wp.grad,
                                             dgate=gate.grad, dw_pre=wr.grad)


def check(got, ref, dtype, what):
    d = got.double() - ref
    assert torch.isfinite(d).all(), what
    if dtype == "f32":
        assert d.abs().max() <= 1e-4 * ref.abs().max(), f"{what}: {float(d.abs().max() / ref.abs().max()):.2e}"
    else:
        rel = float(d.square().mean().sqrt() / ref.square().mean().sqrt())
        assert rel <= 4e-2, f"{what}: {rel:.2e}"


@pytest.mark.parametrize("T,d,E,k,f,cf,dtype,layout,gates", [
    (96, 64, 8, 2, 40, 1.0, "f32", 0, 1), (130, 128, 5, 3, 72, 1.3, "f32", 1, 3), (1, 64, 4, 2, 32, 1.0, "f32", 0, 1),
    (512, 256, 8, 2, 128, 1.0, "bf16", 0, 1), (777, 200, 12, 4, 136, 1.25, "bf16", 1, 4), (1, 128, 16, 2, 64, 1.0, "bf16", 1, 1),
    (64, 512, 16, 2, 256, 1.0, "bf16", 0, 2),
])
def test_layer_forward_and_backward(ms, T, d, E, k, f, cf, dtype, layout, gates):
    s = Setup(ms, T, d, E, k, f, cf, dtype, layout, gates)
    s.forward()
    s.backward()
    torch.cuda.synchronize()
    assert ms.read_stats(s.layer.route.stats).status == 0 and ms.check_internal(s.layer.ctx) == 0
    r, ho, grads = s.reference()
    check(s.r_out, r, dtype, "r_out")
    check(s.h_out, ho, dtype, "h_out")
    for name, ref in grads.items():
        check(s.out[name], ref, dtype, name)


def test_layer_accumulates_and_serves_from_a_graph(ms):
    s = Setup(ms, 64, 128, 8, 2, 64, 1.0, "bf16", 0, 1)
    s.forward()
    s.backward()
    once = {n: t.clone() for n, t in s.out.items()}
    s.backward(accumulate=1)
    for n in ("dw_up", "dw_down"):
        assert torch.equal(s.out[n], 2 * once[n])
    want = s.r_out.clone(), s.h_out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.forward()
        s.backward()
    for t in (s.r_out, s.h_out, *s.out.values()):
        t.fill_(float("nan"))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(s.r_out, want[0]) and torch.equal(s.h_out, want[1])
    for n, t in s.out.items():
        if n == "dw_gate":                                   # the router's own gradient
            assert torch.allclose(t, once[n], rtol=1e-4, atol=1e-5)
        else:
            assert torch.equal(t, once[n]), n


def test_layer_without_training_keeps_nothing(ms):
    from paper_2508_12801_b200.layer import MoELayer
    s = Setup(ms, 32, 128, 8, 2, 64, 1.0, "bf16", 1, 1)
    s.forward()
    serve = MoELayer(s.layer.ctx.params, 64, 1, training=False)
    r, h = torch.empty_like(s.r_out), torch.empty_like(s.h_out)
    serve.forward(s.h, s.res, s.wg, s.wu, s.wd, s.norm, r, h)
    assert torch.equal(r, s.r_out) and torch.equal(h, s.h_out)
    with pytest.raises(ValueError):
        serve.backward(s.dro, s.dho, s.h, r, s.wg, s.wu, s.wd, s.norm, **s.out)
