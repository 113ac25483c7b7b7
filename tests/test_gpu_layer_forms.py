"""The forms of the MoE layer: routing by top-k, activations kept in 8 bits, experts in 8-bit integers, against the same layer in
64 bits with the chosen experts held constant.  Bars as for the layer in its usual form: fp32 1e-4 of a tensor's largest entry; bf16 4e-2 of its
root mean square (ten roundings of 2^-8).  Eight-bit forms add the roundings of what they hold in 8 bits: uniform within half a step of
amax / 127, an rms of amax / 440.  A block of 32 kept values has amax near 2.2 rms (0.5 %), twice (g and u); rows and columns of 100 to
256 values 3 to 4 rms, of gated values up to 9 (1 % and 2 %): x, w_up (each through g and u), h, w_down: 1 % * 2 + 2 % + 1 %, as independent
errors 3.5 %.  Bars 4e-2 + 1e-2 and 4e-2 + 3.5e-2."""
import pytest
import torch

from test_gpu_layer import DEV, EPS, Setup, check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ms():
    from paper_2508_12801_b200 import binding
    return binding


def make(ms, T, d, E, k, f, cf, dtype, layout, topk, seed=0, **form):
    from paper_2508_12801_b200.layer import MoELayer
    s = Setup(ms, T, d, E, k, f, cf, dtype, layout, 1, seed)
    s.layer = MoELayer(s.layer.ctx.params, f, layout, topk=topk, **form)
    return s


def reference(s, topk, bias=None, col=None):
    """The layer in 64 bits with the library's choice; pairs beyond an expert's capacity are left out, their scores count."""
    leaf = lambda t: t.double().requires_grad_(True)  # noqa: E731
    h, res, wg, wu, wd, wp, wr, gate = map(leaf, (s.h, s.res, s.wg, s.wu, s.wd, s.w_post, s.w_pre, s.gate))
    idx, slot = s.layer.route.expert_idx.long(), s.layer.route.slot_idx
    L = h @ wg
    A = L.sigmoid() if topk.score else L.softmax(1)
    p = A.gather(1, idx)
    w = topk.scale * (p / (p.sum(1, keepdim=True) + 1e-20) if topk.renorm else p)
    wuT, wdT = (wu, wd) if s.L == 0 else (wu.transpose(1, 2), wd.transpose(1, 2))
    y = torch.zeros_like(h)
    for e in range(s.E):
        tok, c = ((idx == e) & (slot < s.layer.ctx.capacity)).nonzero(as_tuple=True)
        pre = h[tok] @ wuT[e]
        y = y.index_add(0, tok, w[tok, c][:, None] * ((torch.nn.functional.silu(pre[:, :s.f]) * pre[:, s.f:]) @ wdT[e]))
    rms = lambda v: (v.square().mean(1, keepdim=True) + EPS).sqrt()  # noqa: E731
    r = 0.8 * res + gate * (y / rms(y) * wp)
    ho = r / rms(r) * wr
    loss = (r * s.dro.double()).sum() + (ho * s.dho.double()).sum()
    if col is not None:
        loss = loss + (A * col.double()).sum()
    names = ("dh", "dr", "dw_gate", "dw_up", "dw_down", "dw_post", "dgate", "dw_pre")
    return r.detach(), ho.detach(), dict(zip(names, torch.autograd.grad(loss, (h, res, wg, wu, wd, wp, gate, wr))))


def close(got, ref, dtype, what, more=0.0):
    if dtype == "f32":
        return check(got, ref, dtype, what)
    d = got.double() - ref
    assert torch.isfinite(d).all(), what
    rel = float(d.square().mean().sqrt() / ref.square().mean().sqrt())
    assert rel <= 4e-2 + more, f"{what}: {rel:.2e}"


CASES = [(96, 64, 8, 2, 40, 2.0, "f32", 0, dict(score=0)), (130, 128, 6, 3, 72, 1.1, "f32", 1, dict(score=1, scale=1.5, n_group=3, topk_group=2)),
         (1, 128, 16, 2, 64, 1.0, "bf16", 1, dict(score=1, renorm=True)), (777, 208, 12, 4, 144, 1.25, "bf16", 1, dict(score=0, renorm=False, scale=3.0)),
         (512, 256, 8, 2, 128, 3.0, "bf16", 0, dict(score=1, n_group=4, topk_group=2, group_pairs=True, scale=2.5))]


@pytest.mark.parametrize("T, d, E, k, f, cf, dtype, layout, how", CASES)
@pytest.mark.parametrize("keep8", [False, True])
def test_training(ms, T, d, E, k, f, cf, dtype, layout, how, keep8):
    topk = ms.make_topk(**how)
    if keep8 and dtype == "f32":
        with pytest.raises(ValueError):
            make(ms, T, d, E, k, f, cf, dtype, layout, topk, keep8=True)
        return
    s = make(ms, T, d, E, k, f, cf, dtype, layout, topk, keep8=keep8)
    g = torch.Generator().manual_seed(1)
    bias = (torch.randn(E, generator=g) * 0.05).to(DEV)
    col = (torch.rand(E, generator=g) * 0.1).to(DEV)
    s.layer.forward(s.h, s.res, s.wg, s.wu, s.wd, s.norm, s.r_out, s.h_out, balance_bias=bias)
    s.layer.backward(s.dro, s.dho, s.h, s.r_out, s.wg, s.wu, s.wd, s.norm, **s.out, dscores_col=col)
    torch.cuda.synchronize()
    assert ms.check_internal(s.layer.ctx) == 0
    A = (s.layer.route.logits.double().sigmoid() if topk.score else s.layer.route.logits.double().softmax(1)) + bias.double()
    if topk.n_group > 1:
        v = A.view(T, topk.n_group, -1).sort(dim=2, descending=True).values
        v = v[:, :, :2].sum(2) if topk.group_pairs else v[:, :, 0]
        out = torch.ones(T, topk.n_group, dtype=torch.bool, device=DEV).scatter_(1, v.topk(topk.topk_group, 1).indices, False)
        A = A.masked_fill(out.repeat_interleave(E // topk.n_group, 1), float("-inf"))
    assert torch.equal(s.layer.route.expert_idx.long(), A.topk(k, 1).indices.sort(1).values)
    r, ho, grads = reference(s, topk, bias, col)
    close(s.r_out, r, dtype, "r_out")
    close(s.h_out, ho, dtype, "h_out")
    for name, ref in grads.items():
        close(s.out[name], ref, dtype, name, 1e-2 if keep8 else 0.0)


def test_keep8_with_the_paper_router(ms):
    """The same layer with and without 8-bit kept activations: the forward pass is the same, bit for bit, the gradients nearly."""
    from paper_2508_12801_b200.layer import MoELayer
    s = Setup(ms, 700, 256, 8, 2, 96, 1.0, "bf16", 0, 1)
    s.forward()
    s.backward()
    want = {n: t.clone() for n, t in s.out.items()}
    r, ho = s.r_out.clone(), s.h_out.clone()
    s.layer = MoELayer(s.layer.ctx.params, 96, 0, keep8=True)
    s.forward()
    s.backward()
    assert torch.equal(s.r_out, r) and torch.equal(s.h_out, ho)
    for n, t in s.out.items():
        close(t, want[n].double(), "bf16", n, 1e-2)


def test_two_layers_share_their_working_buffers(ms):
    """Forward through two layers, then backward through both: as with buffers of their own, bit for bit, eager and from a graph."""
    from paper_2508_12801_b200.layer import MoELayer
    topk = ms.make_topk(ms.SIGMOID, scale=1.5)
    a, b = (make(ms, 300, 128, 8, 2, 96, 2.0, "bf16", 0, topk, seed=i, keep8=True) for i in range(2))

    def step():
        for s in (a, b):
            s.forward()
        for s in (b, a):
            s.backward()

    step()
    want = [t.clone() for s in (a, b) for t in (s.r_out, s.h_out, *s.out.values())]
    b.layer = MoELayer(b.layer.ctx.params, 96, 0, topk=topk, keep8=True, share=a.layer)
    assert b.layer.x is a.layer.x and b.layer.h is a.layer.h and b.layer.dpre is a.layer.dpre
    assert b.layer.yexp is not a.layer.yexp and b.layer.keep is not a.layer.keep
    out = [t for s in (a, b) for t in (s.r_out, s.h_out, *s.out.values())]

    def same():
        torch.cuda.synchronize()
        for g, w in zip(out, want):
            assert torch.allclose(g, w, rtol=1e-4, atol=1e-4) if g.shape == a.out["dw_gate"].shape else torch.equal(g, w)
            g.fill_(float("nan"))
    for t in out:
        t.fill_(float("nan"))
    step()
    same()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    graph.replay()
    same()
    with pytest.raises(ValueError, match="share"):
        MoELayer(b.layer.ctx.params, 64, 0, topk=topk, keep8=True, share=a.layer)
    with pytest.raises(ValueError, match="share"):
        MoELayer(b.layer.ctx.params, 96, 0, topk=topk, share=a.layer)


@pytest.mark.parametrize("T, d, E, k, f, cf, layout", [(1, 128, 16, 2, 64, 1.0, 1), (64, 512, 16, 2, 256, 1.25, 0), (900, 256, 8, 2, 144, 2.0, 0)])
@pytest.mark.parametrize("router", ["topk", "flow"])
def test_serving_in_integers(ms, T, d, E, k, f, cf, layout, router):
    from paper_2508_12801_b200.layer import MoELayer
    topk = ms.make_topk(ms.SIGMOID) if router == "topk" else None
    s = make(ms, T, d, E, k, f, cf, "bf16", layout, topk, training=False)
    s.forward()
    r, ho, y = s.r_out.clone(), s.h_out.clone(), s.layer.yexp.clone()
    serve = MoELayer(s.layer.ctx.params, f, layout, training=False, topk=topk, int8=True)
    w_up, w_down = serve.quantise(s.wu, s.wd)
    serve.forward(s.h, s.res, s.wg, w_up, w_down, s.norm, s.r_out, s.h_out)
    torch.cuda.synchronize()
    assert ms.check_internal(serve.ctx) == 0
    assert torch.equal(serve.route.expert_idx, s.layer.route.expert_idx)
    close(serve.yexp, y.double(), "bf16", "yexp", 3.5e-2)
    close(s.r_out, r.double(), "bf16", "r_out", 3.5e-2)
    close(s.h_out, ho.double(), "bf16", "h_out", 3.5e-2)
    with pytest.raises(ValueError):
        serve.backward(s.dro, s.dho, s.h, s.r_out, s.wg, s.wu, s.wd, s.norm, **s.out)
    again = MoELayer(s.layer.ctx.params, f, layout, training=False, topk=topk, int8=True, share=serve)
    r1, h1 = torch.empty_like(s.r_out), torch.empty_like(s.h_out)
    again.forward(s.h, s.res, s.wg, w_up, w_down, s.norm, r1, h1)
    assert again.xq is serve.xq and torch.equal(r1, s.r_out) and torch.equal(h1, s.h_out)


def test_refusals(ms):
    from paper_2508_12801_b200.layer import MoELayer
    p = ms.make_params(16, 64, 4, 2, 1.0, io_dtype=ms.BF16)
    for kw in (dict(keep8=True, training=False), dict(int8=True), dict(int8=True, keep8=True)):
        with pytest.raises(ValueError):
            MoELayer(p, 64, **kw)
    with pytest.raises(ValueError):
        MoELayer(ms.make_params(16, 64, 4, 2, 1.0, io_dtype=ms.F32), 64, int8=True, training=False)
    s = Setup(ms, 16, 64, 4, 2, 64, 1.0, "bf16", 0, 1)
    with pytest.raises(ValueError, match="balance_bias"):
        s.layer.forward(s.h, s.res, s.wg, s.wu, s.wd, s.norm, s.r_out, s.h_out, balance_bias=torch.zeros(4, device=DEV))
    s.forward()
    with pytest.raises(ValueError, match="dscores_col"):
        s.backward(dscores_col=torch.zeros(4, device=DEV))
