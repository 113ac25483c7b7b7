"""Routing by top-k against its definition in 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F64 = torch.float64


@pytest.fixture(scope="module")
def ms():
    from paper_2508_12801_b200 import binding
    return binding


def scores64(l, sigmoid):
    l = l.to(F64)
    return torch.sigmoid(l) if sigmoid else torch.softmax(l, 1)


def choose64(l, bias, k, sigmoid, groups=1, keep=1, pairs=False):
    """The chosen experts, ascending: stable sorts put the lowest of equal indices first."""
    T, E = l.shape
    c = scores64(l, sigmoid)
    if bias is not None:
        c = c + bias.to(F64)
    by = c if bias is not None else l.to(F64)
    ok = torch.ones(T, E, dtype=torch.bool)
    if groups > 1:
        v = (c if pairs or bias is not None else by).view(T, groups, -1).sort(dim=2, descending=True).values
        v = v[:, :, :2].sum(2) if pairs else v[:, :, 0]
        best = v.sort(dim=1, descending=True, stable=True).indices[:, :keep]
        ok = torch.zeros(T, groups, dtype=torch.bool).scatter_(1, best, True).repeat_interleave(E // groups, 1)
    # what cannot be chosen goes behind -inf: two stable sorts, the first by value
    order = by.sort(dim=1, descending=True, stable=True).indices
    order = order.gather(1, ok.gather(1, order).to(torch.int8).sort(dim=1, descending=True, stable=True).indices)
    return order[:, :k].sort(1).values


def weights64(s, idx, renorm, scale):
    w = s.gather(1, idx)
    return scale * (w / (w.sum(1, keepdim=True) + 1e-20) if renorm else w)


def rel_tol(l):
    """Steps of 2^-24 that a weight may be off: the rounding of l - max (|l - max| of them), the exponential (4), its row's sum (9), the
    quotients (2), the sum of the chosen (9), the product with the scale (1), rounded up."""
    l = l.to(F64)
    spread = torch.where(torch.isfinite(l), l.amax(1, keepdim=True) - l, torch.zeros_like(l)).amax(1, keepdim=True)
    return (spread + 28) * 2.0 ** -24


def run(ms, l, bias, k, how, want_scores=True):
    T, E = l.shape
    ctx = ms.create(ms.make_params(T, 64, E, k, capacity=T), DEV)
    s = torch.full((T, E), -7.0, device=DEV) if want_scores else None
    idx, w = torch.full((T, k), -7, dtype=torch.int32, device=DEV), torch.full((T, k), -7.0, device=DEV)
    ms.topk_fwd(ctx, l.to(DEV), None if bias is None else bias.to(DEV), how, s, idx, w)
    torch.cuda.synchronize()
    return (None if s is None else s.cpu()), idx.cpu().long(), w.cpu()


def check(ms, l, bias, k, sigmoid, renorm=True, scale=1.0, groups=1, keep=1, pairs=False):
    how = ms.make_topk(ms.SIGMOID if sigmoid else ms.SOFTMAX, groups, keep, pairs, renorm, scale)
    s, idx, w = run(ms, l, bias, k, how)
    want = choose64(l, bias, k, sigmoid, groups, keep, pairs)
    assert torch.equal(idx, want), f"{(idx != want).any(1).sum()} rows differ"
    ref = scores64(l, sigmoid)
    tol = rel_tol(l)
    assert ((s.to(F64) - ref).abs() <= tol * ref + 2.0 ** -125).all()
    rw = weights64(ref, want, renorm, scale)
    tiny = 2.0 ** -125 * (scale if not renorm else 1e21 * scale)        # scores below 2^-126 may have become zero
    assert ((w.to(F64) - rw).abs() <= 2 * tol * rw + min(tiny, 1e-15)).all()
    _, idx2, w2 = run(ms, l, bias, k, how, want_scores=False)
    assert torch.equal(idx, idx2) and torch.equal(w, w2)


SHAPES = [(1, 8, 2, 1, 1), (1, 64, 8, 1, 1), (5, 1, 1, 1, 1), (7, 33, 5, 3, 2), (777, 12, 3, 4, 2), (513, 60, 4, 5, 3), (100, 96, 8, 4, 1),
          (1000, 127, 7, 1, 1), (3000, 128, 8, 8, 4), (129, 128, 8, 32, 2), (64, 32, 8, 32, 8), (40, 65, 8, 13, 2), (9, 8, 8, 1, 1)]


@pytest.mark.parametrize("T, E, k, groups, keep", SHAPES)
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("with_bias", [False, True])
def test_forward(ms, T, E, k, groups, keep, sigmoid, with_bias):
    g = torch.Generator().manual_seed(T * 131 + E * 7 + k)
    l = torch.randn(T, E, generator=g) * 2
    bias = torch.randn(E, generator=g) * 0.05 if with_bias else None
    for pairs in ([False, True] if groups > 1 else [False]):
        for renorm, scale in ((True, 2.5), (False, 1.0)):
            check(ms, l, bias, k, sigmoid, renorm, scale, groups, keep, pairs)


@pytest.mark.parametrize("E, k, groups, keep", [(8, 2, 1, 1), (33, 5, 3, 2), (64, 8, 8, 4), (128, 8, 1, 1), (128, 6, 16, 3)])
@pytest.mark.parametrize("sigmoid", [False, True])
def test_ties_go_to_the_lowest_index(ms, E, k, groups, keep, sigmoid):
    g = torch.Generator().manual_seed(E)
    l = torch.randint(-2, 3, (400, E), generator=g).float()
    l[:3] = torch.tensor([0.0, -0.0, 5.0])[:, None]
    l[3, ::2] = -0.0
    l[3, 1::2] = 0.0
    for bias in (None, torch.zeros(E), torch.randint(0, 2, (E,), generator=g) * 0.25):
        for pairs in ([False, True] if groups > 1 else [False]):
            check(ms, l, bias, k, sigmoid, groups=groups, keep=keep, pairs=pairs)


@pytest.mark.parametrize("sigmoid", [False, True])
def test_values_that_only_64_bits_tell_apart(ms, sigmoid):
    """Every expert's score + bias is 1 + e_i with e_i a few 1e-9: fp32 sees ties."""
    E, T, k = 64, 200, 8
    g = torch.Generator().manual_seed(5)
    l = (torch.randn(1, E, generator=g) * 2).expand(T, E).contiguous() + torch.randn(T, 1, generator=g) * (0.0 if sigmoid else 1.0)
    s = scores64(l[:1], sigmoid)[0]
    bias = (1.0 - s).float()                                  # rounding leaves differences of up to 2^-25
    check(ms, l, bias, k, sigmoid)
    check(ms, l, bias, k, sigmoid, groups=8, keep=3, pairs=True)
    check(ms, l, bias, k, sigmoid, groups=8, keep=3, pairs=False)


def test_sums_of_two_that_only_64_bits_tell_apart(ms):
    """Without a bias the groups' sums need 64 bits, the experts in them do not: big logits saturate in 64 bits too."""
    g = torch.Generator().manual_seed(6)
    l = torch.randint(0, 3, (300, 64), generator=g).float() + torch.randint(0, 4, (300, 64), generator=g) * 2.0 ** -22
    check(ms, l, None, 8, True, groups=8, keep=3, pairs=True)
    check(ms, l + 60, None, 8, True, groups=8, keep=3, pairs=True)
    check(ms, l, None, 8, False, groups=8, keep=3, pairs=True)


@pytest.mark.parametrize("sigmoid", [False, True])
def test_infinite_logits_and_biases(ms, sigmoid):
    g = torch.Generator().manual_seed(7)
    l = torch.randn(500, 40, generator=g)
    l[torch.rand(500, 40, generator=g) < 0.5] = -math.inf
    l[:, 3] = 1.0                                             # something is left in every row
    check(ms, l, None, 6, sigmoid)
    bias = torch.randn(40, generator=g) * 0.1
    bias[::3] = -math.inf
    check(ms, l, bias, 6, sigmoid)
    check(ms, l, bias, 6, sigmoid, groups=5, keep=2, pairs=True)
    check(ms, l, None, 6, sigmoid, renorm=False)


@pytest.mark.parametrize("l0", [-200.0, -95.0, 90.0, 3e38, -3e38])
def test_far_logits(ms, l0):
    g = torch.Generator().manual_seed(8)
    l = torch.randn(50, 16, generator=g) + l0
    for sigmoid in (False, True):
        check(ms, l, None, 4, sigmoid)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_rows_that_are_not_finite(ms, bad):
    g = torch.Generator().manual_seed(9)
    l = torch.randn(300, 128, generator=g)
    rows = torch.arange(0, 300, 3)
    l[rows, torch.randint(0, 128, (100,), generator=g)] = bad
    l[6] = math.nan
    l[9] = -math.inf
    for bias in (None, torch.zeros(128)):
        for groups, keep in ((1, 1), (8, 4)):
            how = ms.make_topk(ms.SOFTMAX, groups, keep, True)
            _, idx, w = run(ms, l, bias, 8, how)
            assert (idx >= 0).all() and (idx < 128).all() and (idx[:, 1:] > idx[:, :-1]).all()
            assert w[rows].isnan().all() and w[6].isnan().all() and w[9].isnan().all()
            keep_rows = torch.ones(300, dtype=torch.bool)
            keep_rows[rows] = False
            assert torch.equal(idx[keep_rows], choose64(l, bias, 8, False, groups, keep, True)[keep_rows]) and w[keep_rows].isfinite().all()


# From some 2 400 tokens on eight lanes own a token instead of a warp (where groups are whole lanes): the same again with rows enough for that.
MANY = 2601          # no multiple of the four tokens of a warp


def many(l):
    return l.repeat(-(-MANY // l.shape[0]), 1)[:MANY].contiguous()


@pytest.mark.parametrize("E, k, groups, keep", [(1, 1, 1, 1), (2, 2, 1, 1), (8, 2, 2, 1), (12, 3, 3, 2), (16, 8, 4, 3), (16, 2, 8, 1), (32, 8, 4, 1), (31, 8, 1, 1),
                                                (33, 5, 1, 1), (40, 6, 5, 3), (64, 8, 8, 4), (64, 1, 2, 1), (96, 8, 3, 2), (100, 7, 1, 1), (127, 8, 1, 1),
                                                (128, 8, 8, 4), (128, 6, 4, 1), (128, 8, 2, 1), (128, 8, 1, 1)])
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("with_bias", [False, True])
def test_many_tokens(ms, E, k, groups, keep, sigmoid, with_bias):
    g = torch.Generator().manual_seed(E * 7 + k)
    l = torch.randn(MANY, E, generator=g) * 2
    l[:200] = torch.randint(-1, 2, (200, E), generator=g).float()            # ties
    l[200:210] = 0.5
    l[210:300][torch.rand(90, E, generator=g) < 0.4] = -math.inf
    l[210:300, E // 2] = 1.0                                              # something is left in every row
    bias = (torch.randn(E, generator=g) * 0.05 if E % 3 else torch.randint(0, 2, (E,), generator=g) * 0.25) if with_bias else None
    for pairs in ([False, True] if groups > 1 else [False]):
        check(ms, l, bias, k, sigmoid, True, 2.5, groups, keep, pairs)
    check(ms, l, bias, k, sigmoid, False, 1.0, groups, keep)


@pytest.mark.parametrize("T", [130, MANY])
@pytest.mark.parametrize("E, groups, keep", [(128, 8, 4), (33, 3, 2), (64, 1, 1), (8, 4, 1)])
@pytest.mark.parametrize("sigmoid", [False, True])
def test_rows_of_one_value(ms, T, E, groups, keep, sigmoid):
    """Padded tokens: every expert has the same logit; between them ordinary rows and rows that differ in the last bit of one expert."""
    g = torch.Generator().manual_seed(E)
    l = torch.randn(T, E, generator=g)
    l[::2] = torch.randn(len(l[::2]), 1, generator=g)
    l[4::10, E // 2] = torch.nextafter(l[4::10, E // 2], torch.tensor(9.0))
    l[6::10] = 0.0
    l[6::10, ::3] = -0.0
    k = min(8, E // groups * keep)
    for bias in (None, torch.zeros(E), torch.full((E,), 0.3), torch.randn(E, generator=g) * 0.05):
        for pairs in ([False, True] if groups > 1 else [False]):
            check(ms, l, bias, k, sigmoid, groups=groups, keep=keep, pairs=pairs)


@pytest.mark.parametrize("sigmoid", [False, True])
def test_many_tokens_that_only_64_bits_tell_apart(ms, sigmoid):
    g = torch.Generator().manual_seed(5)
    E, k = 128, 8
    l = (torch.randn(1, E, generator=g) * 2).expand(40, E).contiguous() + torch.randn(40, 1, generator=g) * (0.0 if sigmoid else 1.0)
    bias = (1.0 - scores64(l[:1], sigmoid)[0]).float()
    check(ms, many(l), bias, k, sigmoid)
    check(ms, many(l), bias, k, sigmoid, groups=8, keep=3, pairs=True)
    l = torch.randint(0, 3, (300, 64), generator=g).float() + torch.randint(0, 4, (300, 64), generator=g) * 2.0 ** -22
    check(ms, many(l), None, 8, sigmoid, groups=8, keep=3, pairs=True)
    # the ten largest in one lane's consecutive experts, the ninth as near to the eighth as 64 bits see it
    l = torch.randn(300, E, generator=g) - 8
    l[:, 32:42] = torch.linspace(1.0, 2.0, 10).flip(0)
    l[:, 41] = l[:, 40]
    bias = torch.zeros(E)
    bias[41] = 2.0 ** -40
    check(ms, many(l), bias, 8, sigmoid)
    l[:, 40] = l[:, 39]
    bias[39] = 2.0 ** -41
    check(ms, many(l), bias, 8, sigmoid)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_many_rows_that_are_not_finite(ms, bad):
    g = torch.Generator().manual_seed(9)
    for E, groups, keep in ((128, 1, 1), (128, 8, 4), (33, 1, 1), (64, 4, 2)):
        l = torch.randn(MANY, E, generator=g)
        rows = torch.arange(0, MANY, 3)
        l[rows, torch.randint(0, E, (len(rows),), generator=g)] = bad
        l[6] = -math.nan
        l[9] = -math.inf
        for bias in (None, torch.zeros(E)):
            _, idx, w = run(ms, l, bias, 8, ms.make_topk(ms.SOFTMAX, groups, keep, True))
            assert (idx >= 0).all() and (idx < E).all() and (idx[:, 1:] > idx[:, :-1]).all()
            assert w[rows].isnan().all()
            fine = torch.ones(MANY, dtype=torch.bool)
            fine[rows] = False
            assert torch.equal(idx[fine], choose64(l, bias, 8, False, groups, keep, True)[fine]) and w[fine].isfinite().all()


def dl64(l, idx, dw, col, sigmoid, renorm, scale):
    l = l.to(F64).requires_grad_(True)
    s = torch.sigmoid(l) if sigmoid else torch.softmax(l, 1)
    w = weights64(s, idx, renorm, scale)
    loss = (w * dw.to(F64)).sum() + (0 if col is None else (s * col.to(F64)).sum())
    return torch.autograd.grad(loss, l)[0]


def backward(ms, l, idx, dw, col, how):
    T, E = l.shape
    ctx = ms.create(ms.make_params(T, 64, E, idx.shape[1], capacity=T), DEV)
    dl = torch.full((T, E), -7.0, device=DEV)
    ms.topk_bwd(ctx, l.to(DEV), idx.to(torch.int32).to(DEV), dw.to(DEV), None if col is None else col.to(DEV), how, dl)
    torch.cuda.synchronize()
    return dl.cpu().to(F64)


@pytest.mark.parametrize("T, E, k, groups, keep", SHAPES + [(MANY, E, k, 1, 1) for E, k in ((1, 1), (2, 2), (8, 2), (12, 3), (16, 8), (32, 8), (31, 8), (33, 5), (40, 6),
                                                                                            (64, 8), (96, 1), (100, 7), (127, 8), (128, 8))])
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("aux", [False, True])
def test_backward(ms, T, E, k, groups, keep, sigmoid, aux):
    g = torch.Generator().manual_seed(T * 17 + E + k)
    l = torch.randn(T, E, generator=g) * 2
    idx = torch.rand(T, E, generator=g).topk(k, 1).indices.sort(1).values
    dw = torch.randn(T, k, generator=g)
    col = torch.randn(E, generator=g) if aux else None
    for renorm, scale in ((True, 2.5), (False, 1.0)):
        how = ms.make_topk(ms.SIGMOID if sigmoid else ms.SOFTMAX, 1, 1, False, renorm, scale)
        got, want = backward(ms, l, idx, dw, col, how), dl64(l, idx, dw, col, sigmoid, renorm, scale)
        # dl_e = s_e (its own terms + a sum over the row): each term is off by the steps of rel_tol at most, and so is s_e
        s = scores64(l, sigmoid)
        p = s.gather(1, idx)
        S = p.sum(1, keepdim=True) + 1e-20 if renorm else torch.ones(T, 1, dtype=F64)
        own = scale * dw.to(F64).abs() / S
        if renorm:
            own = own + (own * p).sum(1, keepdim=True) / S
        mag = torch.zeros(T, E, dtype=F64).scatter_(1, idx, own)
        if aux:
            mag = mag + col.to(F64).abs()
        mag = s * (mag * (1 - s) if sigmoid else mag + (mag * s).sum(1, keepdim=True))
        assert ((got - want).abs() <= 4 * rel_tol(l) * mag + 1e-30).all()


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("renorm", [False, True])
def test_backward_against_differences(ms, sigmoid, renorm):
    g = torch.Generator().manual_seed(3)
    T, E, k = 3, 12, 4
    l = torch.randn(T, E, generator=g)
    idx = torch.rand(T, E, generator=g).topk(k, 1).indices.sort(1).values
    dw, col = torch.randn(T, k, generator=g), torch.randn(E, generator=g)
    how = ms.make_topk(ms.SIGMOID if sigmoid else ms.SOFTMAX, renorm=renorm, scale=1.5)
    got = backward(ms, l, idx, dw, col, how)

    def loss(x):
        s = scores64(x, sigmoid)
        return (weights64(s, idx, renorm, 1.5) * dw.to(F64)).sum(1) + (s * col.to(F64)).sum(1)
    h = 1e-4
    for e in range(E):
        up, down = l.to(F64).clone(), l.to(F64).clone()
        up[:, e] += h
        down[:, e] -= h
        # third derivatives of these are below 10 times the gradients' scale, 10 in all: h^2 10 / 6 < 2e-8; fp32 results 1e-5 of it
        assert ((loss(up) - loss(down)) / (2 * h) - got[:, e]).abs().max() <= 1e-4


def test_backward_skips_empty_pairs(ms):
    g = torch.Generator().manual_seed(4)
    l, dw = torch.randn(20, 16, generator=g), torch.randn(20, 3, generator=g)
    idx = torch.rand(20, 16, generator=g).topk(3, 1).indices.sort(1).values
    empty_pairs(ms, l, dw, idx, lambda got: got)
    tile = lambda t: t.repeat(131, 1)  # noqa: E731
    for j in (0, 7, 130):
        empty_pairs(ms, l, dw, idx, lambda all_rows: all_rows.view(131, 20, 16)[j], tile)


def empty_pairs(ms, l, dw, idx, part, tile=lambda t: t):
    short = idx.clone()
    short[:, 2] = -1
    short[5] = -1
    short[6, 1] = 16
    for sigmoid in (False, True):
        how = ms.make_topk(ms.SIGMOID if sigmoid else ms.SOFTMAX)
        got = part(backward(ms, tile(l), tile(short), tile(dw), None, how))
        want = dl64(l, idx[:, :2], dw[:, :2], None, sigmoid, True, 1.0)
        rows = [i for i in range(20) if i not in (5, 6)]
        assert (got[rows] - want[rows]).abs().max() <= 1e-5 * want.abs().max()
        assert (got[5] == 0).all()
        assert torch.isfinite(got).all()
        one = dl64(l, idx[:, :1], dw[:, :1], None, sigmoid, True, 1.0)
        assert (got[6] - one[6]).abs().max() <= 1e-5 * want.abs().max()


def test_many_tokens_and_graph_replay(ms):
    """The largest batch, twice from a captured graph with new logits in between, and two contexts on two streams."""
    T, E, k = 65536, 128, 8
    ctx = ms.create(ms.make_params(T, 64, E, k), DEV)
    how = ms.make_topk(ms.SIGMOID, 8, 4, True, True, 2.5)
    g = torch.Generator().manual_seed(11)
    a, b = torch.randn(T, E, generator=g).to(DEV), torch.randn(T, E, generator=g).to(DEV)
    bias = (torch.randn(E, generator=g) * 0.05).to(DEV)
    l = a.clone()
    out = lambda: (torch.empty(T, E, device=DEV), torch.empty(T, k, dtype=torch.int32, device=DEV), torch.empty(T, k, device=DEV))  # noqa: E731
    eager = [out(), out()]
    for x, o in zip((a, b), eager):
        ms.topk_fwd(ctx, x, bias, how, *o)
    torch.cuda.synchronize()
    graph, o = torch.cuda.CUDAGraph(), out()
    with torch.cuda.graph(graph):
        ms.topk_fwd(ctx, l, bias, how, *o)
    for x, e in ((a, eager[0]), (b, eager[1])):
        l.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(o, e))
    idx = choose64(a.cpu(), bias.cpu(), k, True, 8, 4, True)
    assert torch.equal(eager[0][1].cpu().long(), idx)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    ctxs = [ctx, ms.create(ms.make_params(T, 64, E, k), DEV)]
    twice = [out(), out()]
    torch.cuda.synchronize()
    for st, c, x, o in zip(streams, ctxs, (a, b), twice):
        ms.topk_fwd(c, x, bias, how, *o, stream=st)
    torch.cuda.synchronize()
    for e, o in zip(eager, twice):
        assert all(torch.equal(p, q) for p, q in zip(o, e))


def test_router_of_a_layer(ms):
    """gate, topk, index build, dispatch, combine, and back: the calls in the order a router makes them, against torch in 64 bits."""
    T, d, E, k = 300, 64, 16, 3
    g = torch.Generator().manual_seed(12)
    H, W = torch.randn(T, d, generator=g), torch.randn(d, E, generator=g) * d ** -0.5
    dY = torch.randn(T, d, generator=g)
    ctx = ms.create(ms.make_params(T, d, E, k, capacity=T, io_dtype=ms.F32), DEV)
    how = ms.make_topk(ms.SIGMOID, 4, 2, True, True, 1.5)
    b = ms.RouterBuffers(ctx)
    Hd, Wd, dYd = H.to(DEV), W.to(DEV), dY.to(DEV)
    ms.gate(ctx, Hd, Wd, None, b.logits)
    ms.topk_fwd(ctx, b.logits, None, how, b.scores, b.expert_idx, b.gate_w)
    ms.index_build(ctx, b.expert_idx, b.slot_idx, b.slot_token, b.expert_load)
    x, y = torch.empty(E, T, d, device=DEV), torch.empty(T, d, device=DEV)
    ms.dispatch(ctx, Hd, b.expert_idx, b.slot_idx, b.slot_token, x)
    ms.combine(ctx, x, b.expert_idx, b.slot_idx, b.gate_w, y)            # identity experts
    loss, col = torch.empty(1, dtype=torch.float64, device=DEV), torch.empty(E, device=DEV)
    ms.aux_loss(ctx, b.scores, b.expert_load, 0.3, loss, col)
    dx, dgw, dL = torch.empty_like(x), torch.empty_like(b.gate_w), torch.empty_like(b.logits)
    dW, dH = torch.empty(d, E, device=DEV), torch.empty(T, d, device=DEV)
    ms.combine_bwd(ctx, dYd, x, b.expert_idx, b.slot_idx, b.gate_w, b.slot_token, dx, dgw)
    ms.topk_bwd(ctx, b.logits, b.expert_idx, dgw, col, how, dL)
    ms.gate_bwd(ctx, Hd, Wd, dL, dW, dH)
    ms.combine(ctx, dx, b.expert_idx, b.slot_idx, None, dH, accumulate=1)
    torch.cuda.synchronize()
    idx = choose64(b.logits.cpu(), None, k, True, 4, 2, True)
    assert torch.equal(b.expert_idx.cpu().long(), idx)
    load = torch.bincount(idx.flatten(), minlength=E)
    assert torch.equal(b.expert_load.cpu().long(), load)
    h64, w64 = H.to(F64).requires_grad_(True), W.to(F64).requires_grad_(True)
    s = torch.sigmoid(h64 @ w64)
    wt = weights64(s, idx, True, 1.5)
    y64 = wt.sum(1, keepdim=True) * h64
    aux = 0.3 / (E * T * T) * (s.sum(0) * load).sum()
    gh, gw = torch.autograd.grad((y64 * dY.to(F64)).sum() + aux, (h64, w64))
    assert (y.cpu() - y64.detach()).abs().max() <= 1e-5 * y64.abs().max()
    assert abs(loss.item() - aux.item()) <= 1e-6 * aux.item()
    assert (dH.cpu() - gh).abs().max() <= 1e-5 * gh.abs().max()
    # The experts are the identity and the weights sum to 1.5, so y does not depend on the logits: what comes through the weights,
    # G_i (1 - sum p / S) / S times s (1 - s) for the chosen with G_i = 1.5 <dY_i, H_i>, cancels and leaves its rounding.  Steps of 2^-24
    # of G_i s (1 - s) / S on the way: s and 1 - s 8, S 4, its inverse 2, products and sums of G p 5, mean 2, difference 1, products 2: 24.
    p64 = s.detach().gather(1, idx)
    G = 1.5 * (dY * H).to(F64).sum(1, keepdim=True).abs() / p64.sum(1, keepdim=True)
    left = torch.zeros(T, E, dtype=F64).scatter_(1, idx, G * p64 * (1 - p64)) * 24 * 2.0 ** -24
    assert ((dW.cpu() - gw).abs() <= H.abs().to(F64).T @ left + 1e-5 * gw.abs().max()).all()


def test_other_device_and_refusals(ms):
    ctx = ms.create(ms.make_params(4, 64, 8, 2, capacity=4), DEV)
    how = ms.make_topk()
    l, i, w = torch.zeros(4, 8, device=DEV), torch.zeros(4, 2, dtype=torch.int32, device=DEV), torch.zeros(4, 2, device=DEV)
    with pytest.raises(ValueError, match="logits"):
        ms.topk_fwd(ctx, l.cpu(), None, how, None, i, w)
    with pytest.raises(ValueError, match="logits"):
        ms.topk_fwd(ctx, torch.zeros(8, 4, device=DEV).t(), None, how, None, i, w)
    with pytest.raises(ms.MaxScoreError):
        ms.topk_fwd(ctx, l, None, how, l, i, w)
    with pytest.raises(ms.MaxScoreError):
        ms.topk_fwd(ctx, l, None, ms.make_topk(n_group=3), None, i, w)
