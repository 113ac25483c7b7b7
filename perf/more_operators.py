"""Measured cases of top-k routing, of expert products in 8-bit integers and of expert activations kept in 8 bits.

Operators (`op` of a case):
  topk       scores of the experts, choice of k by score + balance bias within the best groups, combine weights
  topk_bwd   gradient of the logits through the combine weights (and of a balance loss through the scores)
  glu8       h = silu(x W_g) * (x W_u) per expert on rows and weights in 8-bit integers, a scale per row and per column
  gemm8      y = x W in the same form
  block8     the experts of a serving step from its bf16 token rows: quantise and dispatch, glu8, quantise, gemm8
  keep8      training step of the gated activation with [g | u] kept in 8 bits: forward, then the backward pass from what was kept
  keep8_bwd  the backward pass alone

Buffers are [E, C, width] with `load[e]` rows in use; what lies behind them is zero on output.  A row x in 8 bits is
q = rint(x * fp32(127 / amax)), its scale fp32(amax / 127); kept activations have a scale for each 32 columns of g and of u:
[E, C, 2, fp] integers and behind them, from a multiple of 256 bytes on, [E, 2 fp / 32, C] scales, fp = f rounded up to 32.
"""
import math

import torch

own = False

BF16 = torch.bfloat16
F32, F64 = torch.float32, torch.float64
BLOCK = 32          # columns that share a scale


def _topk(op, T, E, k, score, renorm, **kw):
    c = dict(op=op, T=T, E=E, k=k, score=score, renorm=renorm, groups=1, keep_groups=1, pairs=False, bias=False, scores=False,
             aux=False, scale=1.0, cf=1.0, d=64)
    c.update(kw)
    return c


def _rows(op, T, d, E, k, cf, f, layout=1):
    return dict(op=op, T=T, d=d, E=E, k=k, cf=cf, f=f, layout=layout)


def listed():
    def named(name, c):
        return dict(c, name=name)
    return [
        # one token of a serving loop
        named("topk one token", _topk("topk", 1, 64, 8, "softmax", True)),
        # the largest batch of the router's workloads: sigmoid scores, a balance bias, the better four of eight groups
        named("topk stress", _topk("topk", 65536, 128, 8, "sigmoid", True, groups=8, keep_groups=4, pairs=True, bias=True, scores=True,
                                   scale=2.5)),
        # an odd number of experts and tokens in training, weights as they come from the softmax, with the balance loss
        named("topk_bwd odd", _topk("topk_bwd", 777, 33, 5, "softmax", False, aux=True)),
        # the largest batch, training backward
        named("topk_bwd stress", _topk("topk_bwd", 65536, 128, 8, "sigmoid", True, scale=2.5)),
        # one token of a serving loop: eight experts with a row each, bound by the weights
        named("glu8 one token", _rows("glu8", 1, 2048, 64, 8, 1.0, 1024)),
        # the largest batch, second product of the experts
        named("gemm8 stress", _rows("gemm8", 65536, 4096, 128, 8, 1.0, 1024)),
        # a serving batch of 64 sequences on sixteen experts, all steps of the experts
        named("block8 batch 64", _rows("block8", 64, 1024, 16, 2, 1.25, 512)),
        # prompts of a serving step, an inner width that is no multiple of a tile
        named("block8 prompts", _rows("block8", 8192, 2048, 64, 8, 1.0, 1008)),
        # training step on few large experts
        named("keep8 k2e16", _rows("keep8", 4096, 1024, 16, 2, 1.0, 512, layout=0)),
        # the largest batch, training step
        named("keep8 stress", _rows("keep8", 65536, 4096, 128, 8, 1.0, 1024, layout=0)),
        # a short batch of fine-tuning: few rows an expert
        named("keep8_bwd short", _rows("keep8_bwd", 256, 2048, 64, 8, 1.0, 1024, layout=0)),
        # the skewed workload's ragged loads, an inner width that is no multiple of a tile
        named("keep8_bwd skew", _rows("keep8_bwd", 16384, 2048, 64, 8, 1.25, 1000, layout=1)),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["topk", "topk", "topk_bwd", "glu8", "gemm8", "block8", "keep8", "keep8_bwd"])
    if op in ("topk", "topk_bwd"):
        E, k, groups = rng.choice([(8, 2, 1), (8, 1, 2), (12, 3, 3), (16, 2, 4), (33, 5, 3), (60, 4, 1), (64, 6, 8), (64, 8, 1), (96, 8, 4),
                                   (128, 8, 8), (128, 8, 1), (127, 7, 1)])
        keep = 1 if groups == 1 else rng.randint(-(-k * groups // E), groups)
        return _topk(op, _log(rng, 1, 65536), E, k, rng.choice(["softmax", "sigmoid"]), rng.random() < 0.6, groups=groups, keep_groups=keep,
                     pairs=rng.random() < 0.5, bias=rng.random() < 0.5, scores=rng.random() < 0.5, aux=rng.random() < 0.4,
                     scale=rng.choice([1.0, 1.0, 2.5]))
    E, k = rng.choice([(8, 2), (12, 3), (16, 2), (33, 5), (64, 8), (128, 8)])
    cf = rng.choice([1.0, 1.1, 1.25, 1.5])
    step = 8 if op in ("keep8", "keep8_bwd") else 16
    d, f = step * _log(rng, 128 // step, 2560 // step), step * _log(rng, 64 // step, 1536 // step)
    return _rows(op, _log(rng, 1, 20000), d, E, k, cf, f, layout=rng.randrange(2) if step == 8 else 1)


def _capacity(c):
    return max(1, math.ceil(c["cf"] * c["T"] * c["k"] / c["E"] - 1e-9))


def _loads(c, C, gen):
    """Rows per expert: popularity like a Zipf law cut off at the capacity, T * k rows in all."""
    E, total = c["E"], c["T"] * c["k"]
    share = (torch.randperm(E, generator=gen).double() + 1.0) ** -1.1
    load, left = torch.zeros(E, dtype=torch.int64), total
    while left > 0:
        room = C - load
        s = torch.where(room > 0, share, torch.zeros(E, dtype=F64))
        add = torch.minimum(torch.floor(s / s.sum() * left).long(), room)
        if int(add.sum()) == 0:       # the last few rows, one each to the experts most asked for
            order = torch.argsort(s, descending=True, stable=True)
            order = order[room[order] > 0][:left]
            add = torch.zeros(E, dtype=torch.int64)
            add[order] = 1
        load, left = load + add, left - int(add.sum())
    return load


def _choices(T, E, k, gen):
    """k distinct experts per token in ascending order."""
    return torch.rand(T, E, generator=gen, device="cuda").topk(k, dim=1).indices.sort(dim=1).values


def _int8(x, amax):
    """x in 8 bits for rows (or blocks) of largest magnitude amax: the product is rounded once, hence in 64 bits."""
    inv = torch.where(amax < 2.0 ** -118, torch.zeros_like(amax), 127.0 / amax)
    return torch.round(x.double() * inv.double()).float()


def _fp(f):
    return -(-f // BLOCK) * BLOCK


def _blocks(pre, f):
    """[E, C, 2f] as [E, C, 2, fp / 32, 32] with zeros behind the columns."""
    E, C, _ = pre.shape
    p = torch.nn.functional.pad(pre.view(E, C, 2, f), (0, _fp(f) - f))
    return p.view(E, C, 2, _fp(f) // BLOCK, BLOCK)


def _keep(pre, f):
    """Integers [E, C, 2, fp] (held in 32 bits) and scales [E, C, 2, fp / 32] of [g | u]."""
    b = _blocks(pre, f)
    amax = b.abs().amax(dim=4)
    return _int8(b, amax[..., None]).flatten(3), torch.where(amax < 2.0 ** -118, torch.zeros_like(amax), amax / 127.0)


def _keep_bytes(E, C, f):
    ints = -(-E * C * 2 * _fp(f) // 256) * 256
    return ints, ints + E * 2 * (_fp(f) // BLOCK) * C * 4


def _kept(s):
    """g and u that a buffer of kept activations stands for."""
    c, C, E, f = s["c"], s["C"], s["c"]["E"], s["c"]["f"]
    at, end = _keep_bytes(E, C, f)
    q = s["keep"][:E * C * 2 * _fp(f)].view(torch.int8).view(E, C, 2, _fp(f) // BLOCK, BLOCK)
    scale = s["keep"][at:end].view(F32).view(E, 2, _fp(f) // BLOCK, C).permute(0, 3, 1, 2)
    v = (q.float() * scale[..., None]).flatten(3)[..., :f]
    return v[:, :, 0], v[:, :, 1]


def prepare(case, seed):
    c = dict(case)
    E, T, d, k, op = c["E"], c["T"], c["d"], c["k"], c["op"]
    C = _capacity(c)
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    cpu = torch.Generator().manual_seed(int(seed))

    def normal(*shape, scale=1.0, dtype=BF16):
        x = torch.empty(shape, device="cuda", dtype=dtype).normal_(generator=gen)
        return x.mul_(scale) if scale != 1.0 else x

    new = lambda *shape, dtype=BF16: torch.empty(shape, device="cuda", dtype=dtype)  # noqa: E731
    s = {"c": c, "C": C}
    if op in ("topk", "topk_bwd"):
        s["logits"] = normal(T, E, scale=1.5, dtype=F32)
        s["bias"] = normal(E, scale=0.05, dtype=F32) if c["bias"] else None
        if op == "topk":
            s["out"] = (new(T, E, dtype=F32) if c["scores"] else None, new(T, k, dtype=torch.int32), new(T, k, dtype=F32))
        else:
            s["idx"] = _choices(T, E, k, gen).to(torch.int32)
            s["dw"] = normal(T, k, dtype=F32)
            s["col"] = torch.rand(E, generator=gen, device="cuda") * 0.1 if c["aux"] else None
            s["out"] = new(T, E, dtype=F32)
    elif op == "block8":
        f = c["f"]
        idx = _choices(T, E, k, gen)
        held = torch.zeros(T, E, dtype=torch.int32, device="cuda").scatter_(1, idx, 1)
        slot = (held.cumsum(0, dtype=torch.int32) - 1).gather(1, idx)
        s["load"] = held.sum(0, dtype=torch.int32)
        tok = torch.full((E, C), -1, dtype=torch.int32, device="cuda")
        t, j = (slot < C).nonzero(as_tuple=True)
        tok[idx[t, j], slot[t, j].long()] = t.to(torch.int32)
        s["idx"], s["slot"], s["tok"] = idx.to(torch.int32), slot, tok
        s["x"] = normal(T, d)
        s["w_up"], s["w_up_scale"] = _weight8(gen, E, 2 * f, d)
        s["w_down"], s["w_down_scale"] = _weight8(gen, E, d, f)
        s["out"] = new(E, C, d)
        if own:
            i8 = torch.int8
            s["buf"] = (new(E, C, d, dtype=i8), new(E, C, dtype=F32), new(E, C, f), new(E, C, f, dtype=i8), new(E, C, dtype=F32))
    else:
        f = c["f"]
        load = _loads(c, C, cpu).to(device="cuda", dtype=torch.int32)
        used = (torch.arange(C, device="cuda")[None, :] < load[:, None])[:, :, None]
        s["load"] = load
        rows = lambda w: normal(E, C, w).mul_(used)  # noqa: E731   rows behind the load are zero, as dispatch leaves them
        if op in ("glu8", "gemm8"):
            K, N = (d, 2 * f) if op == "glu8" else (f, d)
            x = rows(K)
            amax = x.abs().amax(dim=2).float()
            s["xq"], s["xs"] = _int8(x, amax[..., None]).to(torch.int8), amax / 127.0
            s["w"], s["ws"] = _weight8(gen, E, N, K)
            s["out"] = new(E, C, f if op == "glu8" else d)
        else:
            if op == "keep8":
                s["x"] = rows(d)
                s["w_up"] = normal(*((E, d, 2 * f) if c["layout"] == 0 else (E, 2 * f, d)), scale=d ** -0.5)
                s["h"] = new(E, C, f)
            s["dy"] = rows(d)
            s["w_down"] = normal(*((E, f, d) if c["layout"] == 0 else (E, d, f)), scale=f ** -0.5)
            s["out"] = (new(E, C, 2 * f), new(E, C, f))
            at, end = _keep_bytes(E, C, f)
            s["keep"] = torch.zeros(end, dtype=torch.uint8, device="cuda")
            if op == "keep8_bwd":
                q, scale = _keep(rows(2 * f).float(), f)
                s["keep"][:q.numel()] = q.to(torch.int8).view(torch.uint8).flatten()
                s["keep"][at:] = scale.permute(0, 2, 3, 1).contiguous().view(torch.uint8).flatten()
    if own:
        from paper_2508_12801_b200 import binding as ms
        s["ms"] = ms
        s["ctx"] = ms.create(ms.make_params(T, d, E, k, capacity=C, io_dtype=ms.BF16))
        if op in ("topk", "topk_bwd"):
            s["how"] = ms.make_topk(score=ms.SOFTMAX if c["score"] == "softmax" else ms.SIGMOID, n_group=c["groups"],
                                    topk_group=c["keep_groups"], group_pairs=c["pairs"], renorm=c["renorm"], scale=c["scale"])
    return s


def _weight8(gen, E, N, K):
    """Weights [E, N, K] in 8 bits with a scale per column of the product, as a serving program keeps them."""
    w = torch.empty(E, N, K, device="cuda", dtype=BF16).normal_(generator=gen).mul_(K ** -0.5)
    amax = w.abs().amax(dim=2).float()
    return _int8(w, amax[..., None]).to(torch.int8), amax / 127.0


def _run_own(s):
    c, ms, ctx, out, op = s["c"], s["ms"], s["ctx"], s["out"], s["c"]["op"]
    if op == "topk":
        ms.topk_fwd(ctx, s["logits"], s["bias"], s["how"], *out)
    elif op == "topk_bwd":
        ms.topk_bwd(ctx, s["logits"], s["idx"], s["dw"], s["col"], s["how"], out)
    elif op == "glu8":
        ms.expert_glu_q8(ctx, s["xq"], s["xs"], s["w"], s["ws"], s["load"], out, c["d"], c["f"])
    elif op == "gemm8":
        ms.expert_gemm_q8(ctx, s["xq"], s["xs"], s["w"], s["ws"], s["load"], out, c["f"], c["d"])
    elif op == "block8":
        xq, xs, h, hq, hs = s["buf"]
        ms.dispatch_q8(ctx, s["x"], s["idx"], s["slot"], s["tok"], xq, xs)
        ms.expert_glu_q8(ctx, xq, xs, s["w_up"], s["w_up_scale"], s["load"], h, c["d"], c["f"])
        ms.expert_quant(ctx, h, s["load"], hq, hs, c["f"])
        ms.expert_gemm_q8(ctx, hq, hs, s["w_down"], s["w_down_scale"], s["load"], out, c["f"], c["d"])
    else:
        if op == "keep8":
            ms.expert_glu_keep8(ctx, s["x"], s["w_up"], s["load"], s["keep"], s["h"], c["d"], c["f"], c["layout"])
            out = (s["h"],) + out
        ms.expert_glu_bwd_keep8(ctx, s["dy"], s["w_down"], s["keep"], s["load"], *out[-2:], c["d"], c["f"], c["layout"])
    return out


def run(s):
    if own:
        return _run_own(s)
    c, C, op = s["c"], s["C"], s["c"]["op"]
    if op == "topk":
        return _plain_topk(s)
    if op == "topk_bwd":
        return _plain_topk_bwd(s)
    used = (torch.arange(C, device="cuda")[None, :] < s["load"][:, None])[:, :, None]
    f = c["f"]
    if op in ("glu8", "gemm8"):
        y = _product8(s["xq"].float(), s["xs"], s["w"], s["ws"]) * used
        return (_silu(y[..., :f]) * y[..., f:] if op == "glu8" else y).to(BF16)
    if op == "block8":
        x = s["x"].float()
        amax = x.abs().amax(dim=1)
        tok, there = s["tok"].long().clamp(min=0), s["tok"] >= 0
        xq, xs = _int8(x, amax[:, None])[tok] * there[:, :, None], (amax / 127.0)[tok] * there
        y = _product8(xq, xs, s["w_up"], s["w_up_scale"]) * used
        h = (_silu(y[..., :f]) * y[..., f:]).to(BF16).float()
        amax = h.abs().amax(dim=2)
        return (_product8(_int8(h, amax[..., None]), amax / 127.0, s["w_down"], s["w_down_scale"]) * used).to(BF16)
    out = ()
    if op == "keep8":
        w = s["w_up"].float()
        pre = torch.bmm(s["x"].float(), w if c["layout"] == 0 else w.transpose(1, 2)) * used
        g, u = pre[..., :f], pre[..., f:]
        out = ((_silu(g) * u).to(BF16),)
        q, scale = _keep(pre, f)
        g, u = (q.view(*scale.shape, BLOCK) * scale[..., None]).flatten(3)[..., :f].unbind(2)
    else:
        g, u = _kept(s)
    w = s["w_down"].float()
    dh = torch.bmm(s["dy"].float(), w.transpose(1, 2) if c["layout"] == 0 else w) * used
    sig = 1.0 / (1.0 + torch.exp(-g))
    dpre = torch.cat([dh * u * sig * (1.0 + g * (1.0 - sig)), dh * g * sig], dim=2)
    return out + (dpre.to(BF16), (g * sig * u * used).to(BF16))


def _silu(g):
    return g / (1.0 + torch.exp(-g))


def _product8(x, x_scale, w, w_scale):
    return torch.bmm(x, w.float().transpose(1, 2)) * (x_scale[:, :, None] * w_scale[:, None, :])


def _scores(l, c):
    if c["score"] == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-l))
    e = torch.exp(l - l.amax(dim=1, keepdim=True))
    return e / e.sum(dim=1, keepdim=True)


def _plain_topk(s):
    c, T, E, G = s["c"], s["c"]["T"], s["c"]["E"], s["c"]["groups"]
    l = s["logits"].double()                     # which of two near values is larger needs 64 bits
    v = _scores(l, c)
    choice = v if s["bias"] is None else v + s["bias"].double()
    if G > 1:
        best = choice.view(T, G, E // G).sort(dim=2, descending=True).values
        value = best[:, :, :2].sum(dim=2) if c["pairs"] else best[:, :, 0]
        place = value.argsort(dim=1, descending=True, stable=True).argsort(dim=1)
        choice = torch.where((place < c["keep_groups"]).repeat_interleave(E // G, dim=1), choice, -math.inf)
    idx = choice.argsort(dim=1, descending=True, stable=True)[:, :c["k"]].sort(dim=1).values
    v = v.float()
    w = v.gather(1, idx)
    if c["renorm"]:
        w = w / (w.sum(dim=1, keepdim=True) + 1e-20)
    return (v if c["scores"] else None, idx.to(torch.int32), w * c["scale"])


def _plain_topk_bwd(s):
    c, idx = s["c"], s["idx"].long()
    v = _scores(s["logits"], c)
    ds = c["scale"] * s["dw"]
    if c["renorm"]:
        p = v.gather(1, idx)
        total = p.sum(dim=1, keepdim=True) + 1e-20
        ds = (ds - (ds * p).sum(dim=1, keepdim=True) / total) / total
    g = torch.zeros_like(v).scatter_(1, idx, ds)
    if s["col"] is not None:
        g = g + s["col"]
    if c["score"] == "sigmoid":
        return g * v * (1.0 - v)
    return v * (g - (g * v).sum(dim=1, keepdim=True))


def work(case):
    c = case
    T, E, k, op = c["T"], c["E"], c["k"], c["op"]
    if op == "topk":
        return {"bytes": T * (4 * E + 8 * k + 4 * E * c["scores"]), "flops": T * E * 10}
    if op == "topk_bwd":
        return {"bytes": T * (8 * E + 8 * k), "flops": T * E * 10}
    d, f, R, Ea = c["d"], c["f"], T * k, min(c["E"], T * k)
    if op == "glu8":
        return {"bytes": R * (d + 2 * f) + 2 * Ea * f * d + 4 * (R + 2 * Ea * f), "flops": 4 * R * d * f}
    if op == "gemm8":
        return {"bytes": R * (f + 2 * d) + Ea * f * d + 4 * (R + Ea * d), "flops": 2 * R * d * f}
    if op == "block8":
        return {"bytes": 2 * T * d + 2 * R * d + 3 * Ea * f * d + 4 * Ea * (2 * f + d) + 8 * R, "flops": 6 * R * d * f}
    kept = R * 2 * _fp(f) * 36 // 32
    bwd = {"bytes": 2 * R * d + 2 * Ea * d * f + kept + 2 * R * 3 * f, "flops": 2 * R * d * f}
    if op == "keep8_bwd":
        return bwd
    return {"bytes": bwd["bytes"] + 2 * R * d + 4 * Ea * d * f + kept + 2 * R * f, "flops": 6 * R * d * f}


def exact(case, seed):
    """From the definitions, in 64 bits: token rows at once, expert rows expert by expert."""
    c = case
    s = prepare(case, seed)
    T, E, k, op, C = c["T"], c["E"], c["k"], c["op"], s["C"]
    if op in ("topk", "topk_bwd"):
        l = s["logits"].to(F64)
        v = torch.sigmoid(l) if c["score"] == "sigmoid" else torch.softmax(l, dim=1)
        if op == "topk":
            by = v.clone() if s["bias"] is None else v + s["bias"].to(F64)
            size = E // c["groups"]
            value = torch.stack([by[:, i:i + size].topk(min(2, size) if c["pairs"] else 1, dim=1).values.sum(1)
                                 for i in range(0, E, size)], dim=1)
            for _ in range(c["groups"] - c["keep_groups"]):        # the worst group leaves, the last one of equals
                worst = c["groups"] - 1 - value.flip(1).argmin(dim=1)
                value[torch.arange(T, device="cuda"), worst] = math.inf
                by[(torch.arange(E, device="cuda") // size)[None, :] == worst[:, None]] = -math.inf
            chosen = torch.zeros(T, E, dtype=torch.bool, device="cuda")
            for _ in range(k):                                     # argmax gives the first of equals
                at = by.argmax(dim=1, keepdim=True)
                chosen.scatter_(1, at, True)
                by.scatter_(1, at, -math.inf)
            idx = chosen.nonzero()[:, 1].view(T, k)
            w = v[chosen].view(T, k)
            w = c["scale"] * (w / (w.sum(1, keepdim=True) + 1e-20) if c["renorm"] else w)
            return (v if c["scores"] else None, idx.to(torch.int32), w)
        idx = s["idx"].long()
        v = v.requires_grad_(True)                                 # the formula's own derivative
        p = v.gather(1, idx)
        w = c["scale"] * (p / (p.sum(1, keepdim=True) + 1e-20) if c["renorm"] else p)
        loss = (w * s["dw"].to(F64)).sum() + (0.0 if s["col"] is None else (v * s["col"].to(F64)).sum())
        g, = torch.autograd.grad(loss, v)
        v = v.detach()
        return g * (v - v * v) if c["score"] == "sigmoid" else g * v - v * (g * v).sum(1, keepdim=True)

    if work(c)["flops"] > 4e13:
        return None
    f, load = c["f"], s["load"].clamp(max=C).tolist()
    silu = lambda g: g * torch.sigmoid(g)  # noqa: E731

    def steps(x, n):        # rows of n columns in 8 bits: values they stand for, from the definition
        x = x.unflatten(1, (-1, n))
        amax = x.abs().amax(dim=2, keepdim=True).to(F32)
        scale = (amax.to(F64) / 127).to(F32).to(F64)
        inv = (127 / amax.to(F64)).to(F32).to(F64)
        return torch.where(amax > 0, torch.round(x * inv) * scale, torch.zeros_like(x)).flatten(1)

    def value(q, scale):
        return q.to(F64) * scale.to(F64)[:, None]

    def per_expert(fn, *widths):
        out = [torch.zeros(E, C, w, dtype=F64, device="cuda") for w in widths]
        for e in range(E):
            if load[e]:
                for o, r in zip(out, fn(e, load[e])):
                    o[e, :load[e]] = r
        return out

    if op == "gemm8":
        return per_expert(lambda e, n: (value(s["xq"][e, :n], s["xs"][e, :n]) @ value(s["w"][e], s["ws"][e]).T,), c["d"])[0]
    if op == "glu8":
        def fn(e, n):
            y = value(s["xq"][e, :n], s["xs"][e, :n]) @ value(s["w"][e], s["ws"][e]).T
            return (silu(y[:, :f]) * y[:, f:],)
        return per_expert(fn, f)[0]
    if op == "block8":
        x = steps(s["x"].to(F64), c["d"])

        def fn(e, n):
            y = x[s["tok"][e, :n].long()] @ value(s["w_up"][e], s["w_up_scale"][e]).T
            h = (silu(y[:, :f]) * y[:, f:]).to(BF16).to(F64)       # what the second product takes is a bf16 row
            return (steps(h, f) @ value(s["w_down"][e], s["w_down_scale"][e]).T,)
        return per_expert(fn, c["d"])[0]

    if op == "keep8_bwd":
        kept = [t.to(F64) for t in _kept(s)]

    def fn(e, n):
        out = ()
        if op == "keep8":
            w = s["w_up"][e].to(F64)
            pre = s["x"][e, :n].to(F64) @ (w if c["layout"] == 0 else w.T)
            out = (silu(pre[:, :f]) * pre[:, f:],)
            pad = torch.zeros(n, _fp(f) - f, dtype=F64, device="cuda")
            g, u = (steps(torch.cat([t, pad], 1), BLOCK)[:, :f] for t in (pre[:, :f], pre[:, f:]))
        else:
            g, u = kept[0][e, :n], kept[1][e, :n]
        w = s["w_down"][e].to(F64)
        dh = s["dy"][e, :n].to(F64) @ (w.T if c["layout"] == 0 else w)
        sg = torch.sigmoid(g)
        return out + (torch.cat([dh * u * (sg + g * sg * (1 - sg)), dh * g * sg], 1), silu(g) * u)

    widths = ((f,) if op == "keep8" else ()) + (2 * f, f)
    return tuple(per_expert(fn, *widths))
