"""Measured cases of the expert products and of the norms around a MoE block.

Operators (`op` of a case):
  glu       h = silu(x W_g) * (x W_u) per expert on dispatched rows, optionally keeping [g | u] for training
  gemm      y = x W per expert on dispatched rows (the second product of an expert; with the layout
            flipped, the gradient with respect to the rows)
  glu_bwd   gradient of the gated activation through the second product: dh = dy W_down^T, then [dg | du]
  dw        gradient of an expert's weight: x^T dy over the rows the expert holds
  norm      after-norm, gate, scaled residual and before-norm, on combined rows or straight from the expert buffers
  norm_bwd  its gradients

Buffers are [E, C, width] with `load[e]` rows in use; what lies behind them is zero on output.
"""
import math

import torch

own = False

EPS = 1e-5
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _case(op, T, d, E, k, cf, dtype, **kw):
    c = dict(op=op, T=T, d=d, E=E, k=k, cf=cf, dtype=dtype)
    c.update(kw)
    return c


def listed():
    def named(name, **c):
        return dict(_case(**c), name=name)
    return [
        # one token of a serving loop: eight experts with a row each, bound by the weights
        named("glu one token", op="glu", T=1, d=2048, E=64, k=8, cf=1.0, dtype="bf16", f=1024, layout=1, keep=False),
        # the largest batch of the router's own workloads, training forward
        named("glu stress", op="glu", T=65536, d=4096, E=128, k=8, cf=1.0, dtype="bf16", f=1024, layout=0, keep=True),
        # a serving batch of 64 sequences on sixteen experts, second product
        named("gemm batch 64", op="gemm", T=64, d=1024, E=16, k=2, cf=1.25, dtype="bf16", d_in=512, d_out=1024, layout=1),
        # the skewed workload: ragged loads below the capacity; gradient with respect to the rows of the first product
        named("gemm skew dx", op="gemm", T=16384, d=2048, E=64, k=8, cf=1.25, dtype="bf16", d_in=2048, d_out=2048, layout=1),
        # the tiny router in fp32
        named("glu_bwd tiny f32", op="glu_bwd", T=512, d=256, E=8, k=2, cf=1.0, dtype="f32", f=512, layout=0),
        # training step with an inner width that is no multiple of a tile
        named("glu_bwd k8e64", op="glu_bwd", T=8192, d=2048, E=64, k=8, cf=1.0, dtype="bf16", f=1000, layout=0),
        # weight gradients: few large experts, and the skewed workload's ragged loads
        named("dw k2e16", op="dw", T=4096, d=1024, E=16, k=2, cf=1.0, dtype="bf16", d_in=512, d_out=1024, layout=0),
        named("dw skew", op="dw", T=16384, d=2048, E=64, k=8, cf=1.25, dtype="bf16", d_in=2048, d_out=2048, layout=1),
        # sixteen tokens of a serving loop, straight from the expert buffers
        named("norm batch 16", op="norm", T=16, d=2048, E=64, k=8, cf=1.5, dtype="bf16", fused=True, gates=0, post=True),
        # the largest batch, straight from the expert buffers, with a learned gate per channel
        named("norm stress", op="norm", T=65536, d=4096, E=128, k=8, cf=1.25, dtype="bf16", fused=True, gates=1, post=True),
        # an odd batch of eight sequences with a gate of its own each, fp32
        named("norm_bwd odd f32", op="norm_bwd", T=777, d=1000, E=8, k=2, cf=1.0, dtype="f32", gates=8, post=True),
        # the largest batch, training backward
        named("norm_bwd stress", op="norm_bwd", T=65536, d=4096, E=128, k=8, cf=1.0, dtype="bf16", gates=1, post=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["glu", "gemm", "glu_bwd", "dw", "norm", "norm_bwd"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    E, k = rng.choice([(8, 2), (12, 3), (16, 2), (33, 5), (64, 8), (128, 8)])
    cf = rng.choice([1.0, 1.1, 1.25, 1.5])
    if op in ("norm", "norm_bwd"):
        T, d = _log(rng, 1, 40000), 8 * _log(rng, 16, 512)
        c = _case(op, T, d, E, k, cf, dtype, gates=min(T, rng.choice([0, 1, 1, 3, 16])), post=rng.random() < 0.75)
        if op == "norm":
            c["fused"] = rng.random() < 0.6
        return c
    # the rows are spread over serving and training batches; fp32 runs on the plain FMA units and stays smaller
    T = _log(rng, 1, 20000 if dtype == "bf16" else 2500)
    d, f = 8 * _log(rng, 16, 320), 8 * _log(rng, 8, 192)
    c = _case(op, T, d, E, k, cf, dtype, layout=rng.randrange(2))
    if op == "glu":
        c.update(f=f, keep=rng.random() < 0.5)
    elif op == "glu_bwd":
        c.update(f=f)
    elif rng.random() < 0.5:
        c.update(d_in=f, d_out=d)
    else:
        c.update(d_in=d, d_out=f)
    return c


def _capacity(c):
    return max(1, math.ceil(c["cf"] * c["T"] * c["k"] / c["E"] - 1e-9))


def _loads(c, C, gen):
    """Rows per expert: popularity like a Zipf law cut off at the capacity, T * k rows in all."""
    E, total = c["E"], c["T"] * c["k"]
    share = (torch.randperm(E, generator=gen).double() + 1.0) ** -1.1
    load, left = torch.zeros(E, dtype=torch.int64), total
    while left > 0:
        room = C - load
        s = torch.where(room > 0, share, torch.zeros(E, dtype=torch.float64))
        add = torch.minimum(torch.floor(s / s.sum() * left).long(), room)
        if int(add.sum()) == 0:       # the last few rows, one each to the experts most asked for
            order = torch.argsort(s, descending=True, stable=True)
            order = order[room[order] > 0][:left]
            add = torch.zeros(E, dtype=torch.int64)
            add[order] = 1
        load, left = load + add, left - int(add.sum())
    return load


def _assignment(c, C, gen):
    """k distinct experts per token in ascending order, the slots in token order; pairs beyond the capacity stay empty."""
    T, E, k = c["T"], c["E"], c["k"]
    idx = torch.rand(T, E, generator=gen, device="cuda").topk(k, dim=1).indices.sort(dim=1).values
    held = torch.zeros(T, E, dtype=torch.int32, device="cuda").scatter_(1, idx, 1)
    slot = (held.cumsum(0, dtype=torch.int32) - 1).gather(1, idx)
    idx = torch.where(slot < C, idx, torch.full_like(idx, -1))
    return idx.to(torch.int32), torch.where(slot < C, slot, torch.full_like(slot, -1)).to(torch.int32)


def _rows_per_gate(c):
    return -(-c["T"] // c["gates"]) if c["gates"] else 0


def prepare(case, seed):
    c = dict(case)
    C, dt = _capacity(c), DTYPES[c["dtype"]]
    E, T, d = c["E"], c["T"], c["d"]
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    cpu = torch.Generator().manual_seed(int(seed))

    def normal(*shape, scale=1.0):
        x = torch.empty(shape, device="cuda", dtype=dt).normal_(generator=gen)
        return x.mul_(scale) if scale != 1.0 else x

    s = {"c": c, "C": C}
    if c["op"] in ("norm", "norm_bwd"):
        rpg = _rows_per_gate(c)
        n_gates = -(-T // rpg) if rpg else 0
        s["res_scale"], s["rpg"] = 0.75, rpg
        s["w_post"] = 1.0 + normal(d, scale=0.1) if c["post"] else None
        s["w_pre"] = 1.0 + normal(d, scale=0.1)
        s["gate"] = normal(n_gates, d, scale=0.5) if rpg else None
        if c["op"] == "norm":
            s["res"] = normal(T, d)
            if c["fused"]:
                s["idx"], s["slot"] = _assignment(c, C, gen)
                s["gate_w"] = torch.rand(T, c["k"], generator=gen, device="cuda")
                s["src"] = normal(E, C, d)
            else:
                s["y"] = normal(T, d)
        else:
            s["y"], s["r_out"], s["dr_out"], s["dh"] = normal(T, d), normal(T, d), normal(T, d), normal(T, d)
        new = lambda *shape, dtype=dt: torch.empty(shape, device="cuda", dtype=dtype)  # noqa: E731
        if c["op"] == "norm":
            s["out"] = (new(T, d), new(T, d), new(T, d))
        else:
            f32 = torch.float32
            s["out"] = (new(T, d), new(T, d), new(d, dtype=f32) if c["post"] else None,
                        new(n_gates, d, dtype=f32) if rpg else None, new(d, dtype=f32))
    else:
        load = _loads(c, C, cpu).to(device="cuda", dtype=torch.int32)
        used = (torch.arange(C, device="cuda")[None, :] < load[:, None])[:, :, None]
        s["load"] = load
        rows = lambda w: normal(E, C, w).mul_(used)  # noqa: E731   rows behind the load are zero, as dispatch leaves them
        new = lambda w: torch.empty(E, C, w, device="cuda", dtype=dt)  # noqa: E731
        if c["op"] == "glu":
            s["x"] = rows(d)
            s["w"] = normal(*((E, d, 2 * c["f"]) if c["layout"] == 0 else (E, 2 * c["f"], d)), scale=d ** -0.5)
            s["out"] = (new(2 * c["f"]) if c["keep"] else None, new(c["f"]))
        elif c["op"] == "glu_bwd":
            s["dy"], s["pre"] = rows(d), rows(2 * c["f"])
            s["w"] = normal(*((E, c["f"], d) if c["layout"] == 0 else (E, d, c["f"])), scale=c["f"] ** -0.5)
            s["out"] = new(2 * c["f"])
        elif c["op"] == "gemm":
            s["x"] = rows(c["d_in"])
            s["w"] = normal(*((E, c["d_in"], c["d_out"]) if c["layout"] == 0 else (E, c["d_out"], c["d_in"])), scale=c["d_in"] ** -0.5)
            s["out"] = new(c["d_out"])
        else:
            s["x"], s["dy"] = rows(c["d_in"]), rows(c["d_out"])
            s["out"] = torch.empty((E, c["d_in"], c["d_out"]) if c["layout"] == 0 else (E, c["d_out"], c["d_in"]), device="cuda")
    if own:
        from paper_2508_12801_b200 import binding as ms
        s["ms"] = ms
        s["ctx"] = ms.create(ms.make_params(T, d, E, c["k"], capacity=C, io_dtype=ms.BF16 if c["dtype"] == "bf16" else ms.F32))
        if c["op"] in ("norm", "norm_bwd"):
            s["norm"] = ms.make_norm(w_post=s["w_post"], gate=s["gate"], w_pre=s["w_pre"], rows_per_gate=s["rpg"], eps=EPS,
                                     res_scale=s["res_scale"])
    return s


def _run_own(s):
    c, ms, ctx, out = s["c"], s["ms"], s["ctx"], s["out"]
    if c["op"] == "glu":
        ms.expert_glu(ctx, s["x"], s["w"], s["load"], out[0], out[1], c["d"], c["f"], c["layout"])
    elif c["op"] == "gemm":
        ms.expert_gemm(ctx, s["x"], s["w"], s["load"], out, c["d_in"], c["d_out"], c["layout"])
    elif c["op"] == "glu_bwd":
        ms.expert_glu_bwd(ctx, s["dy"], s["w"], s["pre"], s["load"], out, c["d"], c["f"], c["layout"])
    elif c["op"] == "dw":
        ms.expert_gemm_dw(ctx, s["x"], s["dy"], s["load"], out, c["d_in"], c["d_out"], c["layout"], 0)
    elif c["op"] == "norm":
        if c["fused"]:
            ms.combine_norm(ctx, s["src"], s["idx"], s["slot"], s["gate_w"], s["res"], s["norm"], *out)
        else:
            ms.block_norm(ctx, s["y"], s["res"], s["norm"], out[1], out[2])
            out = (None,) + out[1:]
    else:
        ms.block_norm_bwd(ctx, s["dr_out"], s["dh"], s["y"], s["r_out"], s["norm"], *out)
    return out


def run(s):
    if own:
        return _run_own(s)
    c, C = s["c"], s["C"]
    dt = DTYPES[c["dtype"]]
    if c["op"] == "norm":
        return _plain_norm(s, dt)
    if c["op"] == "norm_bwd":
        return _plain_norm_bwd(s, dt)
    used = (torch.arange(C, device="cuda")[None, :] < s["load"][:, None])[:, :, None]
    if c["op"] == "dw":
        x, dy = s["x"].float() * used, s["dy"].float() * used
        return torch.bmm(x.transpose(1, 2), dy) if c["layout"] == 0 else torch.bmm(dy.transpose(1, 2), x)
    w = s["w"].float()
    if c["op"] == "gemm":
        return (torch.bmm(s["x"].float(), w if c["layout"] == 0 else w.transpose(1, 2)) * used).to(dt)
    f = c["f"]
    if c["op"] == "glu":
        pre = torch.bmm(s["x"].float(), w if c["layout"] == 0 else w.transpose(1, 2)) * used
        g, u = pre[..., :f], pre[..., f:]
        h = (g / (1.0 + torch.exp(-g)) * u).to(dt)
        return (pre.to(dt) if c["keep"] else None, h)
    dh = torch.bmm(s["dy"].float(), w.transpose(1, 2) if c["layout"] == 0 else w) * used
    g, u = s["pre"][..., :f].float(), s["pre"][..., f:].float()
    sig = 1.0 / (1.0 + torch.exp(-g))
    return torch.cat([dh * u * sig * (1.0 + g * (1.0 - sig)), dh * g * sig], dim=2).to(dt)


def _gate_rows(s, T):
    if s["gate"] is None:
        return 1.0
    return s["gate"].float()[torch.arange(T, device="cuda") // s["rpg"]]


def _plain_norm(s, dt):
    c = s["c"]
    T, d = c["T"], c["d"]
    if c["fused"]:
        src = s["src"].reshape(-1, d)
        at = (s["idx"].long() * s["C"] + s["slot"].long()).clamp_(min=0)
        wgt = s["gate_w"] * (s["idx"] >= 0)
        y = torch.zeros(T, d, device="cuda")
        for j in range(c["k"]):
            y += wgt[:, j, None] * src[at[:, j]].float()
    else:
        y = s["y"].float()
    n = y
    if s["w_post"] is not None:
        n = y * torch.rsqrt(y.square().mean(dim=1, keepdim=True) + EPS) * s["w_post"].float()
    r = s["res_scale"] * s["res"].float() + _gate_rows(s, T) * n
    h = r * torch.rsqrt(r.square().mean(dim=1, keepdim=True) + EPS) * s["w_pre"].float()
    return (y.to(dt) if c["fused"] else None, r.to(dt), h.to(dt))


def _plain_norm_bwd(s, dt):
    c = s["c"]
    T = c["T"]
    dh, r, y = s["dh"].float(), s["r_out"].float(), s["y"].float()
    inv = torch.rsqrt(r.square().mean(dim=1, keepdim=True) + EPS)
    rn = r * inv
    dw_pre = (dh * rn).sum(dim=0)
    g = dh * s["w_pre"].float()
    dr = s["dr_out"].float() + inv * (g - rn * (g * rn).mean(dim=1, keepdim=True))
    dn = dr * _gate_rows(s, T)
    dw_post = None
    n, dy = y, dn
    if s["w_post"] is not None:
        inv = torch.rsqrt(y.square().mean(dim=1, keepdim=True) + EPS)
        yn = y * inv
        dw_post = (dn * yn).sum(dim=0)
        n = yn * s["w_post"].float()
        g = dn * s["w_post"].float()
        dy = inv * (g - yn * (g * yn).mean(dim=1, keepdim=True))
    dgate = None
    if s["gate"] is not None:
        G = s["gate"].shape[0]
        dgate = torch.nn.functional.pad(dr * n, (0, 0, 0, G * s["rpg"] - T)).view(G, s["rpg"], -1).sum(dim=1)
    return (dy.to(dt), (s["res_scale"] * dr).to(dt), dw_post, dgate, dw_pre)


def work(case):
    c = case
    T, E, k, d = c["T"], c["E"], c["k"], c["d"]
    b = 2 if c["dtype"] == "bf16" else 4
    R, Ea = T * k, min(c["E"], c["T"] * c["k"])
    if c["op"] == "glu":
        f = c["f"]
        return {"bytes": b * (R * d + Ea * d * 2 * f + R * f * (3 if c["keep"] else 1)), "flops": 4 * R * d * f}
    if c["op"] == "glu_bwd":
        f = c["f"]
        return {"bytes": b * (R * d + Ea * d * f + 4 * R * f), "flops": 2 * R * d * f}
    if c["op"] in ("gemm", "dw"):
        i, o = c["d_in"], c["d_out"]
        return {"bytes": b * R * (i + o) + (b * Ea if c["op"] == "gemm" else 4 * E) * i * o, "flops": 2 * R * i * o}
    if c["op"] == "norm":
        return {"bytes": b * T * d * ((k + 4) if c["fused"] else 4), "flops": T * d * (2 * k * c["fused"] + 9)}
    return {"bytes": 6 * b * T * d, "flops": 24 * T * d}


def exact(case, seed):
    """From the definition, in 64 bits, expert by expert and token block by token block."""
    c = case
    if c["op"] not in ("norm", "norm_bwd") and work(c)["flops"] > 4e13:
        return None
    s = prepare(case, seed)
    f64 = torch.float64
    C, E, T, d = s["C"], c["E"], c["T"], c["d"]
    if c["op"] in ("glu", "gemm", "glu_bwd", "dw"):
        load = s["load"].tolist()

        def per_expert(fn, *shape):
            out = torch.zeros(E, *shape, dtype=f64, device="cuda")
            for e in range(E):
                if load[e]:
                    fn(out[e], e, load[e])
            return out

        def weight(e, transpose):
            w = s["w"][e].to(f64)
            return w.T if transpose else w

        if c["op"] == "gemm":
            def fn(o, e, n):
                o[:n] = s["x"][e, :n].to(f64) @ weight(e, c["layout"] == 1)
            return per_expert(fn, C, c["d_out"])
        if c["op"] == "dw":
            def fn(o, e, n):
                g = torch.einsum("si,sj->ij", s["x"][e, :n].to(f64), s["dy"][e, :n].to(f64))
                o.copy_(g if c["layout"] == 0 else g.T)
            return per_expert(fn, *s["out"].shape[1:])
        f = c["f"]
        if c["op"] == "glu":
            def fn(o, e, n):
                o[:n, :2 * f] = s["x"][e, :n].to(f64) @ weight(e, c["layout"] == 1)
                o[:n, 2 * f:] = o[:n, :f] * torch.sigmoid(o[:n, :f]) * o[:n, f:2 * f]
            both = per_expert(fn, C, 3 * f)
            return (both[..., :2 * f] if c["keep"] else None, both[..., 2 * f:])

        def fn(o, e, n):
            dh = s["dy"][e, :n].to(f64) @ weight(e, c["layout"] == 0)
            g, u = s["pre"][e, :n, :f].to(f64), s["pre"][e, :n, f:].to(f64)
            sg = torch.sigmoid(g)
            o[:n, :f] = dh * u * (sg + g * sg * (1 - sg))
            o[:n, f:] = dh * g * sg
        return per_expert(fn, C, 2 * f)

    def unit(v):      # a row over its root mean square, and that
        rms = torch.linalg.vector_norm(v, dim=1, keepdim=True).square().div(d).add(EPS).sqrt()
        return v / rms, rms

    w_pre = s["w_pre"].to(f64)
    w_post = None if s["w_post"] is None else s["w_post"].to(f64)
    outs = None
    block = max(1, (1 << 25) // d)
    for i0 in range(0, T, block):
        i1 = min(T, i0 + block)
        t = torch.arange(i0, i1, device="cuda")
        gate = torch.ones(1, d, dtype=f64, device="cuda") if s["gate"] is None else s["gate"][torch.div(t, s["rpg"], rounding_mode="floor")].to(f64)
        if c["op"] == "norm":
            if c["fused"]:
                y = torch.zeros(i1 - i0, d, dtype=f64, device="cuda")
                for j in range(c["k"]):
                    ok = s["idx"][i0:i1, j] >= 0
                    e, sl = s["idx"][i0:i1, j][ok].long(), s["slot"][i0:i1, j][ok].long()
                    y[ok] += s["gate_w"][i0:i1, j][ok].to(f64)[:, None] * s["src"][e, sl].to(f64)
            else:
                y = s["y"][i0:i1].to(f64)
            n = y if w_post is None else unit(y)[0] * w_post
            r = s["res_scale"] * s["res"][i0:i1].to(f64) + gate * n
            part = (y if c["fused"] else None, r, unit(r)[0] * w_pre)
            if outs is None:
                outs = [None if p is None else torch.empty(T, d, dtype=f64, device="cuda") for p in part]
            for o, p in zip(outs, part):
                if o is not None:
                    o[i0:i1] = p
            continue
        if outs is None:
            outs = [torch.empty(T, d, dtype=f64, device="cuda"), torch.empty(T, d, dtype=f64, device="cuda"),
                    None if w_post is None else torch.zeros(d, dtype=f64, device="cuda"),
                    None if s["gate"] is None else torch.zeros(s["gate"].shape, dtype=f64, device="cuda"),
                    torch.zeros(d, dtype=f64, device="cuda")]
        dh = s["dh"][i0:i1].to(f64)
        ru, rms = unit(s["r_out"][i0:i1].to(f64))
        outs[4] += torch.einsum("td,td->d", dh, ru)
        v = dh * w_pre / rms
        dr = s["dr_out"][i0:i1].to(f64) + v - ru * (v * ru).sum(1, keepdim=True) / d
        y = s["y"][i0:i1].to(f64)
        dn = gate * dr
        if w_post is None:
            n, dy = y, dn
        else:
            yu, rms = unit(y)
            n = yu * w_post
            outs[2] += torch.einsum("td,td->d", dn, yu)
            v = dn * w_post / rms
            dy = v - yu * (v * yu).sum(1, keepdim=True) / d
        if s["gate"] is not None:
            outs[3].index_add_(0, torch.div(t, s["rpg"], rounding_mode="floor"), dr * n)
        outs[0][i0:i1], outs[1][i0:i1] = dy, s["res_scale"] * dr
    return tuple(outs)
