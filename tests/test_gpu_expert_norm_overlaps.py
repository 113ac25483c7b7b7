"""Outputs that share memory with another argument are refused by every expert and norm call before anything runs, whole buffers and
parts of them alike; the two pairs that may be one buffer are not."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INVALID = 1
E, C, T, D, F, K = 4, 8, 16, 64, 32, 2


@pytest.fixture(scope="module")
def ms():
    from paper_2508_12801_b200 import binding
    assert torch.cuda.is_available()
    return binding


class Arena:
    """Buffers of one allocation, 256-byte aligned, filled with a pattern, with room for the largest on either side."""

    def __init__(self, sizes):
        room = -(-max(sizes.values()) // 256) * 256
        self.at, n = {}, room
        for name, b in sizes.items():
            self.at[name] = (n, b)
            n += -(-b // 256) * 256
        self.mem = torch.full((n + room + 256,), 3, dtype=torch.uint8, device=DEV)
        self.base = (self.mem.data_ptr() + 255) // 256 * 256
        self.before = self.mem.clone()

    def ptr(self, name):
        return self.base + self.at[name][0]

    def size(self, name):
        return self.at[name][1]

    def untouched(self):
        torch.cuda.synchronize()
        return torch.equal(self.mem, self.before)


def refuse_overlaps(arena, call, outs, args, allowed=()):
    """Every output in the place of every other argument: at its start, one 16-byte step into it, and ending one step into it."""
    for o in outs:
        for a in args:
            if a == o:
                continue
            spots = [arena.ptr(a) + 16, arena.ptr(a) - arena.size(o) + 16] + ([] if (o, a) in allowed else [arena.ptr(a)])
            for at in spots:
                p = {n: arena.ptr(n) for n in args}
                p[o] = at
                if at == arena.ptr(a) + 16 and arena.size(a) <= 16:
                    continue
                assert call(p) == INVALID, (o, a, at - arena.ptr(a))
    assert arena.untouched()


@pytest.mark.parametrize("dtype,eb", [("bf16", 2), ("f32", 4)])
def test_expert_calls(ms, dtype, eb):
    ctx = ms.create(ms.make_params(C, D, E, 1, capacity=C, io_dtype=ms.BF16 if dtype == "bf16" else ms.F32), DEV)
    lib, h = ms._lib, ctx.handle
    a = Arena(dict(x=E * C * D * eb, w=E * D * F * eb, load=16, y=E * C * F * eb))
    refuse_overlaps(a, lambda p: lib.maxscore_expert_gemm(h, p["x"], p["w"], p["load"], p["y"], D, F, 0, 0), ["y"], ["x", "w", "load", "y"])
    a = Arena(dict(x=E * C * D * eb, dy=E * C * F * eb, load=16, dw=E * D * F * 4))
    refuse_overlaps(a, lambda p: lib.maxscore_expert_gemm_dw(h, p["x"], p["dy"], p["load"], p["dw"], D, F, 0, 1, 0), ["dw"], ["x", "dy", "load", "dw"])
    a = Arena(dict(x=E * C * D * eb, w=E * D * 2 * F * eb, load=16, pre=E * C * 2 * F * eb, h=E * C * F * eb))
    refuse_overlaps(a, lambda p: lib.maxscore_expert_glu(h, p["x"], p["w"], p["load"], p["pre"], p["h"], D, F, 0, 0), ["pre", "h"],
                    ["x", "w", "load", "pre", "h"])
    a = Arena(dict(dy=E * C * D * eb, w=E * D * F * eb, pre=E * C * 2 * F * eb, load=16, dpre=E * C * 2 * F * eb))
    refuse_overlaps(a, lambda p: lib.maxscore_expert_glu_bwd(h, p["dy"], p["w"], p["pre"], p["load"], p["dpre"], D, F, 0, 0), ["dpre"],
                    ["dy", "w", "pre", "load", "dpre"])


@pytest.mark.parametrize("dtype,eb", [("bf16", 2), ("f32", 4)])
def test_norm_calls(ms, dtype, eb):
    ctx = ms.create(ms.make_params(T, D, E, K, capacity=T, io_dtype=ms.BF16 if dtype == "bf16" else ms.F32), DEV)
    lib, h = ms._lib, ctx.handle
    row, pairs, weights = T * D * eb, T * K * 4, dict(w_post=D * eb, gate=4 * D * eb, w_pre=D * eb)
    names = list(weights)

    def norm(p):
        return ms.C.byref(ms.Norm(p["w_post"], p["gate"], p["w_pre"], 4, 1e-5, 0.0, 1.0))
    a = Arena(dict(src=E * T * D * eb, idx=pairs, slot=pairs, gw=pairs, res=row, y=row, r=row, h=row, **weights))
    refuse_overlaps(a, lambda p: lib.maxscore_combine_norm(h, p["src"], p["idx"], p["slot"], p["gw"], p["res"], norm(p), p["y"], p["r"], p["h"], 0),
                    ["y", "r", "h"], ["src", "idx", "slot", "gw", "res", "y", "r", "h"] + names, allowed=[("r", "res")])
    a = Arena(dict(y=row, res=row, r=row, h=row, **weights))
    refuse_overlaps(a, lambda p: lib.maxscore_block_norm(h, p["y"], p["res"], norm(p), p["r"], p["h"], 0), ["r", "h"],
                    ["y", "res", "r", "h"] + names, allowed=[("r", "res")])
    a = Arena(dict(dro=row, dh=row, y=row, r=row, dy=row, dr=row, dw_post=D * 4, dgate=4 * D * 4, dw_pre=D * 4, **weights))
    refuse_overlaps(a, lambda p: lib.maxscore_block_norm_bwd(h, p["dro"], p["dh"], p["y"], p["r"], norm(p), p["dy"], p["dr"], p["dw_post"], p["dgate"],
                                                              p["dw_pre"], 0),
                    ["dy", "dr", "dw_post", "dgate", "dw_pre"], ["dro", "dh", "y", "r", "dy", "dr", "dw_post", "dgate", "dw_pre"] + names,
                    allowed=[("dr", "dro")])


def test_neighbours_in_one_allocation_are_taken(ms):
    """Buffers that touch without sharing a byte, and inputs that share one, are fine."""
    ctx = ms.create(ms.make_params(T, D, E, K, capacity=T, io_dtype=ms.F32), DEV)
    flat = torch.randn(5, T, D, device=DEV)
    w = torch.ones(D, device=DEV)
    n = ms.make_norm(w_post=w, w_pre=w)                                # one weight for both norms
    ms.block_norm(ctx, flat[1], flat[1], n, flat[0], flat[2])          # y and the residual are one buffer, outputs on either side
    want = [torch.empty(T, D, device=DEV) for _ in range(2)]
    ms.block_norm(ctx, flat[1].clone(), flat[1].clone(), n, *want)
    assert torch.equal(flat[0], want[0]) and torch.equal(flat[2], want[1])
    dw = torch.empty(2, D, device=DEV)
    ms.block_norm_bwd(ctx, flat[0], flat[0], flat[1], flat[2], n, flat[3], flat[4], dw[0], None, dw[1])
    assert torch.isfinite(flat).all() and torch.isfinite(dw).all()
