"""The workspace: its size, and that calls that share it do not read one another's scratch."""
import pytest
import torch

from paper_2508_12801_b200 import binding as ms


@pytest.mark.parametrize("T,d,E,k,io,router", [(65536, 4096, 128, 8, "bf16", 131102720), (16384, 2048, 64, 8, "bf16", 47525888),
                                               (8192, 2048, 64, 8, "bf16", 28116992), (65536, 4096, 128, 8, "f32", 76576768)])
def test_norm_partials_add_nothing_to_a_training_batch(T, d, E, k, io, router):
    """`router`: what the router's own calls need.  The norm backward's partial sums lie over their scratch."""
    p = ms.make_params(T, d, E, k, 1.0, io_dtype=ms.BF16 if io == "bf16" else ms.F32)
    assert ms.workspace_bytes(p) <= router


def test_norm_partials_of_wide_rows():
    """Three rows of partial sums for each CTA that a B200 runs, one an SM on wide rows."""
    p = ms.make_params(600, 8192, 128, 8, 1.0, io_dtype=ms.F32)
    assert ms.workspace_bytes(p) <= 3040256 + 3 * 148 * 8192 * 4


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,E,k,io", [(1, 512, 8, 2, "bf16"), (512, 256, 8, 2, "f32"), (4096, 1024, 16, 2, "bf16"), (3000, 2048, 33, 5, "f32")])
def test_norm_backward_between_the_router_calls(T, d, E, k, io):
    dev, dt = "cuda:0", torch.bfloat16 if io == "bf16" else torch.float32
    ctx = ms.create(ms.make_params(T, d, E, k, 1.0, io_dtype=ms.BF16 if io == "bf16" else ms.F32), dev)
    g = torch.Generator(device=dev).manual_seed(5)
    r = lambda *s: torch.empty(*s, device=dev, dtype=dt).normal_(generator=g)  # noqa: E731
    h, wg, dY, yexp, dro, dh, y, rows = r(T, d), r(d, E) * d ** -0.5, r(T, d), r(E, ctx.capacity, d), r(T, d), r(T, d), r(T, d), r(T, d)
    norm = ms.make_norm(w_post=r(d), gate=r(-(-T // 7), d), w_pre=r(d), rows_per_gate=7)

    def norm_bwd():
        out = [torch.full((T, d), float("nan"), dtype=dt, device=dev) for _ in range(2)]
        out += [torch.full(s, float("nan"), device=dev) for s in ((d,), (-(-T // 7), d), (d,))]
        ms.block_norm_bwd(ctx, dro, dh, y, rows, norm, *out)
        return out

    def route(between):
        b = ms.RouterBuffers(ctx)
        ms.route_fwd(ctx, h, wg, None, *b.args())
        extra = norm_bwd() if between else None
        dyexp, dgw, dl, dwg, dH = (torch.empty_like(yexp), torch.empty(T, k, device=dev), torch.empty(T, E, device=dev), torch.empty(d, E, device=dev),
                                   torch.empty_like(h))
        ms.route_bwd(ctx, dY, yexp, h, wg, b.logits, b.expert_idx, b.slot_idx, b.gate_w, b.slot_token, dyexp, dgw, dl, dwg, dH)
        torch.cuda.synchronize()
        assert ms.read_stats(b.stats).status == 0 and ms.check_internal(ctx) == 0
        return [b.expert_idx, b.slot_idx, b.expert_load, b.gate_w, dyexp, dgw, dl, dH], extra
    alone, extra = norm_bwd(), None
    want, _ = route(False)
    got, extra = route(True)
    again, _ = route(False)
    for a, b, c in zip(want, got, again):
        assert torch.equal(a, b) and torch.equal(a, c)
    for a, b in zip(alone, extra):
        assert torch.equal(a, b)
