"""Norm calls whose ring slots are filled again while the first token of a CTA is still being worked on: every repeat of a call gives the
same bits.  The sizes leave some CTAs without tokens beside busy ones (units of three or four tokens), where copies come soonest."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,vecs", [(635, 192), (635, 200), (635, 213), (635, 224), (635, 256), (1077, 214), (635, 96), (1500, 64), (331, 512), (331, 700)])
def test_repeats_bit_for_bit(T, vecs, dtype):
    from paper_2508_12801_b200 import binding as ms
    dt, d = (torch.bfloat16, 8 * vecs) if dtype == "bf16" else (torch.float32, 4 * vecs)
    ctx = ms.create(ms.make_params(T, d, 8, 3, 1.0, io_dtype=ms.BF16 if dtype == "bf16" else ms.F32), DEV)
    g = torch.Generator(device=DEV).manual_seed(vecs)
    r = lambda *s: torch.empty(*s, dtype=dt, device=DEV).normal_(generator=g)  # noqa: E731
    norm = ms.make_norm(w_post=r(d), w_pre=r(d))
    y, rows, dro, dh, src = r(T, d), r(T, d), r(T, d), r(T, d), r(8, ctx.capacity, d)
    idx = torch.rand(T, 8, generator=g, device=DEV).topk(3, dim=1).indices.sort(dim=1).values.to(torch.int32)
    slot = torch.randint(0, ctx.capacity, (T, 3), generator=g, device=DEV, dtype=torch.int32)

    def call():
        dy, dr, r1, h1, y2, r2, h2 = (torch.full((T, d), 7.0, dtype=dt, device=DEV) for _ in range(7))
        a, c = (torch.full((d,), 7.0, device=DEV) for _ in range(2))
        ms.block_norm_bwd(ctx, dro, dh, y, rows, norm, dy, dr, a, None, c)
        ms.block_norm(ctx, y, rows, norm, r1, h1)
        ms.combine_norm(ctx, src, idx, slot, None, rows, norm, y2, r2, h2)
        return dy, dr, a, c, r1, h1, y2, r2, h2
    first, second = call(), call()
    assert same(first, second)
    for _ in range(300):
        assert same(call(), first)
    assert ms.check_internal(ctx) == 0
