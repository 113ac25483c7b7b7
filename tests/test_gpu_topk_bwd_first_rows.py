"""The backward pass of routing by top-k from sigmoid scores without renormalisation: nothing but the gradient's own row passes through shared
memory there, and a warp's first token follows right behind the zeroing of that row."""
import pytest
import torch

from test_gpu_topk import DEV, F64, dl64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ms():
    from paper_2508_12801_b200 import binding
    return binding


@pytest.mark.parametrize("T, E, k", [(1, 128, 8), (8, 33, 5), (9, 100, 1), (1000, 128, 8), (1184, 64, 8), (9472, 96, 3), (9472, 128, 8), (9473, 31, 8)])
@pytest.mark.parametrize("aux", [False, True])
def test_every_chosen_pair_has_its_gradient(ms, T, E, k, aux):
    g = torch.Generator().manual_seed(T + E)
    l = torch.randn(T, E, generator=g)
    idx = torch.rand(T, E, generator=g).topk(k, 1).indices.sort(1).values
    dw = torch.rand(T, k, generator=g) + 0.5                               # none is zero
    col = torch.randn(E, generator=g) if aux else None
    ctx = ms.create(ms.make_params(T, 64, E, k, capacity=T), DEV)
    how = ms.make_topk(ms.SIGMOID, renorm=False, scale=1.5)
    args = l.to(DEV), idx.to(torch.int32).to(DEV), dw.to(DEV), None if col is None else col.to(DEV)
    want = dl64(l, idx, dw, col, True, False, 1.5)
    # ds = 1.5 dw + col in two steps of 2^-24, its products with s and 1 - s (eight steps together) two more: 12 steps of the terms' sizes
    s = torch.sigmoid(l.to(F64))
    size = torch.zeros(T, E, dtype=F64).scatter_(1, idx, 1.5 * dw.to(F64)) + (0 if col is None else col.to(F64).abs())
    bar = 16 * 2.0 ** -24 * size * s * (1 - s)
    first = None
    for _ in range(30):
        dl = torch.full((T, E), -7.0, device=DEV)
        ms.topk_bwd(ctx, *args, how, dl)
        if first is None:
            first = dl
            assert ((dl.cpu().to(F64) - want).abs() <= bar).all()
        assert torch.equal(dl, first)
