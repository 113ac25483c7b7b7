"""Routing by top-k on rows that hold a NaN: it is chosen ahead of every number, counts as nothing in its group's value, and whether it shows does
not depend on how near the row's other values are.  (Sigmoid scores: with the softmax all scores of such a row are NaN.)"""
import math

import pytest
import torch

from test_gpu_topk import F64, run, scores64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ms():
    from paper_2508_12801_b200 import binding
    return binding


def choose(l, bias, k, groups, keep, pairs):
    T, E = l.shape
    c = scores64(l, True)
    if bias is not None:
        c = c + bias.to(F64)
    by = c if bias is not None else l.to(F64)
    ok = torch.ones(T, E, dtype=torch.bool)
    if groups > 1:
        v = (c if pairs else by).view(T, groups, -1)
        v = torch.where(v.isnan(), -math.inf, v).sort(dim=2, descending=True).values
        v = v[:, :, :2].sum(2) if pairs else v[:, :, 0]
        v = torch.where(v.isnan(), -math.inf, v)                       # inf - inf
        best = v.sort(dim=1, descending=True, stable=True).indices[:, :keep]
        ok = torch.zeros(T, groups, dtype=torch.bool).scatter_(1, best, True).repeat_interleave(E // groups, 1)
    # stable sorts, the least important first: by value, NaN ahead, experts of lost groups behind
    order = by.nan_to_num(nan=0.0, posinf=math.inf, neginf=-math.inf).sort(dim=1, descending=True, stable=True).indices
    for first in (by.isnan(), ok):
        order = order.gather(1, first.gather(1, order).to(torch.int8).sort(dim=1, descending=True, stable=True).indices)
    return order[:, :k].sort(1).values


# a warp a token, and eight lanes a token
@pytest.mark.parametrize("T", [130, 2601])
@pytest.mark.parametrize("E, groups, keep", [(128, 8, 4), (64, 1, 1), (33, 3, 2), (40, 5, 3), (128, 1, 1)])
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("pairs", [False, True])
def test_rows_with_a_nan(ms, T, E, groups, keep, with_bias, pairs):
    if pairs and groups == 1:
        pytest.skip("no groups, no pairs")
    g = torch.Generator().manual_seed(E + T)
    l = torch.randn(T, E, generator=g)
    l[1::2] = torch.randint(-1, 2, (len(l[1::2]), E), generator=g).float()         # ties: chosen in 64 bits where there is a bias
    rows = torch.arange(0, T, 3)
    l[rows, torch.randint(0, E, (len(rows),), generator=g)] = math.nan
    l[rows[::2], torch.randint(0, E, (len(rows[::2]),), generator=g)] = -math.nan
    l[rows[::5], torch.randint(0, E, (len(rows[::5]),), generator=g)] = math.inf
    l[6] = math.nan
    l[9] = -math.inf
    l[9, 2] = math.nan
    l[12, :E // groups] = math.nan                                              # the whole first group
    bias = torch.randint(0, 3, (E,), generator=g) * 0.125 if with_bias else None
    k = min(6, E // groups * keep)
    want = choose(l, bias, k, groups, keep, pairs)
    for renorm in (True, False):
        s, idx, w = run(ms, l, bias, k, ms.make_topk(ms.SIGMOID, groups, keep, pairs, renorm))
        assert torch.equal(idx, want), f"{(idx != want).any(1).sum()} rows differ"
        assert torch.equal(s.isnan(), l.isnan())
        shown = l.isnan().gather(1, idx)
        assert torch.equal(w.isnan(), shown.any(1, keepdim=True).expand_as(shown) if renorm else shown)


@pytest.mark.parametrize("T", [130, 2601])
def test_infinite_biases_next_to_nan(ms, T):
    """A bias of +inf comes behind NaN and ahead of every finite value; a pair of +inf and -inf makes its group the last."""
    E, groups, keep, k = 64, 8, 4, 8
    g = torch.Generator().manual_seed(T)
    l = torch.randint(-2, 3, (T, E), generator=g).float()
    l[::4, 5] = math.nan
    bias = torch.randn(E, generator=g) * 0.1
    bias[17] = math.inf
    bias[40] = math.inf
    bias[41:48] = -math.inf                                                  # its group: inf and -inf
    bias[3] = math.nan
    for pairs in (False, True):
        for n, m in ((1, 1), (groups, keep)):
            _, idx, _ = run(ms, l, bias, k, ms.make_topk(ms.SIGMOID, n, m, pairs))
            assert torch.equal(idx, choose(l, bias, k, n, m, pairs))
