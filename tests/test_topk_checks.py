"""What routing by top-k refuses before anything reaches a GPU, and its argument struct."""
import ctypes as C

import pytest
import torch

from paper_2508_12801_b200 import binding as ms

OK, INVALID, UNSUPPORTED = 0, 1, 6


def host_ctx(**kw):
    """A context's leading members (parameters, capacity) in host memory: enough for checks that come before any launch."""
    p = ms.make_params(**{**dict(T=4, d_model=64, E=8, k=2), **kw})
    buf = C.create_string_buffer(8192)
    C.memmove(buf, C.byref(p), C.sizeof(p))
    C.c_int32.from_buffer(buf, C.sizeof(p)).value = ms.capacity(p)
    return buf


def test_struct_matches_header():
    assert C.sizeof(ms.TopK) == 24 and ms.TopK.scale.offset == 20
    h = ms.make_topk(ms.SIGMOID, 8, 4, True, False, 2.5)
    assert (h.score, h.n_group, h.topk_group, h.group_pairs, h.renorm, h.scale) == (1, 8, 4, 1, 0, 2.5)


def calls(ctx, how, logits, bias, scores, idx, w):
    h = None if how is None else C.byref(how)
    return (ms._lib.maxscore_topk_fwd(ctx, logits, bias, h, scores, idx, w, None),
            ms._lib.maxscore_topk_bwd(ctx, logits, idx, w, bias, h, scores, None))


def test_null_arguments():
    a = [0x1000 * (i + 1) for i in range(5)]
    ctx, how = host_ctx(), ms.make_topk()
    assert calls(None, how, *a) == (INVALID, INVALID)
    assert calls(ctx, None, *a) == (INVALID, INVALID)
    assert calls(ctx, how, None, *a[1:]) == (INVALID, INVALID)
    assert calls(ctx, how, *a[:3], None, a[4]) == (INVALID, INVALID)
    assert calls(ctx, how, *a[:4], None) == (INVALID, INVALID)
    assert ms._lib.maxscore_topk_bwd(ctx, a[0], a[3], a[4], None, C.byref(how), None, None) == INVALID


@pytest.mark.parametrize("kw, want", [
    (dict(score=2), INVALID), (dict(score=-1), INVALID), (dict(renorm=2), INVALID), (dict(group_pairs=-1), INVALID),
    (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID), (dict(n_group=-1), INVALID),
    (dict(n_group=3, topk_group=1), INVALID), (dict(n_group=4, topk_group=0), INVALID), (dict(n_group=4, topk_group=5), INVALID),
    (dict(n_group=8, topk_group=1), INVALID)])                  # one group of one expert for k = 2
def test_members(kw, want):
    how = ms.make_topk()
    for n, v in kw.items():
        setattr(how, n, v)
    assert calls(host_ctx(), how, *(0x1000 * (i + 1) for i in range(5))) == (want, want)


def test_too_many_groups():
    ctx = host_ctx(E=128)
    assert calls(ctx, ms.make_topk(n_group=64, topk_group=32), *(0x1000 * (i + 1) for i in range(5))) == (UNSUPPORTED, UNSUPPORTED)


@pytest.mark.parametrize("off", [4, 8])
def test_alignment(off):
    a = [0x1000 * (i + 1) for i in range(5)]
    assert calls(host_ctx(), ms.make_topk(), a[0] + off, *a[1:]) == (INVALID, INVALID)
    assert calls(host_ctx(), ms.make_topk(), *a[:2], a[2] + off, *a[3:]) == (INVALID, INVALID)
    assert calls(host_ctx(), ms.make_topk(), a[0], a[1] + 2, *a[2:]) == (INVALID, INVALID)


def test_overlaps():
    lib, how, ctx = ms._lib, ms.make_topk(), host_ctx()          # T E = 32 floats of 128 bytes, T k = 8 of 32, E = 8 of 32
    fwd = lambda l, b, s, i, w: lib.maxscore_topk_fwd(ctx, l, b, C.byref(how), s, i, w, None)  # noqa: E731
    bwd = lambda l, i, w, c, o: lib.maxscore_topk_bwd(ctx, l, i, w, c, C.byref(how), o, None)  # noqa: E731
    assert fwd(0x1000, None, 0x1000, 0x2000, 0x3000) == INVALID
    assert fwd(0x1000, None, 0x1070, 0x2000, 0x3000) == INVALID
    assert fwd(0x1000, 0x2010, 0x4000, 0x2000, 0x3000) == INVALID
    assert fwd(0x1000, None, 0x4000, 0x2000, 0x201c) == INVALID
    assert bwd(0x1000, 0x2000, 0x3000, None, 0x1000) == INVALID
    assert bwd(0x1000, 0x2000, 0x3000, None, 0x2010) == INVALID
    assert bwd(0x1000, 0x2000, 0x3000, 0x4000, 0x3f90) == INVALID


def test_binding_checks_tensors():
    import types
    ctx = types.SimpleNamespace(device_index=-1, device="cpu", params=ms.make_params(4, 64, 8, 2), handle=None)
    f = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="logits"):
        ms.topk_fwd(ctx, f.double(), None, ms.make_topk(), None, None, None)
    with pytest.raises(ValueError, match="expert_idx"):
        ms.topk_fwd(ctx, f, None, ms.make_topk(), None, torch.zeros(4, 2), torch.zeros(4, 2))
    with pytest.raises(ValueError, match="bias"):
        ms.topk_fwd(ctx, f, torch.zeros(7), ms.make_topk(), None, torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2))
    with pytest.raises(ValueError, match="dscores_col"):
        ms.topk_bwd(ctx, f, torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2), torch.zeros(8, 2), ms.make_topk(), f)
