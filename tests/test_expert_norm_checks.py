"""What the expert and norm calls refuse before anything reaches a GPU."""
import types

import pytest
import torch

from paper_2508_12801_b200 import binding as ms

INVALID = 1


def test_no_context_is_refused_by_every_call():
    lib, z = ms._lib, None
    assert lib.maxscore_expert_gemm(z, z, z, z, z, 8, 8, 0, z) == INVALID
    assert lib.maxscore_expert_gemm_dw(z, z, z, z, z, 8, 8, 0, 0, z) == INVALID
    assert lib.maxscore_expert_glu(z, z, z, z, z, z, 8, 8, 0, z) == INVALID
    assert lib.maxscore_expert_glu_bwd(z, z, z, z, z, z, 8, 8, 0, z) == INVALID
    n = ms.make_norm()
    assert lib.maxscore_combine_norm(z, z, z, z, z, z, ms.C.byref(n), z, z, z, z) == INVALID
    assert lib.maxscore_block_norm(z, z, z, ms.C.byref(n), z, z, z) == INVALID
    assert lib.maxscore_block_norm_bwd(z, z, z, z, z, ms.C.byref(n), z, z, z, z, z, z) == INVALID


def test_norm_struct_matches_header():
    assert ms.C.sizeof(ms.Norm) == 3 * 8 + 4 * 4 and ms.Norm.res_scale.offset == 36
    w = torch.ones(8)
    n = ms.make_norm(w_pre=w, rows_per_gate=3, eps=1e-6, w_offset=1.0, res_scale=0.5)
    assert n.w_pre == w.data_ptr() and n.w_post is None and n.gate is None and n.rows_per_gate == 3
    assert n.w_offset == 1.0 and n.res_scale == 0.5


@pytest.mark.parametrize("t", [torch.zeros(4, 8), torch.zeros(4, 8, dtype=torch.bfloat16)[:, :4], torch.zeros(32, dtype=torch.bfloat16),
                               torch.zeros(8, 4, dtype=torch.bfloat16).t(), None])
def test_tensor_checks(t):
    ctx = types.SimpleNamespace(device_index=0, device="cuda:0")
    with pytest.raises(ValueError, match="x"):
        ms._need(ctx, "x", t, torch.bfloat16, 32)


def test_optional_tensors():
    ctx = types.SimpleNamespace(device_index=-1, device="cpu")
    assert ms._need(ctx, "x", None, torch.float32, 4, optional=True) is None
    t = torch.zeros(4)
    assert ms._need(ctx, "x", t, torch.float32, 4) == t.data_ptr()
