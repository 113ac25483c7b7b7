"""What the 8-bit expert calls refuse before anything reaches a GPU."""
import ctypes as C
import types

import pytest
import torch

from paper_2508_12801_b200 import binding as ms

INVALID, UNSUPPORTED = 1, 6


def host_ctx(**kw):
    """A context's leading members (parameters, capacity) in host memory: enough for checks that come before any launch."""
    p = ms.make_params(**{**dict(T=8, d_model=64, E=4, k=2, io_dtype=ms.BF16), **kw})
    buf = C.create_string_buffer(8192)
    C.memmove(buf, C.byref(p), C.sizeof(p))
    C.c_int32.from_buffer(buf, C.sizeof(p)).value = ms.capacity(p)          # 4
    return buf


A = [0x100000 * (i + 1) for i in range(8)]
CALLS = {        # name: (number of pointers, trailing sizes)
    "dispatch_q8": (6, ()), "expert_quant": (4, (64,)), "expert_quant_weight": (3, (64, 32, 0)), "expert_gemm_q8": (6, (64, 32)),
    "expert_glu_q8": (6, (64, 32)), "expert_glu_keep8": (5, (64, 32, 0)), "expert_glu_bwd_keep8": (6, (64, 32, 0))}


def call(name, ctx, ptrs, sizes):
    return getattr(ms._lib, "maxscore_" + name)(ctx, *ptrs, *sizes, None)


@pytest.mark.parametrize("name", CALLS)
def test_null_arguments(name):
    n, sizes = CALLS[name]
    assert call(name, None, A[:n], sizes) == INVALID
    for i in range(n):
        if name == "expert_glu_bwd_keep8" and i == 5:
            continue                                                         # h may be NULL
        assert call(name, host_ctx(), A[:i] + [None] + A[i + 1:n], sizes) == INVALID, i


@pytest.mark.parametrize("name", CALLS)
def test_fp32_contexts(name):
    n, sizes = CALLS[name]
    assert call(name, host_ctx(io_dtype=ms.F32), A[:n], sizes) == UNSUPPORTED


@pytest.mark.parametrize("name, sizes, want", [
    ("expert_quant", (0,), INVALID), ("expert_quant", (-16,), INVALID), ("expert_quant", (24,), UNSUPPORTED), ("expert_quant", (1 << 17,), UNSUPPORTED),
    ("expert_quant_weight", (64, 32, 2), INVALID), ("expert_quant_weight", (64, 32, -1), INVALID), ("expert_quant_weight", (72, 32, 0), UNSUPPORTED),
    ("expert_quant_weight", (64, 36, 0), UNSUPPORTED), ("expert_quant_weight", (64, (1 << 24) + 8, 0), UNSUPPORTED),
    ("expert_gemm_q8", (0, 32), INVALID), ("expert_gemm_q8", (64, -8), INVALID), ("expert_gemm_q8", (40, 32), UNSUPPORTED),
    ("expert_gemm_q8", (1 << 17, 32), UNSUPPORTED), ("expert_gemm_q8", (64, 20), UNSUPPORTED),
    ("expert_glu_q8", (64, 0), INVALID), ("expert_glu_q8", (8, 32), UNSUPPORTED), ("expert_glu_q8", (64, 12), UNSUPPORTED),
    ("expert_glu_q8", (64, (1 << 23) + 8), UNSUPPORTED),
    ("expert_glu_keep8", (64, 32, 3), INVALID), ("expert_glu_keep8", (64, 0, 0), INVALID), ("expert_glu_keep8", (60, 32, 0), UNSUPPORTED),
    ("expert_glu_keep8", (64, 36, 0), UNSUPPORTED), ("expert_glu_keep8", ((1 << 18) + 8, 32, 0), UNSUPPORTED),
    ("expert_glu_bwd_keep8", (64, 32, -1), INVALID), ("expert_glu_bwd_keep8", (64, 36, 0), UNSUPPORTED),
    ("expert_glu_bwd_keep8", ((1 << 18) + 8, 32, 0), UNSUPPORTED)])
def test_sizes(name, sizes, want):
    assert call(name, host_ctx(), A[:CALLS[name][0]], sizes) == want


def test_dispatch_row_width():
    assert call("dispatch_q8", host_ctx(d_model=72), A[:6], ()) == UNSUPPORTED


@pytest.mark.parametrize("name, arg", [("dispatch_q8", 0), ("dispatch_q8", 4), ("dispatch_q8", 5), ("expert_quant", 0), ("expert_quant", 2),
                                       ("expert_quant_weight", 1), ("expert_gemm_q8", 0), ("expert_gemm_q8", 1), ("expert_gemm_q8", 3),
                                       ("expert_gemm_q8", 5), ("expert_glu_q8", 2), ("expert_glu_keep8", 3), ("expert_glu_keep8", 4),
                                       ("expert_glu_bwd_keep8", 2), ("expert_glu_bwd_keep8", 5)])
def test_alignment(name, arg):
    n, sizes = CALLS[name]
    assert call(name, host_ctx(), A[:arg] + [A[arg] + 8] + A[arg + 1:n], sizes) == INVALID


def test_kept_buffers_start_on_32_bytes():
    assert call("expert_glu_keep8", host_ctx(), A[:3] + [A[3] + 16, A[4]], (64, 32, 0)) == INVALID
    assert call("expert_glu_bwd_keep8", host_ctx(), A[:2] + [A[2] + 16] + A[3:6], (64, 32, 0)) == INVALID


@pytest.mark.parametrize("name, outs", [("dispatch_q8", (4, 5)), ("expert_quant", (2, 3)), ("expert_quant_weight", (1, 2)), ("expert_gemm_q8", (5,)),
                                        ("expert_glu_q8", (5,)), ("expert_glu_keep8", (3, 4)), ("expert_glu_bwd_keep8", (4, 5))])
def test_outputs_that_share_memory(name, outs):
    n, sizes = CALLS[name]
    for o in outs:
        for i in range(n):
            if i != o:
                ptrs = A[:n]
                ptrs[o] = A[i]
                assert call(name, host_ctx(), ptrs, sizes) == INVALID, (o, i)


def test_kept_scales_count_as_the_buffer():
    # E 4, C 4, d_ff 40: 4 * 4 * 2 * 64 integers = 2048 bytes, then 4 * 4 * 4 scales of 4 bytes
    n = C.c_size_t()
    ctx = host_ctx()
    assert ms._lib.maxscore_keep8_bytes(ctx, 40, C.byref(n)) == 0 and n.value == 2048 + 256
    assert call("expert_glu_keep8", ctx, A[:3] + [A[4] - 2272, A[4]], (64, 40, 0)) == INVALID
    assert ms._lib.maxscore_keep8_bytes(ctx, 40, None) == INVALID
    assert ms._lib.maxscore_keep8_bytes(None, 40, C.byref(n)) == INVALID
    assert ms._lib.maxscore_keep8_bytes(ctx, 0, C.byref(n)) == INVALID
    assert ms._lib.maxscore_keep8_bytes(ctx, 36, C.byref(n)) == UNSUPPORTED
    assert ms._lib.maxscore_keep8_bytes(host_ctx(io_dtype=ms.F32), 40, C.byref(n)) == UNSUPPORTED


@pytest.mark.parametrize("E, T, k, d_ff", [(4, 8, 2, 40), (1, 1, 1, 8), (128, 65536, 8, 1024), (33, 777, 5, 1000), (3, 100, 3, 31 * 8)])
def test_size_of_a_kept_buffer(E, T, k, d_ff):
    ctx = types.SimpleNamespace(handle=host_ctx(E=E, T=T, k=k), params=ms.make_params(T, 64, E, k), capacity=ms.capacity(ms.make_params(T, 64, E, k)))
    assert ms._keep8_numel(ctx, d_ff) == ms.keep8_bytes(ctx, d_ff)


def test_binding_checks_tensors():
    ctx = types.SimpleNamespace(device_index=-1, device="cpu", params=ms.make_params(8, 64, 4, 2), capacity=4, io_torch=torch.bfloat16, handle=None)
    x = torch.zeros(4, 4, 64, dtype=torch.bfloat16)
    load, q, s = torch.zeros(4, dtype=torch.int32), torch.zeros(4, 4, 64, dtype=torch.int8), torch.zeros(4, 4)
    with pytest.raises(ValueError, match="q:"):
        ms.expert_quant(ctx, x, load, q.view(torch.uint8), s, 64)
    with pytest.raises(ValueError, match="q_scale"):
        ms.expert_quant(ctx, x, load, q, s[:2], 64)
    with pytest.raises(ValueError, match="x_scale"):
        ms.expert_gemm_q8(ctx, q, s.double(), q, s, load, x, 64, 64)
    with pytest.raises(ValueError, match="src"):
        ms.dispatch_q8(ctx, x.float(), None, None, None, q, s)
