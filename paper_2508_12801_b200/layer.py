"""One MoE layer of a decoder from the library's calls: routing, dispatch, SwiGLU experts, combine, and the norms,
gate and residual around them.  The paper's models (Sec. 4.1) have SwiGLU experts and a plain RMSNorm before each block: a norm with
w_pre alone; after-norm and gate are for models that have them.

    r' = res_scale * r + gate * norm_post(combine(experts(dispatch(h))))        h' = norm_pre(r')

h is the normalised stream that the norm in front of the block left (binding.block_norm without y for a first layer); h' is what
the next block takes.  Every step is one call of the C library on buffers that the layer allocates once; forward and backward
enqueue work on the current stream and can be captured into a CUDA graph.  The auxiliary loss is not part of it: a caller who wants
it takes the calls below with combine_bwd, softtopk_bwd_aux and gate_bwd in route_bwd's place.
"""
from __future__ import annotations

import torch

from . import binding as ms


class MoELayer:
    """Weights: w_gate as params.w_gate_layout says, w_up [E, d, 2 d_ff] and w_down [E, d_ff, d] (w_layout 1: the transposes),
    norm weights and gate as in binding.make_norm (any of them None).  training=False keeps nothing for the backward pass."""

    def __init__(self, params: ms.Params, d_ff: int, w_layout: int = 0, training: bool = True, device="cuda:0"):
        self.ctx = ms.create(params, device)
        self.d_ff, self.w_layout, self.training = d_ff, w_layout, training
        p, C, io, dev = params, self.ctx.capacity, self.ctx.io_torch, self.ctx.device
        new = lambda *s, dtype=io: torch.empty(*s, dtype=dtype, device=dev)  # noqa: E731
        self.route = ms.RouterBuffers(self.ctx)
        self.x = new(p.E, C, p.d_model)                                  # dispatched rows
        self.h = new(p.E, C, d_ff)                                       # activations of the experts
        self.yexp = new(p.E, C, p.d_model)                               # outputs of the experts
        self.y = new(p.T, p.d_model) if training else None
        self.pre = new(p.E, C, 2 * d_ff) if training else None
        if training:
            self.dyexp, self.dpre, self.dx = new(p.E, C, p.d_model), new(p.E, C, 2 * d_ff), new(p.E, C, p.d_model)
            self.dy, self.dgate_w = new(p.T, p.d_model), new(p.T, p.k, dtype=torch.float32)
            self.dlogits = new(p.T, p.E, dtype=torch.float32)

    def forward(self, h, residual, w_gate, w_up, w_down, norm, r_out, h_out, expert_bias=None, stream=None):
        """r_out and h_out [T, d_model] are written (r_out may be residual's buffer; h_out None without norm.w_pre)."""
        c, b, d, f = self.ctx, self.route, self.ctx.params.d_model, self.d_ff
        ms.route_fwd(c, h, w_gate, expert_bias, *b.args(), stream=stream)
        ms.dispatch(c, h, b.expert_idx, b.slot_idx, b.slot_token, self.x, stream=stream)
        ms.expert_glu(c, self.x, w_up, b.expert_load, self.pre, self.h, d, f, self.w_layout, stream=stream)
        ms.expert_gemm(c, self.h, w_down, b.expert_load, self.yexp, f, d, self.w_layout, stream=stream)
        ms.combine_norm(c, self.yexp, b.expert_idx, b.slot_idx, b.gate_w, residual, norm, self.y, r_out, h_out, stream=stream)

    def backward(self, dr_out, dh_out, h, r_out, w_gate, w_up, w_down, norm, dh, dr, dw_gate, dw_up, dw_down, dw_post=None,
                 dgate=None, dw_pre=None, accumulate=0, stream=None):
        """Gradients of the last forward pass with the assignment held constant: dh and dr [T, d_model] of h and residual,
        parameter gradients in fp32 (accumulate != 0 adds to dw_up and dw_down; the others are overwritten).  In bf16 dh is rounded
        twice: route_bwd stores the gate's part of it and combine adds the experts' part, which saves an fp32 image of [T, d_model]."""
        if not self.training:
            raise ValueError("backward: the layer was made with training=False")
        c, b, d, f, L = self.ctx, self.route, self.ctx.params.d_model, self.d_ff, self.w_layout
        ms.block_norm_bwd(c, dr_out, dh_out, self.y, r_out, norm, self.dy, dr, dw_post, dgate, dw_pre, stream=stream)
        ms.route_bwd(c, self.dy, self.yexp, h, w_gate, b.logits, b.expert_idx, b.slot_idx, b.gate_w, b.slot_token, self.dyexp,
                     self.dgate_w, self.dlogits, dw_gate, dh, stream=stream)
        ms.expert_gemm_dw(c, self.h, self.dyexp, b.expert_load, dw_down, f, d, L, accumulate, stream=stream)
        ms.expert_glu_bwd(c, self.dyexp, w_down, self.pre, b.expert_load, self.dpre, d, f, L, stream=stream)
        ms.expert_gemm_dw(c, self.x, self.dpre, b.expert_load, dw_up, d, 2 * f, L, accumulate, stream=stream)
        ms.expert_gemm(c, self.dpre, w_up, b.expert_load, self.dx, 2 * f, d, 1 - L, stream=stream)
        ms.combine(c, self.dx, b.expert_idx, b.slot_idx, None, dh, accumulate=1, stream=stream)      # backward of dispatch
