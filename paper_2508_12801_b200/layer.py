"""One MoE layer of a decoder from the library's calls: routing, dispatch, SwiGLU experts, combine, and the norms,
gate and residual around them.  The paper's models (Sec. 4.1) have SwiGLU experts and a plain RMSNorm before each block: a norm with
w_pre alone; after-norm and gate are for models that have them.

    r' = res_scale * r + gate * norm_post(combine(experts(dispatch(h))))        h' = norm_pre(r')

h is the normalised stream that the norm in front of the block left (binding.block_norm without y for a first layer); h' is what
the next block takes.  Every step is one call of the C library on buffers that the layer allocates once; forward and backward
enqueue work on the current stream and can be captured into a CUDA graph.  With the paper's router the auxiliary loss is not part of
it: a caller who wants it takes the calls below with combine_bwd, softtopk_bwd_aux and gate_bwd in route_bwd's place.

Forms of the layer:
    topk   routing by top-k (binding.make_topk) in place of SoftTopk and the flow; the balance loss enters the backward pass by dscores_col
    keep8  training with the experts' activations kept in 8 bits: [g | u] as integers, h formed again and the rows dispatched again in
           the backward pass, so that between the passes a layer holds yexp, `keep`, y [T, d_model] and the router's rows (logits, scores, indices,
           weights), beside its context's workspace; the other buffers may be another layer's
    int8   serving with rows and weights in 8-bit integers (weights from MoELayer.quantise)
"""
from __future__ import annotations

import torch

from . import binding as ms


class MoELayer:
    """Weights: w_gate as params.w_gate_layout says, w_up [E, d, 2 d_ff] and w_down [E, d_ff, d] (w_layout 1: the transposes),
    norm weights and gate as in binding.make_norm (any of them None).  training=False keeps nothing for the backward pass.
    share: a layer of the same sizes, type and form whose working buffers this one uses too; their calls must not overlap."""

    def __init__(self, params: ms.Params, d_ff: int, w_layout: int = 0, training: bool = True, device="cuda:0", topk: ms.TopK | None = None,
                 keep8: bool = False, int8: bool = False, share: "MoELayer | None" = None):
        if (keep8 or int8) and params.io_dtype != ms.BF16:
            raise ValueError("keep8 and int8 need bf16 I/O")
        if keep8 and not training:
            raise ValueError("keep8 is a form of training")
        if int8 and training:
            raise ValueError("int8 is a form of serving: training=False")
        # what the products take (a backward pass contracts over 2 d_ff columns)
        unit, most = (16, (1 << 17) - 16) if int8 else (8, 1 << 18) if params.io_dtype == ms.BF16 else (4, 1 << 24)
        for name, width, top in (("d_model", params.d_model, most), ("d_ff", d_ff, most // 2 if training else most)):
            if width <= 0 or width % unit or width > top:
                raise ValueError(f"{name} = {width}: a multiple of {unit} up to {top} is needed")
        self.ctx = ms.create(params, device)
        self.d_ff, self.w_layout, self.training, self.topk, self.keep8, self.int8 = d_ff, w_layout, training, topk, keep8, int8
        p, C, io, dev = params, self.ctx.capacity, self.ctx.io_torch, self.ctx.device
        shape = (p.T, p.d_model, p.E, p.k, C, p.io_dtype, d_ff, training, keep8, int8, str(dev))
        if share is not None and share._shape != shape:
            raise ValueError("share: a layer of the same sizes, type, form and device is needed")
        self._shape = shape
        new = lambda *s, dtype=io: torch.empty(*s, dtype=dtype, device=dev)  # noqa: E731
        # buffers that no later call of this layer reads once a pass is over
        work = (lambda name, make: getattr(share, name)) if share is not None else (lambda name, make: make())
        # ... of these, what the backward pass reads unless it is formed again there
        saved = work if keep8 or not training else (lambda name, make: make())
        self.route = ms.RouterBuffers(self.ctx)
        if int8:
            self.xq, self.x_scale = work("xq", lambda: new(p.E, C, p.d_model, dtype=torch.int8)), work("x_scale", lambda: new(p.E, C, dtype=torch.float32))
            self.hq, self.h_scale = work("hq", lambda: new(p.E, C, d_ff, dtype=torch.int8)), work("h_scale", lambda: new(p.E, C, dtype=torch.float32))
        else:
            self.x = saved("x", lambda: new(p.E, C, p.d_model))          # dispatched rows
        self.h = saved("h", lambda: new(p.E, C, d_ff))                   # activations of the experts
        self.yexp = new(p.E, C, p.d_model) if training else work("yexp", lambda: new(p.E, C, p.d_model))      # outputs of the experts
        self.y = new(p.T, p.d_model) if training else None
        self.pre = new(p.E, C, 2 * d_ff) if training and not keep8 else None
        self.keep = new(ms.keep8_bytes(self.ctx, d_ff), dtype=torch.uint8) if keep8 else None
        if training:
            self.dyexp, self.dpre = work("dyexp", lambda: new(p.E, C, p.d_model)), work("dpre", lambda: new(p.E, C, 2 * d_ff))
            self.dx, self.dy = work("dx", lambda: new(p.E, C, p.d_model)), work("dy", lambda: new(p.T, p.d_model))
            self.dgate_w = work("dgate_w", lambda: new(p.T, p.k, dtype=torch.float32))
            self.dlogits = work("dlogits", lambda: new(p.T, p.E, dtype=torch.float32))

    def quantise(self, w_up, w_down, stream=None):
        """The experts' weights as an int8 layer takes them: ((integers, scales) of w_up, the same of w_down), once per weight.  They belong to
        `stream`, the current one if there is none."""
        d, f, E, dev = self.ctx.params.d_model, self.d_ff, self.ctx.params.E, self.ctx.device
        out = []
        if stream is not None and not isinstance(stream, torch.cuda.Stream):
            stream = torch.cuda.ExternalStream(getattr(stream, "cuda_stream", stream), device=dev)
        for w, d_in, d_out in ((w_up, d, 2 * f), (w_down, f, d)):
            # memory of the stream that writes it: the current one's may still be read by what it has queued
            with torch.cuda.stream(stream):
                q, s = torch.empty(E, d_out, d_in, dtype=torch.int8, device=dev), torch.empty(E, d_out, dtype=torch.float32, device=dev)
            ms.expert_quant_weight(self.ctx, w, q, s, d_in, d_out, self.w_layout, stream=stream)
            out.append((q, s))
        return tuple(out)

    def forward(self, h, residual, w_gate, w_up, w_down, norm, r_out, h_out, expert_bias=None, stream=None, balance_bias=None):
        """r_out and h_out [T, d_model] are written (r_out may be residual's buffer; h_out None without norm.w_pre).  expert_bias [E] is added
        to the logits, balance_bias [E] (topk) to the scores for the choice alone.  int8: w_up and w_down as quantise returns them."""
        c, b, d, f = self.ctx, self.route, self.ctx.params.d_model, self.d_ff
        if balance_bias is not None and self.topk is None:
            raise ValueError("balance_bias: routing by top-k is needed")
        if self.topk is None:
            ms.route_fwd(c, h, w_gate, expert_bias, *b.args(), stream=stream)
        else:
            ms.gate(c, h, w_gate, expert_bias, b.logits, stream=stream)
            ms.topk_fwd(c, b.logits, balance_bias, self.topk, b.scores, b.expert_idx, b.gate_w, stream=stream)
            ms.index_build(c, b.expert_idx, b.slot_idx, b.slot_token, b.expert_load, stream=stream)
        if self.int8:
            ms.dispatch_q8(c, h, b.expert_idx, b.slot_idx, b.slot_token, self.xq, self.x_scale, stream=stream)
            ms.expert_glu_q8(c, self.xq, self.x_scale, *w_up, b.expert_load, self.h, d, f, stream=stream)
            ms.expert_quant(c, self.h, b.expert_load, self.hq, self.h_scale, f, stream=stream)
            ms.expert_gemm_q8(c, self.hq, self.h_scale, *w_down, b.expert_load, self.yexp, f, d, stream=stream)
        else:
            ms.dispatch(c, h, b.expert_idx, b.slot_idx, b.slot_token, self.x, stream=stream)
            if self.keep8:
                ms.expert_glu_keep8(c, self.x, w_up, b.expert_load, self.keep, self.h, d, f, self.w_layout, stream=stream)
            else:
                ms.expert_glu(c, self.x, w_up, b.expert_load, self.pre, self.h, d, f, self.w_layout, stream=stream)
            ms.expert_gemm(c, self.h, w_down, b.expert_load, self.yexp, f, d, self.w_layout, stream=stream)
        ms.combine_norm(c, self.yexp, b.expert_idx, b.slot_idx, b.gate_w, residual, norm, self.y, r_out, h_out, stream=stream)

    def backward(self, dr_out, dh_out, h, r_out, w_gate, w_up, w_down, norm, dh, dr, dw_gate, dw_up, dw_down, dw_post=None,
                 dgate=None, dw_pre=None, accumulate=0, stream=None, dscores_col=None):
        """Gradients of the last forward pass with the assignment held constant: dh and dr [T, d_model] of h and residual,
        parameter gradients in fp32 (accumulate != 0 adds to dw_up and dw_down; the others are overwritten).  In bf16 dh is rounded
        twice: route_bwd stores the gate's part of it and combine adds the experts' part, which saves an fp32 image of [T, d_model].
        dscores_col [E] (topk): gradient of every token's scores, binding.aux_loss's."""
        if not self.training:
            raise ValueError("backward: the layer was made with training=False")
        if dscores_col is not None and self.topk is None:
            raise ValueError("dscores_col: routing by top-k is needed")
        c, b, d, f, L = self.ctx, self.route, self.ctx.params.d_model, self.d_ff, self.w_layout
        ms.block_norm_bwd(c, dr_out, dh_out, self.y, r_out, norm, self.dy, dr, dw_post, dgate, dw_pre, stream=stream)
        if self.topk is None:
            ms.route_bwd(c, self.dy, self.yexp, h, w_gate, b.logits, b.expert_idx, b.slot_idx, b.gate_w, b.slot_token, self.dyexp,
                         self.dgate_w, self.dlogits, dw_gate, dh, stream=stream)
        else:
            ms.combine_bwd(c, self.dy, self.yexp, b.expert_idx, b.slot_idx, b.gate_w, b.slot_token, self.dyexp, self.dgate_w, stream=stream)
            ms.topk_bwd(c, b.logits, b.expert_idx, self.dgate_w, dscores_col, self.topk, self.dlogits, stream=stream)
            ms.gate_bwd(c, h, w_gate, self.dlogits, dw_gate, dh, stream=stream)
        if self.keep8:
            ms.dispatch(c, h, b.expert_idx, b.slot_idx, b.slot_token, self.x, stream=stream)
            ms.expert_glu_bwd_keep8(c, self.dyexp, w_down, self.keep, b.expert_load, self.dpre, self.h, d, f, L, stream=stream)
        else:
            ms.expert_glu_bwd(c, self.dyexp, w_down, self.pre, b.expert_load, self.dpre, d, f, L, stream=stream)
        ms.expert_gemm_dw(c, self.h, self.dyexp, b.expert_load, dw_down, f, d, L, accumulate, stream=stream)
        ms.expert_gemm_dw(c, self.x, self.dpre, b.expert_load, dw_up, d, 2 * f, L, accumulate, stream=stream)
        ms.expert_gemm(c, self.dpre, w_up, b.expert_load, self.dx, 2 * f, d, 1 - L, stream=stream)
        ms.combine(c, self.dx, b.expert_idx, b.slot_idx, None, dh, accumulate=1, stream=stream)      # backward of dispatch
