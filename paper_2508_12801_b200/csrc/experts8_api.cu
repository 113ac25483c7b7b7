// C ABI of the experts in 8-bit integers and of expert activations kept in 8 bits (see include/maxscore.h): argument checks and kernel
// launches on the caller's stream.
#include "expert_launch.cuh"
#include "rows8.cuh"

using namespace msr;

namespace {

// Widths of integer rows: multiples of 16 (the copies' granularity), below 2^17 (|sum| < 2^31 whatever the integers).
bool width8(int32_t w) { return w % 16 == 0 && w < (1 << 17); }

maxscore_status check8(const maxscore_ctx* c, std::initializer_list<const void*> ptrs, int32_t w0, int32_t w1) {
  if (!c) return MAXSCORE_ERR_INVALID_ARG;
  for (const void* p : ptrs) if (!p || !aligned16(p)) return MAXSCORE_ERR_INVALID_ARG;
  if (w0 <= 0 || w1 <= 0) return MAXSCORE_ERR_INVALID_ARG;
  if (c->p.io_dtype != MAXSCORE_BF16) return MAXSCORE_ERR_UNSUPPORTED;
  return MAXSCORE_OK;
}

Span ints_span(const maxscore_ctx* c, const void* p, int64_t width) { return {p, (size_t)c->p.E * c->C * width}; }
Span row_scales_span(const maxscore_ctx* c, const void* p) { return {p, sizeof(float) * (size_t)c->p.E * c->C}; }
Span col_scales_span(const maxscore_ctx* c, const void* p, int64_t cols) { return {p, sizeof(float) * (size_t)c->p.E * cols}; }

// A warp holds a row of up to eight 16-element chunks a lane (4096 elements) from the first pass to the second; longer ones are read twice.
template <typename F>
void by_chunks(int chunks, F go) {
  if (chunks <= 32) go(std::integral_constant<int, 1>{});
  else if (chunks <= 64) go(std::integral_constant<int, 2>{});
  else if (chunks <= 128) go(std::integral_constant<int, 4>{});
  else if (chunks <= 256) go(std::integral_constant<int, 8>{});
  else go(std::integral_constant<int, 0>{});
}
int rows8_grid(const maxscore_ctx* c, int64_t rows) { return (int)std::max<int64_t>(1, std::min<int64_t>((rows + kRows8Warps - 1) / kRows8Warps, (int64_t)c->sm_count * 8)); }

maxscore_status launch_rows8(maxscore_ctx* c, const void* x, const int32_t* load, int8_t* q, float* scale, int64_t rows, int32_t width, cudaStream_t st) {
  by_chunks(width / 16, [&](auto v) {
    rows8_kernel<decltype(v)::value><<<rows8_grid(c, rows), kRows8Warps * 32, 0, st>>>((const uint4*)x, load, (uint4*)q, scale, rows, width / 16, c->C);
  });
  MS_LAUNCH_CHECK("rows8_kernel");
  c->launches += 1;
  return MAXSCORE_OK;
}

template <int EPI>
maxscore_status launch_int8(maxscore_ctx* c, const int8_t* xq, const float* xs, const int8_t* wq, const float* ws, const int32_t* load, void* out,
                            int32_t d_in, int32_t d_out, cudaStream_t st) {
  ExpertArgs a = expert_args(c, load, 0, d_out, d_in);
  a.x_scale = xs; a.w_scale = ws;
  // Few rows: weights on the MMA's M side, read once.  us, against the 256-row tiles: gated, 2048 -> 1024, E 64: C 16 49 / 55, 64 53 / 56,
  // 96 60 / 57, 128 72 / 59; 1024 -> 2048: C 16 26 / 37, 64 33 / 38, 96 41 / 39, 128 48 / 40; E 128, 2320 -> 400 and back: C 96 58 / 64, 70 / 78.
  if (c->C <= 80) return launch_few<EPI, false, kInt8>(c, xq, wq, out, nullptr, a, st);
  return launch_tc<EPI, false, kInt8>(c, xq, wq, nullptr, out, nullptr, a, st);
}

size_t keep_ints(const maxscore_ctx* c, int32_t d_ff) { return align_up((size_t)c->p.E * c->C * 2 * keep_width(d_ff), 256); }
size_t keep_bytes(const maxscore_ctx* c, int32_t d_ff) {
  return keep_ints(c, d_ff) + sizeof(float) * (size_t)c->p.E * (2 * keep_width(d_ff) / kKeepBlock) * c->C;
}
bool aligned32(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 31u) == 0; }

ExpertArgs keep_args(const maxscore_ctx* c, const int32_t* load, int32_t d_ff, int32_t K, void* keep) {
  ExpertArgs a = expert_args(c, load, 0, d_ff, K);
  a.keep = (int8_t*)keep; a.keep_scale = (float*)((char*)keep + keep_ints(c, d_ff));
  return a;
}

}  // namespace

extern "C" {

maxscore_status maxscore_dispatch_q8(maxscore_ctx* c, const void* src, const int32_t* expert_idx, const int32_t* slot_idx,
                                     const int32_t* slot_token, int8_t* dst, float* dst_scale, void* stream) {
  if (!c) return MAXSCORE_ERR_INVALID_ARG;
  const int32_t d = c->p.d_model;
  maxscore_status s = check8(c, {src, dst, dst_scale}, d, d);
  if (s) return s;
  if (!expert_idx || !slot_idx || !slot_token) return MAXSCORE_ERR_INVALID_ARG;
  if (!width8(d)) return MAXSCORE_ERR_UNSUPPORTED;
  const size_t pairs = sizeof(int32_t) * (size_t)c->p.T * c->p.k;
  if (!apart({ints_span(c, dst, d), row_scales_span(c, dst_scale)},
             {{src, (size_t)c->p.T * d * 2}, {expert_idx, pairs}, {slot_idx, pairs}, {slot_token, sizeof(int32_t) * (size_t)c->p.E * c->C}}))
    return MAXSCORE_ERR_INVALID_ARG;
  const int64_t work = std::max<int64_t>(c->p.T, ((int64_t)c->p.E * c->C + 31) / 32);
  by_chunks(d / 16, [&](auto v) {
    dispatch8_kernel<decltype(v)::value><<<rows8_grid(c, work), kRows8Warps * 32, 0, (cudaStream_t)stream>>>(
        (const uint4*)src, expert_idx, slot_idx, slot_token, (uint4*)dst, dst_scale, c->p.T, d / 16, c->p.E, c->p.k, c->C);
  });
  MS_LAUNCH_CHECK("dispatch8_kernel");
  c->launches += 1;
  return MAXSCORE_OK;
}

maxscore_status maxscore_expert_quant(maxscore_ctx* c, const void* x, const int32_t* expert_load, int8_t* q, float* q_scale, int32_t width,
                                      void* stream) {
  maxscore_status s = check8(c, {x, q, q_scale}, width, width);
  if (s) return s;
  if (!expert_load) return MAXSCORE_ERR_INVALID_ARG;
  if (!width8(width)) return MAXSCORE_ERR_UNSUPPORTED;
  if (!apart({ints_span(c, q, width), row_scales_span(c, q_scale)}, {rows_span(c, x, width), load_span(c, expert_load)})) return MAXSCORE_ERR_INVALID_ARG;
  return launch_rows8(c, x, expert_load, q, q_scale, (int64_t)c->p.E * c->C, width, (cudaStream_t)stream);
}

maxscore_status maxscore_expert_quant_weight(maxscore_ctx* c, const void* w, int8_t* wq, float* w_scale, int32_t d_in, int32_t d_out,
                                             int32_t w_layout, void* stream) {
  maxscore_status s = check8(c, {w, wq, w_scale}, d_in, d_out);
  if (s) return s;
  if (w_layout != 0 && w_layout != 1) return MAXSCORE_ERR_INVALID_ARG;
  if (!width8(d_in) || d_out % 8 || d_out > (1 << 24)) return MAXSCORE_ERR_UNSUPPORTED;
  if (!apart({weight_span(c, wq, d_in, d_out, 1), col_scales_span(c, w_scale, d_out)}, {weight_span(c, w, d_in, d_out, 2)})) return MAXSCORE_ERR_INVALID_ARG;
  if (w_layout == 1) return launch_rows8(c, w, nullptr, wq, w_scale, (int64_t)c->p.E * d_out, d_in, (cudaStream_t)stream);
  turn8_kernel<<<dim3((d_out + kTurnCols - 1) / kTurnCols, c->p.E), 256, 0, (cudaStream_t)stream>>>((const __nv_bfloat16*)w, wq, w_scale, d_in, d_out);
  MS_LAUNCH_CHECK("turn8_kernel");
  c->launches += 1;
  return MAXSCORE_OK;
}

maxscore_status maxscore_expert_gemm_q8(maxscore_ctx* c, const int8_t* xq, const float* x_scale, const int8_t* wq, const float* w_scale,
                                        const int32_t* expert_load, void* y, int32_t d_in, int32_t d_out, void* stream) {
  maxscore_status s = check8(c, {xq, x_scale, wq, w_scale, y}, d_in, d_out);
  if (s) return s;
  if (!expert_load) return MAXSCORE_ERR_INVALID_ARG;
  if (!width8(d_in) || d_out % 8 || d_out > (1 << 24)) return MAXSCORE_ERR_UNSUPPORTED;
  if (!apart({rows_span(c, y, d_out)}, {ints_span(c, xq, d_in), row_scales_span(c, x_scale), weight_span(c, wq, d_in, d_out, 1),
                                        col_scales_span(c, w_scale, d_out), load_span(c, expert_load)}))
    return MAXSCORE_ERR_INVALID_ARG;
  return launch_int8<kEpiPlain>(c, xq, x_scale, wq, w_scale, expert_load, y, d_in, d_out, (cudaStream_t)stream);
}

maxscore_status maxscore_expert_glu_q8(maxscore_ctx* c, const int8_t* xq, const float* x_scale, const int8_t* wq, const float* w_scale,
                                       const int32_t* expert_load, void* h, int32_t d_in, int32_t d_ff, void* stream) {
  maxscore_status s = check8(c, {xq, x_scale, wq, w_scale, h}, d_in, d_ff);
  if (s) return s;
  if (!expert_load) return MAXSCORE_ERR_INVALID_ARG;
  if (!width8(d_in) || d_ff % 8 || d_ff > (1 << 23)) return MAXSCORE_ERR_UNSUPPORTED;
  if (!apart({rows_span(c, h, d_ff)}, {ints_span(c, xq, d_in), row_scales_span(c, x_scale), weight_span(c, wq, d_in, 2 * (int64_t)d_ff, 1),
                                       col_scales_span(c, w_scale, 2 * (int64_t)d_ff), load_span(c, expert_load)}))
    return MAXSCORE_ERR_INVALID_ARG;
  return launch_int8<kEpiGlu>(c, xq, x_scale, wq, w_scale, expert_load, h, d_in, d_ff, (cudaStream_t)stream);
}

maxscore_status maxscore_keep8_bytes(const maxscore_ctx* c, int32_t d_ff, size_t* bytes) {
  if (!c || !bytes || d_ff <= 0) return MAXSCORE_ERR_INVALID_ARG;
  if (c->p.io_dtype != MAXSCORE_BF16 || d_ff % 8 || d_ff > (1 << 24)) return MAXSCORE_ERR_UNSUPPORTED;
  *bytes = keep_bytes(c, d_ff);
  return MAXSCORE_OK;
}

maxscore_status maxscore_expert_glu_keep8(maxscore_ctx* c, const void* x, const void* w_up, const int32_t* expert_load, void* keep, void* h,
                                          int32_t d_in, int32_t d_ff, int32_t w_layout, void* stream) {
  maxscore_status s = check_expert(c, {x, w_up, keep, h}, d_in, d_ff, d_in, w_layout);
  if (s) return s;
  if (c->p.io_dtype != MAXSCORE_BF16) return MAXSCORE_ERR_UNSUPPORTED;
  if (!expert_load || !aligned32(keep) ||
      !apart({rows_span(c, h, d_ff), {keep, keep_bytes(c, d_ff)}},
             {rows_span(c, x, d_in), weight_span(c, w_up, d_in, 2 * (int64_t)d_ff, 2), load_span(c, expert_load)}))
    return MAXSCORE_ERR_INVALID_ARG;
  const ExpertArgs a = keep_args(c, expert_load, d_ff, d_in, keep);
  cudaStream_t st = (cudaStream_t)stream;
  // Few rows against the 256-row tiles, us: the former while the weights' bytes count for more than what each row costs in the epilogue.
  // C 64: 248 -> 288 19 / 20, 1024 -> 512 11 / 12, 2048 -> 1024 90 / 102;  C 128: 32 / 20, 16 / 13, 102 / 110, 2320 -> 400 109 / 123.
  if (c->C <= 64 || (c->C <= kFewRows && d_in >= 2048))
    return w_layout == 0 ? launch_few<kEpiGlu, true, kKeep8>(c, x, w_up, h, nullptr, a, st) : launch_few<kEpiGlu, false, kKeep8>(c, x, w_up, h, nullptr, a, st);
  return w_layout == 0 ? launch_tc<kEpiGlu, true, kKeep8>(c, x, w_up, nullptr, h, nullptr, a, st)
                       : launch_tc<kEpiGlu, false, kKeep8>(c, x, w_up, nullptr, h, nullptr, a, st);
}

maxscore_status maxscore_expert_glu_bwd_keep8(maxscore_ctx* c, const void* dy, const void* w_down, const void* keep, const int32_t* expert_load,
                                              void* dpre, void* h, int32_t d_out, int32_t d_ff, int32_t w_layout, void* stream) {
  maxscore_status s = check_expert(c, {dy, w_down, keep, dpre}, d_out, d_ff, d_out, w_layout);
  if (s) return s;
  if (c->p.io_dtype != MAXSCORE_BF16) return MAXSCORE_ERR_UNSUPPORTED;
  if (!expert_load || !aligned32(keep) || !aligned16(h) ||
      !apart({rows_span(c, dpre, 2 * (int64_t)d_ff), rows_span(c, h, d_ff)},
             {rows_span(c, dy, d_out), weight_span(c, w_down, d_ff, d_out, 2), {keep, keep_bytes(c, d_ff)}, load_span(c, expert_load)}))
    return MAXSCORE_ERR_INVALID_ARG;
  const ExpertArgs a = keep_args(c, expert_load, d_ff, d_out, const_cast<void*>(keep));
  cudaStream_t st = (cudaStream_t)stream;
  // us, against the 256-row tiles, C 16: 248 -> 288 10 / 33, 1024 -> 512 8.5 / 17, 2048 -> 1024 51 / 67;  C 128: 36 / 39, 21 / 21, 89 / 91.
  if (c->C <= kFewRows)
    return w_layout == 1 ? launch_few<kEpiDact, true, kKeep8>(c, dy, w_down, dpre, h, a, st) : launch_few<kEpiDact, false, kKeep8>(c, dy, w_down, dpre, h, a, st);
  return w_layout == 1 ? launch_tc<kEpiDact, true, kKeep8>(c, dy, w_down, nullptr, dpre, h, a, st)
                       : launch_tc<kEpiDact, false, kKeep8>(c, dy, w_down, nullptr, dpre, h, a, st);
}

}  // extern "C"
