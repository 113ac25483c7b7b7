// C ABI of the experts between dispatch and combine and of the norms around a block (see include/maxscore.h): argument checks and
// kernel launches on the caller's stream.
#include <math.h>

#include <algorithm>
#include <initializer_list>
#include <type_traits>

#include "common.cuh"
#include "context.cuh"
#include "expert.cuh"
#include "expert_tc.cuh"
#include "expert_few.cuh"
#include "norm.cuh"

using namespace msr;

namespace {

constexpr int kNormRing = 210 * 1024;    // shared memory of an SM that the norms' row rings share

// One matrix per expert: [E][rows][inner] with given strides, boxes of one expert each, 128-byte swizzle.  chunks: the
// 64-column chunks are a dimension of their own and a box takes two of them (inner % 64 == 0).
maxscore_status make_tmap_expert(const maxscore_ctx* c, CUtensorMap* tm, const void* base, uint64_t inner, uint64_t rows,
                                 uint64_t row_stride, uint64_t expert_stride, uint32_t box_rows, bool chunks = false) {
  const uint64_t E = (uint64_t)c->p.E;
  cuuint64_t dims3[3] = {inner, rows, E}, dims4[4] = {64, rows, inner / 64, E};
  cuuint64_t strides3[2] = {row_stride * 2, expert_stride * 2}, strides4[3] = {row_stride * 2, 128, expert_stride * 2};
  cuuint32_t box3[3] = {64, box_rows, 1}, box4[4] = {64, box_rows, 2, 1};
  cuuint32_t estr[4] = {1, 1, 1, 1};
  CUresult r = c->encode(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, chunks ? 4 : 3, const_cast<void*>(base), chunks ? dims4 : dims3,
                         chunks ? strides4 : strides3, chunks ? box4 : box3, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                         CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) {
    snprintf(g_last_error, sizeof(g_last_error), "cuTensorMapEncodeTiled failed with CUresult %d", (int)r);
    return MAXSCORE_ERR_CUDA;
  }
  return MAXSCORE_OK;
}

// Asks for a kernel's shared memory on a context's first call of it: maxscore_create would have to load a hundred kernels for that,
// of which a router uses none (first context of a process 48 ms, 7 without).
template <typename K>
maxscore_status room_for(maxscore_ctx* c, K kernel, int bytes) {
  const void* key = reinterpret_cast<const void*>(kernel);
  for (int i = 0; i < c->n_roomy; ++i) if (c->roomy[i] == key) return MAXSCORE_OK;
  MS_CUDA(cudaFuncSetAttribute(key, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
  if (c->n_roomy < kRoomyMax) c->roomy[c->n_roomy++] = key;
  return MAXSCORE_OK;
}

// A caller's buffer.  Outputs must share no byte with an input or with one another.
struct Span { const void* p; size_t bytes; };
bool apart(std::initializer_list<Span> outs, std::initializer_list<Span> ins) {
  auto meet = [](const Span& a, const Span& b) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
    return a.p && b.p && (x < y ? y - x < a.bytes : x - y < b.bytes);
  };
  for (const Span* o = outs.begin(); o != outs.end(); ++o) {
    for (const Span* i = outs.begin(); i != o; ++i) if (meet(*o, *i)) return false;
    for (const Span& i : ins) if (meet(*o, i)) return false;
  }
  return true;
}
Span load_span(const maxscore_ctx* c, const int32_t* load) { return {load, sizeof(int32_t) * (size_t)c->p.E}; }
Span rows_span(const maxscore_ctx* c, const void* p, int64_t width) { return {p, (size_t)c->p.E * c->C * width * elem_bytes(c)}; }
Span weight_span(const maxscore_ctx* c, const void* p, int64_t d_in, int64_t d_out, size_t elem) { return {p, (size_t)c->p.E * d_in * d_out * elem}; }

// contracted: the width that is summed over (0: the rows are)
maxscore_status check_expert(const maxscore_ctx* c, std::initializer_list<const void*> ptrs, int32_t w0, int32_t w1, int32_t contracted,
                             int32_t w_layout) {
  if (!c) return MAXSCORE_ERR_INVALID_ARG;
  for (const void* p : ptrs) if (!p || !aligned16(p)) return MAXSCORE_ERR_INVALID_ARG;
  if (w0 <= 0 || w1 <= 0 || (w_layout != 0 && w_layout != 1)) return MAXSCORE_ERR_INVALID_ARG;
  const int m = c->p.io_dtype == MAXSCORE_BF16 ? 8 : 4;
  if (w0 % m || w1 % m || w0 > (1 << 24) || w1 > (1 << 24)) return MAXSCORE_ERR_UNSUPPORTED;
  // adding 16 products cuts off about two steps of a long sum's last bit: 2^18 terms lose 2e-3 of it, as much as a rounding to bf16
  if (c->p.io_dtype == MAXSCORE_BF16 && contracted > (1 << 18)) return MAXSCORE_ERR_UNSUPPORTED;
  return MAXSCORE_OK;
}

template <int EPI, bool A_MN, bool B_MN>
maxscore_status launch_fma(maxscore_ctx* c, const void* A, const void* B, const void* pre_in, void* out, void* pre_out,
                           const ExpertArgs& a, cudaStream_t st) {
  // 128 x 128 tiles where they give every SM two of them, else 64 x 64; tiles of 16 or 32 rows where an expert cannot have more
  // (a tile multiplies all of its rows, absent ones too: E 8, C 6, 952 -> 1120 56 us instead of 70, E 128, C 12, 168 -> 248 41
  // instead of 52)
  const long long rows = (long long)c->p.T * c->p.k, cols = (long long)a.N * (EPI == kEpiGlu ? 2 : 1);
  auto tiles = [&](int m, int n) {
    return (EPI == kEpiDw ? (long long)a.E * ((a.M + m - 1) / m) : (rows + m - 1) / m) * ((cols + n - 1) / n);
  };
  auto go = [&](auto kernel, int per_sm) {
    kernel<<<c->sm_count * per_sm, 256, 0, st>>>((const float*)A, (const float*)B, (const float*)pre_in, (float*)out, (float*)pre_out, a);
  };
  auto by_tiles = [&] {
    if (tiles(128, 128) >= 2 * c->sm_count) go(expert_fma_kernel<128, 128, 16, EPI, A_MN, B_MN>, 2);
    else go(expert_fma_kernel<64, 64, 16, EPI, A_MN, B_MN>, 4);
  };
  if constexpr (EPI == kEpiDw) by_tiles();                             // its tiles are of the weight, whatever the rows
  else if (c->C <= 16) go(expert_fma_kernel<16, 64, 32, EPI, A_MN, B_MN>, 4);
  else if (c->C <= 32) go(expert_fma_kernel<32, 64, 32, EPI, A_MN, B_MN>, 4);
  else by_tiles();
  MS_LAUNCH_CHECK("expert_fma_kernel");
  c->launches += 1;
  return MAXSCORE_OK;
}

template <int EPI, bool B_MN>
maxscore_status launch_tc(maxscore_ctx* c, const void* A, const void* B, const void* pre_in, void* out, void* pre_out,
                          ExpertArgs a, cudaStream_t st) {
  constexpr bool kDw = EPI == kEpiDw;
  a.a_chunks = kDw && a.M % 64 == 0;
  a.b_chunks = B_MN && a.N % 64 == 0;
  const uint64_t C = (uint64_t)c->C, M = (uint64_t)a.M, N = (uint64_t)a.N, K = (uint64_t)a.K;
  typedef const __nv_bfloat16* P;
  CUtensorMap tA, tB0, tB1, tO0, tO1, tO2;
  maxscore_status s;
#define MS_MAP(...) do { s = make_tmap_expert(c, __VA_ARGS__); if (s) return s; } while (0)
  if (kDw) {
    MS_MAP(&tA, A, M, C, M, C * M, 64, a.a_chunks);
    MS_MAP(&tB0, B, N, C, N, C * N, 64, a.b_chunks);
    tB1 = tB0;
  } else {
    MS_MAP(&tA, A, K, C, K, C * K, 128);
    const uint64_t cols = EPI == kEpiGlu ? 2 * N : N;
    if (B_MN) MS_MAP(&tB0, B, N, K, cols, K * cols, 64, a.b_chunks);
    else MS_MAP(&tB0, B, K, N, K, cols * K, 128);
    tB1 = tB0;
    if (EPI == kEpiGlu) {
      if (B_MN) MS_MAP(&tB1, (P)B + N, N, K, cols, K * cols, 64, a.b_chunks);
      else MS_MAP(&tB1, (P)B + N * K, K, N, K, cols * K, 128);
    }
    if (EPI != kEpiDact) MS_MAP(&tO0, out, N, C, N, C * N, 32);
    if (EPI == kEpiGlu && pre_out) {
      MS_MAP(&tO1, pre_out, N, C, 2 * N, C * 2 * N, 32);
      MS_MAP(&tO2, (P)pre_out + N, N, C, 2 * N, C * 2 * N, 32);
    }
  }
#undef MS_MAP
  if (kDw || EPI == kEpiDact) tO0 = tA;                  // not used
  if (EPI != kEpiGlu || !pre_out) tO1 = tO2 = tO0;       // not used
  const long long tile_n = EPI == kEpiGlu ? 128 : kXTile;
  const long long tiles = (long long)a.E * (((kDw ? M : C) + kXTile - 1) / kXTile) * ((N + tile_n - 1) / tile_n);
  const int pairs = (int)std::min<long long>(c->sm_count / 2, tiles);
  auto go = [&](auto kernel, int w) {
    s = room_for(c, kernel, x_smem(EPI, w));
    if (!s) kernel<<<2 * pairs, x_threads(EPI), x_smem(EPI, w), st>>>(tA, tB0, tB1, tO0, tO1, tO2, (char*)out, (char*)pre_out, (const char*)pre_in, a, error_flag_of(c));
  };
  // Two column tiles at a time read a quarter less per flop, but their epilogues hide less well.  Long runs, 256 x 512 against
  // 256 x 256: y at C 4096, K 4096 1 248 / 1 234 TFLOP/s, at C 1024, K 2048 1 150 / 1 145, K 1024 1 041 / 1 055, K 512 853 / 904;
  // h 1 286 / 1 257 at K 4096, 1 125 / 1 178 at K 2048.  dW takes them where one accumulator holds its sum (E 64, C 128, 2048 x 1024:
  // 112 us / 136 us); the backward of the activation loses at every size (1 022 / 1 058 at K 4096, 561 / 705 at 1024).
  if constexpr (kDw) {
    if (a.C <= kXPartRows) { if (a.accumulate) go(expert_tc_kernel<EPI, B_MN, 2, true>, 2); else go(expert_tc_kernel<EPI, B_MN, 2>, 2); }
    else if (a.accumulate) go(expert_tc_kernel<EPI, B_MN, 1, true>, 1);
    else go(expert_tc_kernel<EPI, B_MN, 1>, 1);
  }
  else if constexpr (EPI == kEpiDact) go(expert_tc_kernel<EPI, B_MN, 1>, 1);
  else if (a.K >= 4096 && tiles >= 4 * pairs) go(expert_tc_kernel<EPI, B_MN, 2>, 2);
  else go(expert_tc_kernel<EPI, B_MN, 1>, 1);
  if (s) return s;
  MS_LAUNCH_CHECK("expert_tc_kernel");
  c->launches += 1;
  return MAXSCORE_OK;
}

template <int EPI, bool B_MN>
maxscore_status launch_few(maxscore_ctx* c, const void* x, const void* w, void* out, void* pre_out, ExpertArgs a, cudaStream_t st) {
  const uint64_t C = (uint64_t)c->C, N = (uint64_t)a.N, K = (uint64_t)a.K, cols = EPI == kEpiGlu ? 2 * N : N;
  const int pad = few_pad(c->C);
  typedef const __nv_bfloat16* P;
  CUtensorMap tW0, tW1, tX;
  maxscore_status s;
  a.b_chunks = EPI == kEpiPlain && B_MN && N % 64 == 0;
  s = make_tmap_expert(c, &tX, x, K, C, K, C * K, (uint32_t)pad);
  if (s) return s;
  const uint32_t box = B_MN || EPI == kEpiGlu ? 64 : 128;
  s = B_MN ? make_tmap_expert(c, &tW0, w, N, K, cols, K * cols, box, a.b_chunks) : make_tmap_expert(c, &tW0, w, K, N, K, cols * K, box);
  if (s) return s;
  tW1 = tW0;
  if (EPI == kEpiGlu) {
    s = B_MN ? make_tmap_expert(c, &tW1, (P)w + N, N, K, cols, K * cols, box) : make_tmap_expert(c, &tW1, (P)w + N * K, K, N, K, cols * K, box);
    if (s) return s;
  }
  const long long items = (long long)a.E * ((a.N + (EPI == kEpiGlu ? 63 : 127)) / (EPI == kEpiGlu ? 64 : 128));
  const int grid = (int)std::min<long long>(c->sm_count, items);
  s = room_for(c, expert_few_kernel<EPI, B_MN>, few_smem(EPI, kFewRows));
  if (s) return s;
  expert_few_kernel<EPI, B_MN><<<grid, kFewThreads, few_smem(EPI, pad), st>>>(tW0, tW1, tX, (__nv_bfloat16*)out, (__nv_bfloat16*)pre_out, a, pad,
                                                                             error_flag_of(c));
  MS_LAUNCH_CHECK("expert_few_kernel");
  c->launches += 1;
  return MAXSCORE_OK;
}

// b_mn: the product's columns (N) run along memory in B
template <int EPI>
maxscore_status launch_expert(maxscore_ctx* c, const void* A, const void* B, const void* pre_in, void* out, void* pre_out,
                              const ExpertArgs& a, bool b_mn, cudaStream_t st) {
  if (c->p.io_dtype == MAXSCORE_BF16) {
    if constexpr (EPI == kEpiPlain || EPI == kEpiGlu)
      if (c->C <= kFewRows)
        return b_mn ? launch_few<EPI, true>(c, A, B, out, pre_out, a, st) : launch_few<EPI, false>(c, A, B, out, pre_out, a, st);
    if constexpr (EPI == kEpiDw) return launch_tc<EPI, true>(c, A, B, pre_in, out, pre_out, a, st);
    else return b_mn ? launch_tc<EPI, true>(c, A, B, pre_in, out, pre_out, a, st)
                     : launch_tc<EPI, false>(c, A, B, pre_in, out, pre_out, a, st);
  }
  if constexpr (EPI == kEpiDw) return launch_fma<EPI, true, true>(c, A, B, pre_in, out, pre_out, a, st);
  else return b_mn ? launch_fma<EPI, false, true>(c, A, B, pre_in, out, pre_out, a, st)
                   : launch_fma<EPI, false, false>(c, A, B, pre_in, out, pre_out, a, st);
}

ExpertArgs expert_args(const maxscore_ctx* c, const int32_t* load, int M, int N, int K, int accumulate = 0) {
  ExpertArgs a{};
  a.load = load; a.E = c->p.E; a.C = c->C; a.M = M; a.N = N; a.K = K; a.accumulate = accumulate;
  return a;
}

// `y`: whether the call has a block output
maxscore_status check_norm(const maxscore_ctx* c, const maxscore_norm* n, bool y) {
  if (!c || !n) return MAXSCORE_ERR_INVALID_ARG;
  if (!aligned16(n->w_post) || !aligned16(n->gate) || !aligned16(n->w_pre)) return MAXSCORE_ERR_INVALID_ARG;
  if (!(n->eps > 0.f) || !isfinite(n->eps) || !isfinite(n->w_offset) || !isfinite(n->res_scale)) return MAXSCORE_ERR_INVALID_ARG;
  if (n->gate && n->rows_per_gate <= 0) return MAXSCORE_ERR_INVALID_ARG;
  if (!y && (n->w_post || n->gate)) return MAXSCORE_ERR_INVALID_ARG;
  if ((size_t)c->p.d_model * elem_bytes(c) > 32768) return MAXSCORE_ERR_UNSUPPORTED;
  return MAXSCORE_OK;
}

struct NormSpans {
  size_t token, d;                         // bytes of [T, d_model] in io_dtype, and of [d_model]
  Span w_post, gate, w_pre;
  size_t gate_rows;
};
NormSpans norm_spans(const maxscore_ctx* c, const maxscore_norm* n) {
  NormSpans s{};
  s.d = (size_t)c->p.d_model * elem_bytes(c); s.token = s.d * c->p.T;
  s.gate_rows = n->gate ? ((size_t)c->p.T + n->rows_per_gate - 1) / n->rows_per_gate : 0;
  s.w_post = {n->w_post, s.d}; s.gate = {n->gate, s.gate_rows * s.d}; s.w_pre = {n->w_pre, s.d};
  return s;
}

NormArgs norm_args(const maxscore_ctx* c, const maxscore_norm* n) {
  NormArgs a{};
  a.T = c->p.T; a.d = c->p.d_model; a.nvec = (int)(c->p.d_model * elem_bytes(c) / 16);
  a.rows_per_gate = n->gate && n->rows_per_gate < c->p.T ? n->rows_per_gate : c->p.T;
  a.eps = n->eps; a.w_offset = n->w_offset; a.res_scale = n->res_scale;
  a.w_post = n->w_post; a.gate = n->gate; a.w_pre = n->w_pre;
  return a;
}

// How a row of nvec 16-byte vectors is worked on: V vectors a thread, G threads, CTAs of an SM, and the ring of slots (of
// `rows` row buffers each) that a CTA's share of shared memory holds.
struct NormShape { int V, G, ctas, slots; size_t smem; bool full; };
NormShape norm_shape(int nvec, bool bwd, bool gathers, int rows) {
  NormShape s{};
  s.V = bwd ? norm_bwd_vecs(nvec) : nvec <= 1024 ? 2 : 4;
  s.G = norm_threads(nvec, s.V);
  s.ctas = bwd ? norm_bwd_ctas(nvec) : norm_ctas(s.G);
  s.full = nvec == s.V * s.G;
  // How much to have in flight matters more than how much fits: with 210 KB of rows on their way per SM reads and writes get in
  // each other's way (combine and norms at T 65536, d 4096, k 8: 1 018 us; 105 KB 926 us, 70 KB 977 us, 52 KB 1 049 us; without
  // combine 387, 379, 355, 378 us).  Two slots at least where they fit, or nothing runs ahead (only the backward of four given rows of
  // more than 26 KB has a single one).
  const size_t slot = (size_t)nvec * 16 * rows, share = kNormRing / s.ctas - sizeof(NormSmem);
  const size_t wanted = (size_t)kNormRing / (gathers ? 2 : 3) / s.ctas / slot;
  s.slots = (int)std::min<size_t>({kNormSlots, share / slot, std::max<size_t>(2, wanted)});
  s.smem = s.slots * slot;
  return s;
}

template <typename T, int SRC>
maxscore_status launch_norm_fwd(maxscore_ctx* c, const void* y_in, const void* src, const int32_t* expert_idx, const int32_t* slot_idx,
                                const float* gate_w, const void* residual, const maxscore_norm* n, void* y_out, void* r_out, void* h,
                                cudaStream_t st) {
  const maxscore_params& p = c->p;
  const NormArgs a = norm_args(c, n);
  const NormShape f = norm_shape(a.nvec, false, SRC == 2, SRC == 1 ? 2 : 1);
  const int grid = std::min(p.T, c->sm_count * f.ctas);
  maxscore_status s = MAXSCORE_OK;
  auto go = [&](auto kernel) {
    s = room_for(c, kernel, kNormRing / f.ctas);
    if (!s) kernel<<<grid, f.G + 32, f.smem, st>>>((const T*)y_in, (const T*)src, expert_idx, slot_idx, gate_w, p.E, p.k, c->C, (const T*)residual,
                                           (T*)y_out, (T*)r_out, (T*)h, a, f.slots, error_flag_of(c));
  };
  auto pick = [&](auto full) {
    constexpr bool F = decltype(full)::value;
    if (f.G > 256) go(norm_fwd_kernel<T, 2, SRC, F, 512, 1>);
    else if (f.G > 128) go(norm_fwd_kernel<T, 2, SRC, F, 256, 2>);
    else if (f.G > 64) go(norm_fwd_kernel<T, 2, SRC, F, 128, 4>);
    else go(norm_fwd_kernel<T, 2, SRC, F, 64, 8>);
  };
  // Threads that know that their vectors are exactly the row, against threads that compare, us: behind combine, k 8, T 32768, fp32,
  // d 4096 939 / 1 000, d 1024 233 / 252, bf16 at T 65536, d 4096 930 / 938, T 8192, d 16384 623 / 665; four vectors a thread with y
  // given 275 / 291.  With two vectors and y given, or without y, it makes no difference or loses (T 65536, d 1024: 101 / 99).
  if (f.V == 4 && SRC > 0 && f.full) { if constexpr (SRC > 0) go(norm_fwd_kernel<T, 4, SRC, true, 512, 1>); }
  else if (f.V == 4) go(norm_fwd_kernel<T, 4, SRC, false, 512, 1>);
  else if (SRC == 2 && f.full) { if constexpr (SRC == 2) pick(std::true_type{}); }
  else pick(std::false_type{});
  if (s) return s;
  MS_LAUNCH_CHECK("norm_fwd_kernel");
  c->launches += 1;
  return MAXSCORE_OK;
}

template <typename T>
maxscore_status launch_norm_bwd(maxscore_ctx* c, const void* dr_out, const void* dh, const void* y, const void* r_out,
                                const maxscore_norm* n, void* dy, void* dr, float* dw_post, float* dgate, float* dw_pre,
                                cudaStream_t st) {
  const maxscore_params& p = c->p;
  const NormArgs a = norm_args(c, n);
  const NormShape f = norm_shape(a.nvec, true, false, std::max(1, (dh ? 2 : 0) + (y ? 1 : 0) + (dr_out ? 1 : 0)));
  const int parts = norm_parts(p);                                   // rows of each partial matrix in the workspace
  const int ctas = std::min(parts, c->sm_count * f.ctas);
  const int gate_rows = (p.T + a.rows_per_gate - 1) / a.rows_per_gate;
  NormUnits u{};
  u.per_gate = std::max(1, std::min(a.rows_per_gate, ctas / gate_rows));
  u.rows = (a.rows_per_gate + u.per_gate - 1) / u.per_gate;
  u.n_units = gate_rows * u.per_gate;                                // at most `ctas` whenever per_gate > 1
  const int grid = std::min(u.n_units, ctas);
  float* part = reinterpret_cast<float*>(c->ws + c->lay.normpart);
  const size_t one = (size_t)parts * p.d_model;
  float* pp = n->w_post ? part : nullptr;
  float* pr = n->w_pre ? part + one : nullptr;
  float* pg = !n->gate ? nullptr : u.per_gate > 1 ? part + 2 * one : dgate;
  maxscore_status s = MAXSCORE_OK;
  auto go = [&](auto kernel) {
    s = room_for(c, kernel, kNormRing / f.ctas);
    if (!s) kernel<<<grid, f.G + 32, f.smem, st>>>((const T*)dr_out, (const T*)dh, (const T*)y, (const T*)r_out, (T*)dy, (T*)dr, pp, pr, pg, u, a, f.slots,
                                           error_flag_of(c));
  };
  // exactly the row or compared (see above): bf16, d 8192 1 046 / 1 124 us, d 16384 1 322 / 1 332; no difference with one vector a thread
  if (f.V == 4) { if (f.full) go(norm_bwd_kernel<T, 4, true, 512, 1>); else go(norm_bwd_kernel<T, 4, false, 512, 1>); }
  else if (f.V == 2) { if (f.full) go(norm_bwd_kernel<T, 2, true, 512, 1>); else go(norm_bwd_kernel<T, 2, false, 512, 1>); }
  else if (f.G > 256) go(norm_bwd_kernel<T, 1, false, 512, 1>);
  else if (f.G > 128) go(norm_bwd_kernel<T, 1, false, 256, 2>);
  else if (f.G > 64) go(norm_bwd_kernel<T, 1, false, 128, 4>);
  else go(norm_bwd_kernel<T, 1, false, 64, 8>);
  if (s) return s;
  MS_LAUNCH_CHECK("norm_bwd_kernel");
  c->launches += 1;
  const bool reduce_gate = n->gate && u.per_gate > 1;
  if (n->w_post || n->w_pre || reduce_gate) {
    norm_reduce_kernel<<<dim3((p.d_model + 31) / 32, 2 + (reduce_gate ? gate_rows : 0)), kNormReduceWarps * 32, 0, st>>>(
        pp, pr, pg, dw_post, dw_pre, dgate, grid, u.per_gate, p.d_model);
    MS_LAUNCH_CHECK("norm_reduce_kernel");
    c->launches += 1;
  }
  return MAXSCORE_OK;
}

}  // namespace

extern "C" {

maxscore_status maxscore_expert_gemm(maxscore_ctx* c, const void* x, const void* w, const int32_t* expert_load, void* y,
                                     int32_t d_in, int32_t d_out, int32_t w_layout, void* stream) {
  maxscore_status s = check_expert(c, {x, w, y}, d_in, d_out, d_in, w_layout);
  if (s) return s;
  if (!expert_load || !apart({rows_span(c, y, d_out)}, {rows_span(c, x, d_in), weight_span(c, w, d_in, d_out, elem_bytes(c)), load_span(c, expert_load)}))
    return MAXSCORE_ERR_INVALID_ARG;
  return launch_expert<kEpiPlain>(c, x, w, nullptr, y, nullptr, expert_args(c, expert_load, 0, d_out, d_in), w_layout == 0,
                                  (cudaStream_t)stream);
}

maxscore_status maxscore_expert_gemm_dw(maxscore_ctx* c, const void* x, const void* dy, const int32_t* expert_load, float* dw,
                                        int32_t d_in, int32_t d_out, int32_t w_layout, int accumulate, void* stream) {
  maxscore_status s = check_expert(c, {x, dy, dw}, d_in, d_out, 0, w_layout);
  if (s) return s;
  if (!expert_load || !apart({weight_span(c, dw, d_in, d_out, sizeof(float))}, {rows_span(c, x, d_in), rows_span(c, dy, d_out), load_span(c, expert_load)}))
    return MAXSCORE_ERR_INVALID_ARG;
  // layout 1 is the transposed product: the two operands change places
  const bool t = w_layout == 1;
  return launch_expert<kEpiDw>(c, t ? dy : x, t ? x : dy, nullptr, dw, nullptr,
                               expert_args(c, expert_load, t ? d_out : d_in, t ? d_in : d_out, 0, accumulate != 0), true,
                               (cudaStream_t)stream);
}

maxscore_status maxscore_expert_glu(maxscore_ctx* c, const void* x, const void* w_up, const int32_t* expert_load, void* pre,
                                    void* h, int32_t d_in, int32_t d_ff, int32_t w_layout, void* stream) {
  maxscore_status s = check_expert(c, {x, w_up, h}, d_in, d_ff, d_in, w_layout);
  if (s) return s;
  if (!expert_load || !aligned16(pre) ||
      !apart({rows_span(c, h, d_ff), rows_span(c, pre, 2 * (int64_t)d_ff)},
             {rows_span(c, x, d_in), weight_span(c, w_up, d_in, 2 * (int64_t)d_ff, elem_bytes(c)), load_span(c, expert_load)}))
    return MAXSCORE_ERR_INVALID_ARG;
  return launch_expert<kEpiGlu>(c, x, w_up, nullptr, h, pre, expert_args(c, expert_load, 0, d_ff, d_in), w_layout == 0,
                                (cudaStream_t)stream);
}

maxscore_status maxscore_expert_glu_bwd(maxscore_ctx* c, const void* dy, const void* w_down, const void* pre,
                                        const int32_t* expert_load, void* dpre, int32_t d_out, int32_t d_ff, int32_t w_layout,
                                        void* stream) {
  maxscore_status s = check_expert(c, {dy, w_down, pre, dpre}, d_out, d_ff, d_out, w_layout);
  if (s) return s;
  if (!expert_load || !apart({rows_span(c, dpre, 2 * (int64_t)d_ff)}, {rows_span(c, dy, d_out), weight_span(c, w_down, d_ff, d_out, elem_bytes(c)),
                                                                         rows_span(c, pre, 2 * (int64_t)d_ff), load_span(c, expert_load)}))
    return MAXSCORE_ERR_INVALID_ARG;
  // dh = dy . W_down^T: the weight's d_ff side is the product's N side, contiguous in layout 1 ([E, d_out, d_ff])
  return launch_expert<kEpiDact>(c, dy, w_down, pre, dpre, nullptr, expert_args(c, expert_load, 0, d_ff, d_out), w_layout == 1,
                                 (cudaStream_t)stream);
}

maxscore_status maxscore_combine_norm(maxscore_ctx* c, const void* src, const int32_t* expert_idx, const int32_t* slot_idx,
                                      const float* gate_w, const void* residual, const maxscore_norm* n, void* y, void* r_out,
                                      void* h, void* stream) {
  maxscore_status s = check_norm(c, n, true);
  if (s) return s;
  if (!src || !expert_idx || !slot_idx || !residual || !r_out || (h == nullptr) != (n->w_pre == nullptr)) return MAXSCORE_ERR_INVALID_ARG;
  for (const void* p : {src, residual, (const void*)y, (const void*)r_out, (const void*)h})
    if (!aligned16(p)) return MAXSCORE_ERR_INVALID_ARG;
  const NormSpans sp = norm_spans(c, n);
  const size_t pairs = sizeof(int32_t) * (size_t)c->p.T * c->p.k;
  if (!apart({{y, sp.token}, {r_out, sp.token}, {h, sp.token}},
             {rows_span(c, src, c->p.d_model), {expert_idx, pairs}, {slot_idx, pairs}, {gate_w, pairs}, {r_out == residual ? nullptr : residual, sp.token},
              sp.w_post, sp.gate, sp.w_pre}))
    return MAXSCORE_ERR_INVALID_ARG;
  if (c->p.io_dtype == MAXSCORE_BF16)
    return launch_norm_fwd<__nv_bfloat16, 2>(c, nullptr, src, expert_idx, slot_idx, gate_w, residual, n, y, r_out, h, (cudaStream_t)stream);
  return launch_norm_fwd<float, 2>(c, nullptr, src, expert_idx, slot_idx, gate_w, residual, n, y, r_out, h, (cudaStream_t)stream);
}

maxscore_status maxscore_block_norm(maxscore_ctx* c, const void* y, const void* residual, const maxscore_norm* n, void* r_out,
                                    void* h, void* stream) {
  maxscore_status s = check_norm(c, n, y != nullptr);
  if (s) return s;
  if (!residual || (!r_out && !h) || (h == nullptr) != (n->w_pre == nullptr)) return MAXSCORE_ERR_INVALID_ARG;
  for (const void* p : {y, residual, (const void*)r_out, (const void*)h})
    if (!aligned16(p)) return MAXSCORE_ERR_INVALID_ARG;
  const NormSpans sp = norm_spans(c, n);
  if (!apart({{r_out, sp.token}, {h, sp.token}}, {{y, sp.token}, {r_out == residual ? nullptr : residual, sp.token}, sp.w_post, sp.gate, sp.w_pre}))
    return MAXSCORE_ERR_INVALID_ARG;
  const bool bf = c->p.io_dtype == MAXSCORE_BF16;
  cudaStream_t st = (cudaStream_t)stream;
  if (y)
    return bf ? launch_norm_fwd<__nv_bfloat16, 1>(c, y, nullptr, nullptr, nullptr, nullptr, residual, n, nullptr, r_out, h, st)
              : launch_norm_fwd<float, 1>(c, y, nullptr, nullptr, nullptr, nullptr, residual, n, nullptr, r_out, h, st);
  return bf ? launch_norm_fwd<__nv_bfloat16, 0>(c, nullptr, nullptr, nullptr, nullptr, nullptr, residual, n, nullptr, r_out, h, st)
            : launch_norm_fwd<float, 0>(c, nullptr, nullptr, nullptr, nullptr, nullptr, residual, n, nullptr, r_out, h, st);
}

maxscore_status maxscore_block_norm_bwd(maxscore_ctx* c, const void* dr_out, const void* dh, const void* y, const void* r_out,
                                        const maxscore_norm* n, void* dy, void* dr, float* dw_post, float* dgate, float* dw_pre,
                                        void* stream) {
  maxscore_status s = check_norm(c, n, y != nullptr);
  if (s) return s;
  if (!dr || (dy == nullptr) != (y == nullptr) || (dh == nullptr) != (n->w_pre == nullptr) || (n->w_pre && !r_out) ||
      (dw_post == nullptr) != (n->w_post == nullptr) || (dgate == nullptr) != (n->gate == nullptr) ||
      (dw_pre == nullptr) != (n->w_pre == nullptr))
    return MAXSCORE_ERR_INVALID_ARG;
  for (const void* p : {dr_out, dh, y, r_out, (const void*)dy, (const void*)dr, (const void*)dw_post, (const void*)dgate, (const void*)dw_pre})
    if (!aligned16(p)) return MAXSCORE_ERR_INVALID_ARG;
  const NormSpans sp = norm_spans(c, n);
  const size_t col = sizeof(float) * (size_t)c->p.d_model;
  if (!apart({{dy, sp.token}, {dr, sp.token}, {dw_post, col}, {dgate, sp.gate_rows * col}, {dw_pre, col}},
             {{dr == dr_out ? nullptr : dr_out, sp.token}, {dh, sp.token}, {y, sp.token}, {r_out, sp.token}, sp.w_post, sp.gate, sp.w_pre}))
    return MAXSCORE_ERR_INVALID_ARG;
  if (c->p.io_dtype == MAXSCORE_BF16)
    return launch_norm_bwd<__nv_bfloat16>(c, dr_out, dh, y, r_out, n, dy, dr, dw_post, dgate, dw_pre, (cudaStream_t)stream);
  return launch_norm_bwd<float>(c, dr_out, dh, y, r_out, n, dy, dr, dw_post, dgate, dw_pre, (cudaStream_t)stream);
}

}  // extern "C"
