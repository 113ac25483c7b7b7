// Checks and launches of the tensor-core expert products that the C entry points share: maps of the operands, choice of the tile.
#pragma once
#include <algorithm>

#include "common.cuh"
#include "context.cuh"
#include "expert.cuh"
#include "expert_tc.cuh"
#include "expert_few.cuh"

namespace msr {

// One matrix per expert: [E][rows][inner] with given strides, boxes of one expert each, 128-byte swizzle.  chunks: the
// 64-column chunks are a dimension of their own and a box takes two of them (inner % 64 == 0).  elem: 2 for bf16, 1 for bytes.
inline maxscore_status make_tmap_expert(const maxscore_ctx* c, CUtensorMap* tm, const void* base, uint64_t inner, uint64_t rows,
                                 uint64_t row_stride, uint64_t expert_stride, uint32_t box_rows, bool chunks = false, uint64_t elem = 2) {
  const uint64_t E = (uint64_t)c->p.E;
  cuuint64_t dims3[3] = {inner, rows, E}, dims4[4] = {64, rows, inner / 64, E};
  cuuint64_t strides3[2] = {row_stride * elem, expert_stride * elem}, strides4[3] = {row_stride * 2, 128, expert_stride * 2};
  cuuint32_t box3[3] = {(cuuint32_t)(128 / elem), box_rows, 1}, box4[4] = {64, box_rows, 2, 1};
  cuuint32_t estr[4] = {1, 1, 1, 1};
  CUresult r = c->encode(tm, elem == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, chunks ? 4 : 3, const_cast<void*>(base), chunks ? dims4 : dims3,
                         chunks ? strides4 : strides3, chunks ? box4 : box3, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                         CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) {
    snprintf(g_last_error, sizeof(g_last_error), "cuTensorMapEncodeTiled failed with CUresult %d", (int)r);
    return MAXSCORE_ERR_CUDA;
  }
  return MAXSCORE_OK;
}

inline Span load_span(const maxscore_ctx* c, const int32_t* load) { return {load, sizeof(int32_t) * (size_t)c->p.E}; }
inline Span rows_span(const maxscore_ctx* c, const void* p, int64_t width) { return {p, (size_t)c->p.E * c->C * width * elem_bytes(c)}; }
inline Span weight_span(const maxscore_ctx* c, const void* p, int64_t d_in, int64_t d_out, size_t elem) { return {p, (size_t)c->p.E * d_in * d_out * elem}; }

// contracted: the width that is summed over (0: the rows are)
inline maxscore_status check_expert(const maxscore_ctx* c, std::initializer_list<const void*> ptrs, int32_t w0, int32_t w1, int32_t contracted,
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

template <int EPI, bool B_MN, int Form = kBf16>
maxscore_status launch_tc(maxscore_ctx* c, const void* A, const void* B, const void* pre_in, void* out, void* pre_out,
                          ExpertArgs a, cudaStream_t st) {
  constexpr bool kDw = EPI == kEpiDw;
  a.a_chunks = kDw && a.M % 64 == 0;
  a.b_chunks = B_MN && a.N % 64 == 0;
  const uint64_t C = (uint64_t)c->C, M = (uint64_t)a.M, N = (uint64_t)a.N, K = (uint64_t)a.K;
  constexpr uint64_t elem = Form == kInt8 ? 1 : 2;
  typedef const __nv_bfloat16* P;
  CUtensorMap tA, tB0, tB1, tO0, tO1, tO2;
  maxscore_status s;
#define MS_MAP(...) do { s = make_tmap_expert(c, __VA_ARGS__); if (s) return s; } while (0)
  if (kDw) {
    MS_MAP(&tA, A, M, C, M, C * M, 64, a.a_chunks);
    MS_MAP(&tB0, B, N, C, N, C * N, 64, a.b_chunks);
    tB1 = tB0;
  } else {
    MS_MAP(&tA, A, K, C, K, C * K, 128, false, elem);
    const uint64_t cols = EPI == kEpiGlu ? 2 * N : N;
    if (B_MN) MS_MAP(&tB0, B, N, K, cols, K * cols, 64, a.b_chunks);
    else MS_MAP(&tB0, B, K, N, K, cols * K, 128, false, elem);
    tB1 = tB0;
    if (EPI == kEpiGlu) {
      if (B_MN) MS_MAP(&tB1, (P)B + N, N, K, cols, K * cols, 64, a.b_chunks);
      else MS_MAP(&tB1, (const char*)B + N * K * elem, K, N, K, cols * K, 128, false, elem);
    }
    if (EPI != kEpiDact) MS_MAP(&tO0, out, N, C, N, C * N, 32);
    if (EPI == kEpiGlu && Form == kBf16 && pre_out) {
      MS_MAP(&tO1, pre_out, N, C, 2 * N, C * 2 * N, 32);
      MS_MAP(&tO2, (P)pre_out + N, N, C, 2 * N, C * 2 * N, 32);
    }
  }
#undef MS_MAP
  if (kDw || EPI == kEpiDact) tO0 = tA;                  // not used
  if (EPI != kEpiGlu || Form != kBf16 || !pre_out) tO1 = tO2 = tO0;       // not used
  const long long tile_n = EPI == kEpiGlu ? 128 : kXTile;
  const long long tiles = (long long)a.E * (((kDw ? M : C) + kXTile - 1) / kXTile) * ((N + tile_n - 1) / tile_n);
  const int pairs = (int)std::min<long long>(c->sm_count / 2, tiles);
  auto go = [&](auto kernel, int w) {
    s = room_for(c, kernel, x_smem(EPI, w, Form));
    if (!s) kernel<<<2 * pairs, x_threads(EPI), x_smem(EPI, w, Form), st>>>(tA, tB0, tB1, tO0, tO1, tO2, (char*)out, (char*)pre_out, (const char*)pre_in, a, error_flag_of(c));
  };
  // Two column tiles at a time read a quarter less per flop, but their epilogues hide less well.  Long runs, 256 x 512 against
  // 256 x 256: y at C 4096, K 4096 1 248 / 1 234 TFLOP/s, at C 1024, K 2048 1 150 / 1 145, K 1024 1 041 / 1 055, K 512 853 / 904;
  // h 1 286 / 1 257 at K 4096, 1 125 / 1 178 at K 2048.  dW takes them where one accumulator holds its sum (E 64, C 128, 2048 x 1024:
  // 112 us / 136 us).  Integers, twice as fast on the same slices, never gain (TOPS, h: 2 612 / 2 812 at K 4096, 2 071 / 2 622 at 2048; y: 1 912 / 2 154
  // at K 1024).  The backward of the activation loses at every size (1 022 / 1 058 at K 4096, 561 / 705 at 1024).
  if constexpr (kDw) {
    if (a.C <= kXPartRows) { if (a.accumulate) go(expert_tc_kernel<EPI, B_MN, 2, true>, 2); else go(expert_tc_kernel<EPI, B_MN, 2>, 2); }
    else if (a.accumulate) go(expert_tc_kernel<EPI, B_MN, 1, true>, 1);
    else go(expert_tc_kernel<EPI, B_MN, 1>, 1);
  }
  else if constexpr (EPI == kEpiDact || Form == kInt8) go(expert_tc_kernel<EPI, B_MN, 1, false, Form>, 1);
  else if (a.K >= 4096 && tiles >= 4 * pairs) go(expert_tc_kernel<EPI, B_MN, 2, false, Form>, 2);
  else go(expert_tc_kernel<EPI, B_MN, 1, false, Form>, 1);
  if (s) return s;
  MS_LAUNCH_CHECK("expert_tc_kernel");
  c->launches += 1;
  return MAXSCORE_OK;
}

template <int EPI, bool B_MN, int Form = kBf16>
maxscore_status launch_few(maxscore_ctx* c, const void* x, const void* w, void* out, void* pre_out, ExpertArgs a, cudaStream_t st) {
  const uint64_t C = (uint64_t)c->C, N = (uint64_t)a.N, K = (uint64_t)a.K, cols = EPI == kEpiGlu ? 2 * N : N;
  const int pad = few_pad(c->C);
  constexpr uint64_t elem = Form == kInt8 ? 1 : 2;
  typedef const __nv_bfloat16* P;
  CUtensorMap tW0, tW1, tX;
  maxscore_status s;
  a.b_chunks = EPI != kEpiGlu && B_MN && N % 64 == 0;
  s = make_tmap_expert(c, &tX, x, K, C, K, C * K, (uint32_t)pad, false, elem);
  if (s) return s;
  const uint32_t box = B_MN || EPI == kEpiGlu ? 64 : 128;
  s = B_MN ? make_tmap_expert(c, &tW0, w, N, K, cols, K * cols, box, a.b_chunks) : make_tmap_expert(c, &tW0, w, K, N, K, cols * K, box, false, elem);
  if (s) return s;
  tW1 = tW0;
  if (EPI == kEpiGlu) {
    s = B_MN ? make_tmap_expert(c, &tW1, (P)w + N, N, K, cols, K * cols, box) : make_tmap_expert(c, &tW1, (const char*)w + N * K * elem, K, N, K, cols * K, box, false, elem);
    if (s) return s;
  }
  const long long items = (long long)a.E * ((a.N + (EPI == kEpiGlu ? 63 : 127)) / (EPI == kEpiGlu ? 64 : 128));
  const int grid = (int)std::min<long long>(c->sm_count, items);
  s = room_for(c, expert_few_kernel<EPI, B_MN, Form>, few_smem(EPI, kFewRows, Form));
  if (s) return s;
  expert_few_kernel<EPI, B_MN, Form><<<grid, kFewThreads, few_smem(EPI, pad, Form), st>>>(tW0, tW1, tX, (__nv_bfloat16*)out, (__nv_bfloat16*)pre_out, a,
                                                                                   pad, error_flag_of(c));
  MS_LAUNCH_CHECK("expert_few_kernel");
  c->launches += 1;
  return MAXSCORE_OK;
}

inline ExpertArgs expert_args(const maxscore_ctx* c, const int32_t* load, int M, int N, int K, int accumulate = 0) {
  ExpertArgs a{};
  a.load = load; a.E = c->p.E; a.C = c->C; a.M = M; a.N = N; a.K = K; a.accumulate = accumulate;
  return a;
}

}  // namespace msr
