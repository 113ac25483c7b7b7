// What the C entry points share on the host: the context, the workspace's layout, error texts.
//
// The entry points are two translation units, and so two modules on the device: the first kernel that a process uses loads its module
// whole, and the experts' and norms' kernels are many (first context of a process 41 ms with them, 7 without).
#pragma once
#include "../../include/maxscore.h"

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <stdio.h>

namespace msr {

extern thread_local char g_last_error[256] __attribute__((visibility("hidden")));

inline maxscore_status cuda_fail(cudaError_t e, const char* where) {
  snprintf(g_last_error, sizeof(g_last_error), "%s: %s", where, cudaGetErrorString(e));
  return MAXSCORE_ERR_CUDA;
}
#define MS_CUDA(call)                                              \
  do {                                                             \
    cudaError_t e_ = (call);                                       \
    if (e_ != cudaSuccess) return cuda_fail(e_, #call);            \
  } while (0)
#define MS_LAUNCH_CHECK(name)                                      \
  do {                                                             \
    cudaError_t e_ = cudaGetLastError();                           \
    if (e_ != cudaSuccess) return cuda_fail(e_, name);             \
  } while (0)

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

struct Layout {          // byte offsets inside the workspace
  size_t state, aux, cand, rec_val, rec_meta, rec_pos, rec_bxc, rec_ndv, rec_off, rec_cnt, rec_aarg, rr_choice, rr_rank, rr_cnt, rr_base, rr_held, rr_dropped, rr_bc, rr_blk, rr_dtok, rr_order, rr_dnum, a1_v, a1_partial, a1_ticket, cache_x, cache_id, cache_bound, cache_raw, block_counts, wt, error_flag, dls, wk, dwpart, normpart, total;
  int Npad, n_idx_blocks;
  int rec_cap;                                // entries of the exact phase's candidate records
  int Kpad, dw_splits, dw_tokens_per_split;   // tensor-core backward GEMMs (bf16 I/O)
};

// The norm backward on rows of nvec 16-byte vectors: vectors a thread, threads (without the producer's warp), CTAs of an SM, and
// the rows of partial column sums in the workspace (units, and CTAs, at most; a B200 has 148 SMs).
inline int norm_bwd_vecs(int nvec) { return nvec <= 512 ? 1 : nvec <= 1024 ? 2 : 4; }
inline int norm_threads(int nvec, int vecs) { return ((nvec + vecs - 1) / vecs + 31) / 32 * 32; }
inline int norm_ctas(int threads) { return threads <= 64 ? 8 : threads <= 128 ? 4 : threads <= 256 ? 2 : 1; }
inline int norm_bwd_ctas(int nvec) { return norm_bwd_vecs(nvec) == 1 ? norm_ctas(norm_threads(nvec, 1)) : 1; }
inline int norm_parts(const maxscore_params& p) {
  const int nvec = (int)((size_t)p.d_model * (p.io_dtype == MAXSCORE_BF16 ? 2 : 4) / 16), parts = 148 * (norm_bwd_ctas(nvec) < 4 ? norm_bwd_ctas(nvec) : 4);
  return p.T < parts ? p.T : parts;
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

constexpr int kRoomyMax = 32;            // more than the kernels that one context's sizes and type can choose

}  // namespace msr

struct maxscore_ctx {
  maxscore_params p;
  int32_t C;
  msr::Layout lay;
  char* ws;
  msr::EncodeTiledFn encode;
  int sm_count;
  int sweep_grid_max;   // CTAs of the sweeps kernel that are resident at once
  long long launches;   // kernels launched through this context so far
  const void* roomy[msr::kRoomyMax];         // expert and norm kernels whose shared-memory limit this context has asked for
  int n_roomy = 0;
  // host path (maxscore_route_dispatch_host): a copy stream and its events, made on the first call
  cudaStream_t copy_stream = nullptr;
  cudaEvent_t ev_start = nullptr, ev_routed = nullptr, ev_copied = nullptr, ev_chunk[8] = {};
};

namespace msr {

inline unsigned* error_flag_of(const maxscore_ctx* c) { return reinterpret_cast<unsigned*>(c->ws + c->lay.error_flag); }
inline size_t elem_bytes(const maxscore_ctx* c) { return c->p.io_dtype == MAXSCORE_BF16 ? 2 : 4; }

}  // namespace msr
