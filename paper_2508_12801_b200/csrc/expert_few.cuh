// Expert products when every expert has few rows (bf16 I/O, capacity up to kFewRows): serving batches, down to one token.
//
// The weights of the experts in use are read once and that read is the whole cost (2 flops per weight byte and row), so the
// product is turned round: 128 weight columns are the M side of the MMA and the expert's rows its N side, 16 to 128 of them.
// Nothing of a weight tile is wasted on absent rows, and a stage is little more than its 16 KB of weights: a ring of 6 to 10
// stages keeps 96 to 160 KB of weights in flight on every SM.  One CTA per SM walks (expert with rows, 128 columns) items.
//   warp 0: TMA loads;  warp 1: TMEM and MMAs;  warps 2-5: epilogue, a TMEM lane (= output column) per thread.
// Measured (cold caches): E 64 with 2 rows each, 2048 -> 1024 gated 104 us, 5.1 TB/s; E 128 with 4 rows, 4096 -> 1024 346 us,
// 6.2 TB/s; one token 15 us on the device (10 by its bytes).  At C 128 it still leads the 256-row tiles (112 against 135 us,
// E 64, 2048 -> 2048): those would be half empty.
// Gated form: 64 gate and 64 up columns share a tile; the up half passes through shared memory to the threads of the gate half.
#pragma once
#include "expert_tc.cuh"

namespace msr {

constexpr int kFewRows = 128, kFewThreads = 192, kFewRing = 196608;       // bytes of the operand ring
__host__ __device__ constexpr int few_pad(int rows) { return (rows + 15) / 16 * 16; }
__host__ __device__ constexpr int few_stage_bytes(int pad) { return 16384 + pad * 128; }
__host__ __device__ constexpr int few_smem(int epi, int pad) { return kFewRing + (epi == kEpiGlu ? pad * 256 : 0) + 1024; }
constexpr int kFewMaxStages = 10;

struct FewSmem {
  uint64_t full[kFewMaxStages], empty[kFewMaxStages], acc_full[2], acc_empty[2];
  uint32_t tmem;
  int failed;
  int rows[kMaxE], first[kMaxE + 1];     // rows in use; items before each expert
};

// Whether a condition holds on all 128 epilogue threads; a barrier for them too.
__device__ __forceinline__ bool all_epilogue_threads(bool x) {
  int r;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.s32 q, %1, 0;\n\tbar.red.and.pred p, 1, 128, q;\n\tselp.s32 %0, 1, 0, p;\n\t}"
               : "=r"(r) : "r"((int)x) : "memory");
  return r != 0;
}

// W_MN: the weights' columns are contiguous.  tW0 / tW1: weights (gated: gate / up columns); tX: the rows.
template <int EPI, bool W_MN>
__global__ void __launch_bounds__(kFewThreads)
expert_few_kernel(const __grid_constant__ CUtensorMap tW0, const __grid_constant__ CUtensorMap tW1, const __grid_constant__ CUtensorMap tX,
                  __nv_bfloat16* __restrict__ out, __nv_bfloat16* __restrict__ pre_out, ExpertArgs a, int pad, unsigned* error_flag) {
  constexpr int kCols = EPI == kEpiGlu ? 64 : 128;                    // output columns of an item
  extern __shared__ unsigned char fsm_raw[];
  unsigned char* base = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(fsm_raw) + 1023) & ~(uintptr_t)1023);
  float* up = reinterpret_cast<float*>(base + kFewRing);              // [pad][64], gated only
  __shared__ FewSmem sm;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int ntn = (a.N + kCols - 1) / kCols, nkb = (a.K + kXBK - 1) / kXBK;
  const int stage_bytes = few_stage_bytes(pad), stages = min(kFewMaxStages, kFewRing / stage_bytes);
  uint32_t tmem_cols = 32;
  while ((int)tmem_cols < 2 * pad) tmem_cols <<= 1;

  if (threadIdx.x == 0) {
    prefetch_tmap(&tW0); prefetch_tmap(&tX);
    if (EPI == kEpiGlu) prefetch_tmap(&tW1);
    for (int s = 0; s < stages; ++s) { mbar_init(&sm.full[s], 1); mbar_init(&sm.empty[s], 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(&sm.acc_full[b], 1); mbar_init(&sm.acc_empty[b], 4); }
    sm.failed = 0;
    fence_barrier_init();
  }
  if (warp == 1) tmem_alloc(&sm.tmem, tmem_cols);
  if (warp == 2) expert_prefix(a, sm.rows, sm.first, [&](int r) { return r > 0 ? ntn : 0; });
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm.tmem;
  const int total = sm.first[a.E];

  if (warp == 0) {
    if (lane == 0) {
      int s = 0, e = 0; uint32_t ph = 1; bool ok = true;
      for (int t = blockIdx.x; t < total && ok; t += gridDim.x) {
        while (t >= sm.first[e + 1]) ++e;
        const int n0 = (t - sm.first[e]) * kCols;
        for (int kb = 0; kb < nkb; ++kb) {
          ok = mbar_wait_bounded(&sm.empty[s], ph);
          if (!ok) break;
          unsigned char* w = base + (size_t)s * stage_bytes;
          const uint32_t sw = smem_u32(w);
          const int k0 = kb * kXBK;
          mbar_expect_tx(&sm.full[s], stage_bytes);
          if (EPI == kEpiGlu) {
            if (W_MN) { tma_load_3d(sw, &tW0, n0, k0, e, &sm.full[s]); tma_load_3d(sw + 8192, &tW1, n0, k0, e, &sm.full[s]); }
            else { tma_load_3d(sw, &tW0, k0, n0, e, &sm.full[s]); tma_load_3d(sw + 8192, &tW1, k0, n0, e, &sm.full[s]); }
          } else if (!W_MN) {
            tma_load_3d(sw, &tW0, k0, n0, e, &sm.full[s]);
          } else if (a.b_chunks) {
            tma_load_4d(sw, &tW0, k0, n0 >> 6, e, &sm.full[s]);
          } else {
            tma_load_3d(sw, &tW0, n0, k0, e, &sm.full[s]); tma_load_3d(sw + 8192, &tW0, n0 + 64, k0, e, &sm.full[s]);
          }
          tma_load_3d(sw + 16384, &tX, k0, 0, e, &sm.full[s]);
          if (++s == stages) { s = 0; ph ^= 1; }
        }
      }
      if (!ok) sm.failed = 1;
    }
  } else if (warp == 1) {
    const uint32_t idesc = idesc_bf16_m128(pad) | (W_MN ? 1u << 15 : 0u);
    constexpr uint32_t kWStep = W_MN ? 128 : 2;
    int s = 0, turn = 0; uint32_t ph = 0; bool ok = true;
    for (int t = blockIdx.x; t < total && ok; t += gridDim.x, ++turn) {
      const int buf = turn & 1;
      const uint32_t acc = tmem + (uint32_t)(buf * pad);
      ok = mbar_wait_bounded(&sm.acc_empty[buf], (uint32_t)(((turn >> 1) & 1) ^ 1));
      for (int kb = 0; kb < nkb && ok; ++kb) {
        ok = mbar_wait_bounded(&sm.full[s], ph);
        if (!ok) break;
        tc_fence_after();
        const uint32_t sw = smem_u32(base) + (uint32_t)(s * stage_bytes);
        const uint64_t wd = W_MN ? smem_desc_mn128(sw, 8192u) : smem_desc_k128(sw), xd = smem_desc_k128(sw + 16384);
        const int left = a.K - kb * kXBK;
        if (elect_one()) {
          umma_bf16(acc, wd, xd, idesc, kb > 0 ? 1u : 0u);
          if (left > 16) umma_bf16(acc, wd + kWStep, xd + 2, idesc, 1u);
          if (left > 32) umma_bf16(acc, wd + 2 * kWStep, xd + 4, idesc, 1u);
          if (left > 48) umma_bf16(acc, wd + 3 * kWStep, xd + 6, idesc, 1u);
          umma_commit(&sm.empty[s]);
          if (kb == nkb - 1) umma_commit(&sm.acc_full[buf]);
        }
        __syncwarp();
        if (++s == stages) { s = 0; ph ^= 1; }
      }
    }
    if (!ok && lane == 0) sm.failed = 1;
  } else {
    const int q = warp & 3;                             // TMEM lanes this warp may read
    {
      const int w = blockIdx.x * 4 + warp - 2, ws = gridDim.x * 4;
      expert_zero_behind_rows(a, sm.rows, (char*)out, 2 * (size_t)a.N, w, ws);
      if (EPI == kEpiGlu && pre_out) expert_zero_behind_rows(a, sm.rows, (char*)pre_out, 4 * (size_t)a.N, w, ws);
    }
    int turn = 0, e = 0; bool ok = true;
    for (int t = blockIdx.x; t < total; t += gridDim.x, ++turn) {
      while (t >= sm.first[e + 1]) ++e;
      const int rows = sm.rows[e], buf = turn & 1;
      const int col = (t - sm.first[e]) * kCols + (EPI == kEpiGlu ? (q & 1) * 32 : q * 32) + lane;
      const uint32_t acc = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(buf * pad);
      const size_t row0 = (size_t)e * a.C;
      ok = mbar_wait_bounded(&sm.acc_full[buf], (uint32_t)((turn >> 1) & 1));
      if (EPI == kEpiGlu) ok = all_epilogue_threads(ok);   // (also: the last item's values have been read from `up`)
      if (!ok) break;
      tc_fence_after();
      if constexpr (EPI == kEpiPlain) {
        for (int c0 = 0; c0 < rows; c0 += 16) {
          float r[16];
          tmem_ld16(acc + c0, r);
          if (col < a.N) {
#pragma unroll
            for (int j = 0; j < 16; ++j)
              if (c0 + j < rows) out[(row0 + c0 + j) * a.N + col] = __float2bfloat16(r[j]);
          }
        }
      } else {
        if (q >= 2)
          for (int c0 = 0; c0 < rows; c0 += 16) {
            float r[16];
            tmem_ld16(acc + c0, r);
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              up[(c0 + j) * 64 + (q & 1) * 32 + lane] = r[j];
              if (pre_out && col < a.N && c0 + j < rows) pre_out[(row0 + c0 + j) * 2 * a.N + a.N + col] = __float2bfloat16(r[j]);
            }
          }
        asm volatile("bar.sync 1, 128;" ::: "memory");
        if (q < 2)
          for (int c0 = 0; c0 < rows; c0 += 16) {
            float r[16];
            tmem_ld16(acc + c0, r);
            if (col < a.N) {
#pragma unroll
              for (int j = 0; j < 16; ++j)
                if (c0 + j < rows) {
                  out[(row0 + c0 + j) * a.N + col] = __float2bfloat16(silu_mul<true>(r[j], up[(c0 + j) * 64 + (q & 1) * 32 + lane]));
                  if (pre_out) pre_out[(row0 + c0 + j) * 2 * a.N + col] = __float2bfloat16(r[j]);
                }
            }
          }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.acc_empty[buf]);
    }
    if (!ok && lane == 0) sm.failed = 1;
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && sm.failed) {
    atomicOr(error_flag, 4u);
    for (int i = 0; i < 1000; ++i) __nanosleep(1000);   // a wait gave up: let the copies that were in flight land
  }
  __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_dealloc(tmem, tmem_cols);
}

}  // namespace msr
