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
// 8-bit forms (integers; kept activations, forward and backward): half the weight bytes or all of them, and epilogues of their own.
// E 64, 2048 -> 1024: integers, gated, 16 rows 49 us (5.5 TB/s), one token of eight experts 10; kept, 16 rows 88, its backward 51 (5.4 TB/s).
#pragma once
#include "expert_tc.cuh"

namespace msr {

constexpr int kFewRows = 128, kFewThreads = 192;
// Bytes of the operand ring, and of each epilogue warp's staging (8-bit forms: three boxes of 16 rows of 64 bytes, and 16 of kept g and u)
__host__ __device__ constexpr int few_ring(int form) { return form == kBf16 ? 196608 : 180224; }
__host__ __device__ constexpr int few_box(int form) { return form == kBf16 ? 0 : 4096; }
__host__ __device__ constexpr int few_pad(int rows) { return (rows + 15) / 16 * 16; }
__host__ __device__ constexpr int few_stage_bytes(int pad) { return 16384 + pad * 128; }
__host__ __device__ constexpr int few_smem(int epi, int pad, int form) { return few_ring(form) + (epi == kEpiGlu ? pad * 256 : 0) + 4 * few_box(form) + 1024; }
constexpr int kFewMaxStages = 10;

struct FewSmem {
  uint64_t full[kFewMaxStages], empty[kFewMaxStages], acc_full[2], acc_empty[2];
  uint32_t tmem;
  int failed;
  int rows[kMaxE], first[kMaxE + 1];     // rows in use; items before each expert
  int start;                             // expert of the CTA's first item
};

// Whether a condition holds on all 128 epilogue threads; a barrier for them too.
__device__ __forceinline__ bool all_epilogue_threads(bool x) {
  int r;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.s32 q, %1, 0;\n\tbar.red.and.pred p, 1, 128, q;\n\tselp.s32 %0, 1, 0, p;\n\t}"
               : "=r"(r) : "r"((int)x) : "memory");
  return r != 0;
}

// W_MN: the weights' columns are contiguous.  tW0 / tW1: weights (gated: gate / up columns); tX: the rows.
// out, pre_out: y; h and [g | u] kept or null; dpre and h or null (backward of kKeep8).
template <int EPI, bool W_MN, int Form = kBf16>
__global__ void __launch_bounds__(kFewThreads)
expert_few_kernel(const __grid_constant__ CUtensorMap tW0, const __grid_constant__ CUtensorMap tW1, const __grid_constant__ CUtensorMap tX,
                  __nv_bfloat16* __restrict__ out, __nv_bfloat16* __restrict__ pre_out, ExpertArgs a, int pad, unsigned* error_flag) {
  constexpr int kCols = EPI == kEpiGlu ? 64 : 128;                    // output columns of an item
  extern __shared__ unsigned char fsm_raw[];
  unsigned char* base = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(fsm_raw) + 1023) & ~(uintptr_t)1023);
  float* up = reinterpret_cast<float*>(base + few_ring(Form));        // [pad][64], gated only
  __shared__ FewSmem sm;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr int kBK = Form == kInt8 ? 2 * kXBK : kXBK, kDepth = kBK / 4;      // depths of a slice (128 bytes) and of an MMA
  const int ntn = (a.N + kCols - 1) / kCols, nkb = (a.K + kBK - 1) / kBK;
  const int stage_bytes = few_stage_bytes(pad), stages = min(kFewMaxStages, few_ring(Form) / stage_bytes);
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
  if (warp == 2) expert_prefix(a, sm.rows, sm.first, blockIdx.x, &sm.start, [&](int r) { return r > 0 ? ntn : 0; });
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm.tmem;
  const int total = sm.first[a.E];

  if (warp == 0) {
    if (lane == 0) {
      int s = 0, e = sm.start; uint32_t ph = 1; bool ok = true;
      for (int t = blockIdx.x; t < total && ok; t += gridDim.x) {
        while (t >= sm.first[e + 1]) ++e;
        const int n0 = (t - sm.first[e]) * kCols;
        for (int kb = 0; kb < nkb; ++kb) {
          ok = mbar_wait_bounded(&sm.empty[s], ph);
          if (!ok) break;
          unsigned char* w = base + (size_t)s * stage_bytes;
          const uint32_t sw = smem_u32(w);
          const int k0 = kb * kBK;
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
    const uint32_t idesc = idesc_types(Form) | ((uint32_t)(pad >> 3) << 17) | ((128u >> 4) << 24) | (W_MN ? 1u << 15 : 0u);
    auto mma = [](uint32_t d, uint64_t wd, uint64_t xd, uint32_t id, uint32_t add) {
      if constexpr (Form == kInt8) umma_i8(d, wd, xd, id, add); else umma_bf16(d, wd, xd, id, add);
    };
    constexpr uint32_t kWStep = W_MN ? 128 : 2;
    int s = 0, turn = 0; uint32_t ph = 0; bool ok = true;
    for (int t = blockIdx.x; t < total && ok; t += gridDim.x, ++turn) {
      const int buf = turn & 1;
      const uint32_t acc = tmem + (uint32_t)(buf * pad);
      ok = mbar_wait_warp(&sm.acc_empty[buf], (uint32_t)(((turn >> 1) & 1) ^ 1));
      for (int kb = 0; kb < nkb && ok; ++kb) {
        ok = mbar_wait_warp(&sm.full[s], ph);
        if (!ok) break;
        tc_fence_after();
        const uint32_t sw = smem_u32(base) + (uint32_t)(s * stage_bytes);
        const uint64_t wd = W_MN ? smem_desc_mn128(sw, 8192u) : smem_desc_k128(sw), xd = smem_desc_k128(sw + 16384);
        const int left = a.K - kb * kBK;
        if (elect_one()) {
          mma(acc, wd, xd, idesc, kb > 0 ? 1u : 0u);
          if (left > kDepth) mma(acc, wd + kWStep, xd + 2, idesc, 1u);
          if (left > 2 * kDepth) mma(acc, wd + 2 * kWStep, xd + 4, idesc, 1u);
          if (left > 3 * kDepth) mma(acc, wd + 3 * kWStep, xd + 6, idesc, 1u);
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
      expert_zero_behind_rows(a, sm.rows, (char*)out, (EPI == kEpiDact ? 4 : 2) * (size_t)a.N, w, ws);
      if (EPI == kEpiDact && pre_out) expert_zero_behind_rows(a, sm.rows, (char*)pre_out, 2 * (size_t)a.N, w, ws);
      if (EPI == kEpiGlu && pre_out) expert_zero_behind_rows(a, sm.rows, (char*)pre_out, 4 * (size_t)a.N, w, ws);
    }
    int turn = 0, e = sm.start; bool ok = true;
    for (int t = blockIdx.x; t < total; t += gridDim.x, ++turn) {
      while (t >= sm.first[e + 1]) ++e;
      const int rows = sm.rows[e], buf = turn & 1;
      const int col = (t - sm.first[e]) * kCols + (EPI == kEpiGlu ? (q & 1) * 32 : q * 32) + lane;
      const uint32_t acc = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(buf * pad);
      const size_t row0 = (size_t)e * a.C;
      const int first = col - lane;                                    // of the warp's 32 columns: a block of kept activations
      // backward from kept activations: a lane brings 16 bytes of g and of u, and lane j the step of g (lanes 16 on: of u) of row j
      uint4 kg, ku;
      float steps = 0.f;
      auto fetch = [&](int c0) {
        const int fp = keep_width(a.N), blocks = fp / kKeepBlock, r = c0 + (lane & 15);
        const bool in = first < a.N && c0 + (lane >> 1) < rows;
        const uint4* p = reinterpret_cast<const uint4*>(a.keep + (row0 + c0 + (lane >> 1)) * 2 * fp + first + (lane & 1) * 16);
        kg = in ? __ldg(p) : make_uint4(0, 0, 0, 0);
        ku = in ? __ldg(p + fp / 16) : make_uint4(0, 0, 0, 0);
        if (first < a.N && r < rows) steps = __ldg(a.keep_scale + ((size_t)e * 2 * blocks + (lane >> 4) * blocks + first / kKeepBlock) * a.C + r);
      };
      if constexpr (EPI == kEpiDact) fetch(0);
      // integers: the column's scale and the scales of 16 rows, those of the first rows ahead of the accumulator too
      float col_scale = 0.f, first_rows = 0.f;
      auto row_scales = [&](int c0) { return c0 + (lane & 15) < rows ? __ldg(a.x_scale + row0 + c0 + (lane & 15)) : 0.f; };
      if constexpr (Form == kInt8) {
        if (col < a.N) col_scale = __ldg(a.w_scale + (EPI == kEpiGlu ? (size_t)e * 2 * a.N + (q >= 2 ? a.N : 0) : (size_t)e * a.N) + col);
        first_rows = row_scales(0);
        __syncwarp();
      }
      ok = mbar_wait_warp(&sm.acc_full[buf], (uint32_t)((turn >> 1) & 1));
      if (EPI == kEpiGlu) ok = all_epilogue_threads(ok);   // (also: the last item's values have been read from `up`)
      if (!ok) break;
      tc_fence_after();
      if constexpr (Form != kBf16) {
        // What a row costs here bounds these forms from a few dozen rows on.  Results pass through 16-row boxes so that they leave as
        // 16-byte stores, and what belongs to a row (its scale, a block's step) is read or worked out once, by one lane.
        unsigned char* box = base + few_ring(Form) + (EPI == kEpiGlu ? pad * 256 : 0) + (warp - 2) * few_box(Form);
        auto take = [&](int c0, float (&r)[16]) {                      // 16 rows of the column; integers become the values they stand for
          float xs = first_rows;
          if (Form == kInt8 && c0 > 0) xs = row_scales(c0);
          __syncwarp();
          tmem_ld16(acc + c0, r);
          if constexpr (Form == kInt8) {
            if (__any_sync(0xffffffffu, far8(xs) || far8(col_scale))) {
#pragma unroll
              for (int j = 0; j < 16; ++j) r[j] = value8(__float_as_int(r[j]), __shfl_sync(0xffffffffu, xs, j), col_scale);
            } else {
#pragma unroll
              for (int j = 0; j < 16; ++j) r[j] = (float)__float_as_int(r[j]) * (__shfl_sync(0xffffffffu, xs, j) * col_scale);
            }
          }
        };
        auto put = [&](int b, int j, float v) { reinterpret_cast<__nv_bfloat16*>(box + b * 1024 + j * 64)[lane] = __float2bfloat16(v); };
        auto flush = [&](int b, __nv_bfloat16* dst, size_t stride, int c0) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int r = i * 8 + (lane >> 2), c = first + (lane & 3) * 8;
            if (c0 + r < rows && c < a.N)
              *reinterpret_cast<uint4*>(dst + (row0 + c0 + r) * stride + c) = *reinterpret_cast<const uint4*>(box + b * 1024 + r * 64 + (lane & 3) * 16);
          }
        };
        // columns behind d_ff are zero, as the copies filled the weights up
        auto keep = [&](int c0, const float (&r)[16]) {
          const int fp = keep_width(a.N), blocks = fp / kKeepBlock, half = q >= 2;
          uint32_t amax = 0;
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const uint32_t m = __reduce_max_sync(0xffffffffu, abs_bits(__float_as_uint(r[j])));
            if ((lane & 15) == j) amax = m;
          }
          const Step8 st8 = step8(amax);
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const float inv = __shfl_sync(0xffffffffu, st8.inv, j);
            box[j * 32 + lane] = inv > 0.f ? (unsigned char)round8(r[j], inv) : (unsigned char)0;
          }
          __syncwarp();
          if (first < a.N) {
            if (c0 + (lane >> 1) < rows)
              *reinterpret_cast<uint4*>(a.keep + ((row0 + c0 + (lane >> 1)) * 2 + half) * fp + first + (lane & 1) * 16) = *reinterpret_cast<const uint4*>(box + lane * 16);
            if (lane < 16 && c0 + lane < rows) a.keep_scale[((size_t)e * 2 * blocks + half * blocks + first / kKeepBlock) * a.C + c0 + lane] = st8.scale;
          }
          __syncwarp();
        };
        if constexpr (EPI == kEpiPlain) {
          for (int c0 = 0; c0 < rows; c0 += 16) {
            float r[16];
            take(c0, r);
#pragma unroll
            for (int j = 0; j < 16; ++j) put(0, j, r[j]);
            __syncwarp();
            flush(0, out, a.N, c0);
            __syncwarp();
          }
        } else if constexpr (EPI == kEpiDact) {
          const unsigned char* kept = box + 3 * 1024;
          for (int c0 = 0; c0 < rows; c0 += 16) {
            *reinterpret_cast<uint4*>(box + 3 * 1024 + lane * 16) = kg;
            *reinterpret_cast<uint4*>(box + 3 * 1024 + 512 + lane * 16) = ku;
            const float now = steps;
            __syncwarp();
            if (c0 + 16 < rows) fetch(c0 + 16);
            float r[16];
            take(c0, r);
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              const float g = (float)(int8_t)kept[j * 32 + lane] * __shfl_sync(0xffffffffu, now, j);
              const float u = (float)(int8_t)kept[512 + j * 32 + lane] * __shfl_sync(0xffffffffu, now, 16 + j);
              const float s = sigmoid_f<true>(g);
              put(0, j, r[j] * u * s * (1.f + g * (1.f - s)));
              put(1, j, r[j] * g * s);
              put(2, j, g * s * u);
            }
            __syncwarp();
            flush(0, out, 2 * (size_t)a.N, c0);
            flush(1, out + a.N, 2 * (size_t)a.N, c0);
            if (pre_out) flush(2, pre_out, a.N, c0);
            __syncwarp();
          }
        } else {
          // The lower rows' u goes over to the warps that hold g, the upper rows' g to those that hold u: each half forms its part of h.
          const bool gate = q < 2;
          const int mid = (rows + 31) / 32 * 16;
          for (int c0 = 0; c0 < rows; c0 += 16) {
            const bool give = gate == (c0 >= mid);
            if (Form != kKeep8 && !give) continue;
            float r[16];
            take(c0, r);
            if constexpr (Form == kKeep8) keep(c0, r);
            if (give) {
#pragma unroll
              for (int j = 0; j < 16; ++j) up[(c0 + j) * 64 + (q & 1) * 32 + lane] = r[j];
            }
          }
          asm volatile("bar.sync 1, 128;" ::: "memory");
          for (int c0 = gate ? 0 : mid; c0 < (gate ? min(mid, rows) : rows); c0 += 16) {
            float r[16];
            take(c0, r);
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              const float o = up[(c0 + j) * 64 + (q & 1) * 32 + lane];
              put(0, j, gate ? silu_mul<true>(r[j], o) : silu_mul<true>(o, r[j]));
            }
            __syncwarp();
            flush(0, out, a.N, c0);
            __syncwarp();
          }
        }
      } else if constexpr (EPI == kEpiPlain) {
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
