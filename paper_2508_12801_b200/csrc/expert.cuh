// Expert products: matrix products grouped by expert over the [E, C, width] buffers that dispatch fills.
// Expert e owns the first min(expert_load[e], C) rows of its block; the loads are only known on the device, so
// every kernel here is persistent and walks tiles that it counts from the loads itself.
//
//   y_e  = x_e W_e                      (kEpiPlain; with the layout flipped: the gradient with respect to x)
//   h_e  = silu(x_e W_g) * (x_e W_u)    (kEpiGlu)
//   dpre = [dh u s(1 + g(1-s)) | dh g s] with dh = dy_e W_down^T, s = 1 / (1 + e^-g)     (kEpiDact)
//   dW_e = x_e^T dy_e                   (kEpiDw, fp32 output)
//
// fp32 I/O: plain FMA tiles (tensor cores would round the inputs to tf32).
#pragma once
#include "common.cuh"
#include "gate.cuh"

namespace msr {

enum ExpertEpi { kEpiPlain = 0, kEpiGlu = 1, kEpiDact = 2, kEpiDw = 3 };

struct ExpertArgs {
  const int32_t* load;      // [E]
  int E, C;
  int M, N, K;              // dW: M = d_in, N = d_out, K per expert; else M per expert, N = columns (d_ff for the gated ones)
  int accumulate;           // dW only
  int a_chunks, b_chunks;   // tensor cores: the operand's map has the 64-column chunks as a dimension of their own
};

__device__ __forceinline__ int expert_rows(const ExpertArgs& a, int e) {
  const int r = __ldg(a.load + e);
  return r < 0 ? 0 : r < a.C ? r : a.C;
}
// sigmoid(g) = 1 / (1 + e^-g): for g far below zero e^-g is infinite and the quotient 0, which is the limit.
// Fast: for values that are rounded to bf16 afterwards (the approximate exponential is good to about 2^-20).
template <bool Fast>
__device__ __forceinline__ float sigmoid_f(float g) {
  return Fast ? __fdividef(1.f, 1.f + __expf(-g)) : 1.f / (1.f + expf(-g));
}
template <bool Fast>
__device__ __forceinline__ float silu_mul(float g, float u) { return g * sigmoid_f<Fast>(g) * u; }
template <bool Fast>
__device__ __forceinline__ void dact(float dh, float g, float u, float& dg, float& du) {
  const float s = sigmoid_f<Fast>(g);
  dg = dh * u * s * (1.f + g * (1.f - s));
  du = dh * g * s;
}

// Rows behind the loads of an [E, C, row] buffer become zero.  `grain`: rows that the tiles of the caller write anyway
// (their last tile is written whole, zeros behind the load).
__device__ void expert_zero_behind(const ExpertArgs& a, const int* rows, char* y, size_t row_bytes, int grain, int worker,
                                   int workers) {
  const int vecs = (int)(row_bytes / 16);
  for (int e = 0; e < a.E; ++e) {
    const int r0 = (rows[e] + grain - 1) / grain * grain;
    if (r0 >= a.C) continue;
    uint4* p = reinterpret_cast<uint4*>(y + ((size_t)e * a.C + r0) * row_bytes);
    const size_t n = (size_t)(a.C - r0) * vecs;
    for (size_t i = worker; i < n; i += workers) p[i] = make_uint4(0, 0, 0, 0);
  }
}

// The same where rows are few: a warp per row of the whole buffer, so that many experts with next to nothing cost one step.
__device__ void expert_zero_behind_rows(const ExpertArgs& a, const int* rows, char* y, size_t row_bytes, int warp, int warps) {
  const int vecs = (int)(row_bytes / 16), lane = threadIdx.x & 31;
  for (int r = warp; r < a.E * a.C; r += warps) {
    const int e = r / a.C;
    if (r - e * a.C < rows[e]) continue;
    uint4* p = reinterpret_cast<uint4*>(y + (size_t)r * row_bytes);
    for (int v = lane; v < vecs; v += 32) p[v] = make_uint4(0, 0, 0, 0);
  }
}

// ---- FMA tiles -----------------------------------------------------------------------------------------------------
// A CTA of 256 threads owns a BM x BN tile, a thread TM x TN of it in two halves along each side (so that shared-memory
// reads are conflict-free and a thread of the gated product holds the gate and the up value of the same column).  The
// next 16-deep slice is in registers while the current one is multiplied.
constexpr int kFmaBK = 16;
__device__ __forceinline__ float4 load4(const float* p) { return __ldg(reinterpret_cast<const float4*>(p)); }
__device__ __forceinline__ float4 load4(const __nv_bfloat16* p) {
  const uint2 v = __ldg(reinterpret_cast<const uint2*>(p));
  return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16),
                     __uint_as_float(v.y & 0xffff0000u));
}
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16(v); }

template <typename T, int BM, int BN, int EPI, bool A_MN, bool B_MN>
__global__ void __launch_bounds__(256)
expert_fma_kernel(const T* __restrict__ A, const T* __restrict__ B, const T* __restrict__ pre_in, void* __restrict__ out_raw,
                  T* __restrict__ pre_out, ExpertArgs a) {
  T* out = reinterpret_cast<T*>(out_raw);
  constexpr int TM = BM / 16, TN = BN / 16, HM = TM / 2, HN = TN / 2;
  constexpr int LA = BM * kFmaBK / 4 / 256, LB = BN * kFmaBK / 4 / 256;   // float4 loads per thread and slice
  static_assert(LA >= 1 && LB >= 1, "tile too small for 256 threads");
  __shared__ __align__(16) float sa[2][kFmaBK][BM + 4], sb[2][kFmaBK][BN + 4];
  __shared__ int srows[kMaxE];
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  if (tid < a.E) srows[tid] = expert_rows(a, tid);
  __syncthreads();
  constexpr int BNU = EPI == kEpiGlu ? BN / 2 : BN;       // output columns per tile
  const int ntn = (a.N + BNU - 1) / BNU, ntm_dw = (a.M + BM - 1) / BM;
  const int ldb_cols = EPI == kEpiGlu ? 2 * a.N : a.N;    // columns of the weight matrix
  long long tile = blockIdx.x, first = 0;
  for (int e = 0; e < a.E; ++e) {
    const int rows = srows[e];
    const int ntm = EPI == kEpiDw ? ntm_dw : (rows + BM - 1) / BM;
    const int K = EPI == kEpiDw ? rows : a.K, M = EPI == kEpiDw ? a.M : rows;
    const long long n_tiles = (long long)ntm * ntn;
    const T* Ae = A + (EPI == kEpiDw ? (size_t)e * a.C * a.M : (size_t)e * a.C * a.K);
    const T* Be = B + (EPI == kEpiDw ? (size_t)e * a.C * a.N : (size_t)e * ldb_cols * a.K);
    for (; tile < first + n_tiles; tile += gridDim.x) {
      const int m0 = (int)((tile - first) / ntn) * BM, n0 = (int)((tile - first) % ntn) * BNU;
      float4 ra[LA], rb[LB];
      auto load = [&](int k0) {
#pragma unroll
        for (int i = 0; i < LA; ++i) {
          const int q = tid + i * 256;
          const int m = m0 + (A_MN ? (q % (BM / 4)) * 4 : q / 4), k = k0 + (A_MN ? q / (BM / 4) : (q % 4) * 4);
          ra[i] = (m < M && k < K) ? load4(A_MN ? Ae + (size_t)k * a.M + m : Ae + (size_t)m * a.K + k)
                                   : make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll
        for (int i = 0; i < LB; ++i) {
          const int q = tid + i * 256;
          int c = B_MN ? (q % (BN / 4)) * 4 : q / 4;
          const int k = k0 + (B_MN ? q / (BN / 4) : (q % 4) * 4);
          int n = n0 + c; bool in = n < a.N;
          if (EPI == kEpiGlu && c >= BNU) { n = n0 + c - BNU; in = n < a.N; n += a.N; }
          rb[i] = (in && k < K) ? load4(B_MN ? Be + (size_t)k * ldb_cols + n : Be + (size_t)n * a.K + k)
                                : make_float4(0.f, 0.f, 0.f, 0.f);
        }
      };
      auto stash = [&](int s) {
#pragma unroll
        for (int i = 0; i < LA; ++i) {
          const int q = tid + i * 256;
          if (A_MN) *reinterpret_cast<float4*>(&sa[s][q / (BM / 4)][(q % (BM / 4)) * 4]) = ra[i];
          else { const int k = (q % 4) * 4, m = q / 4; sa[s][k][m] = ra[i].x; sa[s][k + 1][m] = ra[i].y; sa[s][k + 2][m] = ra[i].z; sa[s][k + 3][m] = ra[i].w; }
        }
#pragma unroll
        for (int i = 0; i < LB; ++i) {
          const int q = tid + i * 256;
          if (B_MN) *reinterpret_cast<float4*>(&sb[s][q / (BN / 4)][(q % (BN / 4)) * 4]) = rb[i];
          else { const int k = (q % 4) * 4, n = q / 4; sb[s][k][n] = rb[i].x; sb[s][k + 1][n] = rb[i].y; sb[s][k + 2][n] = rb[i].z; sb[s][k + 3][n] = rb[i].w; }
        }
      };
      float acc[TM][TN];
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = 0.f;
      const int slices = (K + kFmaBK - 1) / kFmaBK;
      if (slices > 0) { load(0); stash(0); }
      __syncthreads();
      for (int s = 0; s < slices; ++s) {
        if (s + 1 < slices) load((s + 1) * kFmaBK);
#pragma unroll
        for (int k = 0; k < kFmaBK; ++k) {
          float x[TM], w[TN];
#pragma unroll
          for (int i = 0; i < HM; ++i) { x[i] = sa[s & 1][k][ty * HM + i]; x[HM + i] = sa[s & 1][k][BM / 2 + ty * HM + i]; }
#pragma unroll
          for (int j = 0; j < HN; ++j) { w[j] = sb[s & 1][k][tx * HN + j]; w[HN + j] = sb[s & 1][k][BN / 2 + tx * HN + j]; }
#pragma unroll
          for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = fmaf(x[i], w[j], acc[i][j]);
        }
        if (s + 1 < slices) stash((s + 1) & 1);
        __syncthreads();
      }
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const int m = m0 + (i < HM ? ty * HM + i : BM / 2 + ty * HM + i - HM);
        if (m >= M) continue;
        if constexpr (EPI == kEpiGlu) {
#pragma unroll
          for (int j = 0; j < HN; ++j) {
            const int n = n0 + tx * HN + j;
            if (n >= a.N) continue;
            const size_t row = (size_t)e * a.C + m;
            if (pre_out) { put(pre_out + row * 2 * a.N + n, acc[i][j]); put(pre_out + row * 2 * a.N + a.N + n, acc[i][HN + j]); }
            put(out + row * a.N + n, silu_mul<false>(acc[i][j], acc[i][HN + j]));
          }
        } else {
#pragma unroll
          for (int j = 0; j < TN; ++j) {
            const int n = n0 + (j < HN ? tx * HN + j : BN / 2 + tx * HN + j - HN);
            if (n >= a.N) continue;
            if constexpr (EPI == kEpiDw) {
              float* o = reinterpret_cast<float*>(out_raw) + ((size_t)e * a.M + m) * a.N + n;
              *o = a.accumulate ? *o + acc[i][j] : acc[i][j];
            } else if constexpr (EPI == kEpiDact) {
              const size_t row = ((size_t)e * a.C + m) * 2 * a.N;
              float dg, du;
              dact<false>(acc[i][j], to_f(pre_in[row + n]), to_f(pre_in[row + a.N + n]), dg, du);
              put(out + row + n, dg); put(out + row + a.N + n, du);
            } else {
              put(out + ((size_t)e * a.C + m) * a.N + n, acc[i][j]);
            }
          }
        }
      }
    }
    first += n_tiles;
  }
  if constexpr (EPI != kEpiDw) {
    const int worker = blockIdx.x * 256 + tid, workers = gridDim.x * 256;
    expert_zero_behind(a, srows, (char*)out, sizeof(T) * (size_t)(EPI == kEpiDact ? 2 * a.N : a.N), 1, worker, workers);
    if (EPI == kEpiGlu && pre_out) expert_zero_behind(a, srows, (char*)pre_out, sizeof(T) * 2 * (size_t)a.N, 1, worker, workers);
  }
}

}  // namespace msr
