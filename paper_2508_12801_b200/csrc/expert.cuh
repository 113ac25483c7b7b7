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
#include "tc.cuh"

namespace msr {

enum ExpertEpi { kEpiPlain = 0, kEpiGlu = 1, kEpiDact = 2, kEpiDw = 3 };
// kBf16: operands and results in bf16.  kInt8: operands in 8-bit integers with a scale per row and per column.  kKeep8: as kBf16, with
// [g | u] kept in 8 bits.
enum ExpertForm { kBf16 = 0, kInt8 = 1, kKeep8 = 2 };

struct ExpertArgs {
  const int32_t* load;      // [E]
  int E, C;
  int M, N, K;              // dW: M = d_in, N = d_out, K per expert; else M per expert, N = columns (d_ff for the gated ones)
  int accumulate;           // dW only
  const float *x_scale, *w_scale;      // kInt8: [E, C], and a column's in the order of the weights' columns
  int8_t* keep;             // kKeep8: integers [E, C, 2, keep_width], g first
  float* keep_scale;        // kKeep8: [E, 2 keep_width / 32, C]
  int a_chunks, b_chunks;   // tensor cores: the operand's map has the 64-column chunks as a dimension of their own
};

__device__ __forceinline__ int expert_rows(const ExpertArgs& a, int e) {
  const int r = __ldg(a.load + e);
  return r < 0 ? 0 : r < a.C ? r : a.C;
}
// sigmoid(g) = 1 / (1 + e^-g): for g far below zero e^-g is infinite and the quotient 0, which is the limit.
// Fast: for values that are rounded to bf16 (half a step is 2^-9) afterwards.  The approximate exponential is off by 2 + 1.2 |g| steps
// of 2^-23, 2^-17 at g = -80; below g = -87.3 the quotient is 0 where the exact one is below 2^-126.
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
__device__ inline void expert_zero_behind(const ExpertArgs& a, const int* rows, char* y, size_t row_bytes, int grain, int worker,
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
__device__ inline void expert_zero_behind_rows(const ExpertArgs& a, const int* rows, char* y, size_t row_bytes, int warp, int warps) {
  const int vecs = (int)(row_bytes / 16), lane = threadIdx.x & 31;
  for (int r = warp; r < a.E * a.C; r += warps) {
    const int e = r / a.C;
    if (r - e * a.C < rows[e]) continue;
    uint4* p = reinterpret_cast<uint4*>(y + (size_t)r * row_bytes);
    for (int v = lane; v < vecs; v += 32) p[v] = make_uint4(0, 0, 0, 0);
  }
}

// ---- FMA tiles -----------------------------------------------------------------------------------------------------
// A CTA of 256 threads owns a BM x BN tile, a thread TM x TN of it in groups of four rows and four columns (one 16-byte
// shared-memory read each, conflict-free; what bounds these tiles is those reads).  In the gated product a thread's columns are
// half gate and half up, so that it holds both values of a column.  Products are packed two columns at a time, and the next
// BK-deep slice is in registers while the current one is multiplied.  35 TFLOP/s at E 64, C 256, 1024 x 1024 (72 by the FMA rate; the
// 128 x 128 tiles spill 28 to 120 bytes at their 128 registers).  With few rows a slice is a load latency and a barrier: E 8, C 6,
// 952 -> 1120 56 us, where the library takes 23 and the weights' bytes 5.
__device__ __forceinline__ float4 load4(const float* p) { return __ldg(reinterpret_cast<const float4*>(p)); }

template <int BM, int BN, int BK, int EPI, bool A_MN, bool B_MN>
__global__ void __launch_bounds__(256, BM == 128 ? 2 : 4)
expert_fma_kernel(const float* __restrict__ A, const float* __restrict__ B, const float* __restrict__ pre_in,
                  float* __restrict__ out, float* __restrict__ pre_out, ExpertArgs a) {
  constexpr int TM = BM / 16, TN = BN / 16;
  constexpr int GM = TM < 4 ? TM : 4, GN = EPI == kEpiGlu ? TN / 2 : TN < 4 ? TN : 4;      // rows and columns of a group
  constexpr int HN = TN / 2;
  static_assert(GN == 4 || GN == 2, "columns are read in fours or (gated small tiles) pairs");
  // where a thread's i-th row / j-th column lies in the tile: groups are spread over the tile's halves
  auto row_of = [](int i, int ty) { return i / GM * (BM / (TM / GM)) + ty * GM + i % GM; };
  auto col_of = [](int j, int tx) { return j / GN * (BN / (TN / GN)) + tx * GN + j % GN; };
  // Operands with the contraction contiguous are transposed on the way into shared memory: there the groups of eight rows are
  // permuted with the depth, so that neither those scattered stores nor the reads meet in a bank.
  auto swa = [](int k, int m) { return A_MN || BM < 32 ? m : m ^ (((k >> 2) & 3) << 3); };
  auto swb = [](int k, int n) { return B_MN ? n : n ^ (((k >> 2) & 3) << 3); };
  constexpr int QA = BM * BK / 4, LA = (QA + 255) / 256, LB = BN * BK / 4 / 256;   // float4 loads of a slice; per thread
  static_assert(LB >= 1 && (QA % 256 == 0 || LA == 1), "tile too small for 256 threads");
  __shared__ __align__(16) float sa[2][BK][BM + 4], sb[2][BK][BN + 4];
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
    const float* Ae = A + (EPI == kEpiDw ? (size_t)e * a.C * a.M : (size_t)e * a.C * a.K);
    const float* Be = B + (EPI == kEpiDw ? (size_t)e * a.C * a.N : (size_t)e * ldb_cols * a.K);
    for (; tile < first + n_tiles; tile += gridDim.x) {
      const int m0 = (int)((tile - first) / ntn) * BM, n0 = (int)((tile - first) % ntn) * BNU;
      float4 ra[LA], rb[LB];
      auto load = [&](int k0) {
#pragma unroll
        for (int i = 0; i < LA; ++i) {
          const int q = tid + i * 256;
          const int m = m0 + (A_MN ? (q % (BM / 4)) * 4 : q / (BK / 4)), k = k0 + (A_MN ? q / (BM / 4) : (q % (BK / 4)) * 4);
          ra[i] = (q < QA && m < M && k < K) ? load4(A_MN ? Ae + (size_t)k * a.M + m : Ae + (size_t)m * a.K + k)
                                   : make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll
        for (int i = 0; i < LB; ++i) {
          const int q = tid + i * 256;
          const int c = B_MN ? (q % (BN / 4)) * 4 : q / (BK / 4);
          const int k = k0 + (B_MN ? q / (BN / 4) : (q % (BK / 4)) * 4);
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
          if (q >= QA) break;
          if (A_MN) *reinterpret_cast<float4*>(&sa[s][q / (BM / 4)][(q % (BM / 4)) * 4]) = ra[i];
          else { const int k = (q % (BK / 4)) * 4, m = q / (BK / 4); const int w = swa(k, m); sa[s][k][w] = ra[i].x; sa[s][k + 1][w] = ra[i].y; sa[s][k + 2][w] = ra[i].z; sa[s][k + 3][w] = ra[i].w; }
        }
#pragma unroll
        for (int i = 0; i < LB; ++i) {
          const int q = tid + i * 256;
          if (B_MN) *reinterpret_cast<float4*>(&sb[s][q / (BN / 4)][(q % (BN / 4)) * 4]) = rb[i];
          else { const int k = (q % (BK / 4)) * 4, n = q / (BK / 4); const int w = swb(k, n); sb[s][k][w] = rb[i].x; sb[s][k + 1][w] = rb[i].y; sb[s][k + 2][w] = rb[i].z; sb[s][k + 3][w] = rb[i].w; }
        }
      };
      float2 acc[TM][TN / 2];
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN / 2; ++j) acc[i][j] = both(0.f);
      const int slices = (K + BK - 1) / BK;
      if (slices > 0) { load(0); stash(0); }
      __syncthreads();
      for (int s = 0; s < slices; ++s) {
        if (s + 1 < slices) load((s + 1) * BK);
#pragma unroll
        for (int k = 0; k < BK; ++k) {
          float x[TM];
          float2 w[TN / 2];
#pragma unroll
          for (int i = 0; i < TM; i += GM) {
            if constexpr (GM == 4) *reinterpret_cast<float4*>(&x[i]) = *reinterpret_cast<const float4*>(&sa[s & 1][k][swa(k, row_of(i, ty))]);
            else
#pragma unroll
              for (int u = 0; u < GM; ++u) x[i + u] = sa[s & 1][k][swa(k, row_of(i + u, ty))];
          }
          if constexpr (GN == 4) {
#pragma unroll
            for (int j = 0; j < TN / 2; j += 2) {
              const float4 v = *reinterpret_cast<const float4*>(&sb[s & 1][k][swb(k, col_of(2 * j, tx))]);
              w[j] = make_float2(v.x, v.y); w[j + 1] = make_float2(v.z, v.w);
            }
          } else {
#pragma unroll
            for (int j = 0; j < TN / 2; ++j) w[j] = *reinterpret_cast<const float2*>(&sb[s & 1][k][swb(k, col_of(2 * j, tx))]);
          }
#pragma unroll
          for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN / 2; ++j) acc[i][j] = fma2(both(x[i]), w[j], acc[i][j]);
        }
        if (s + 1 < slices) stash((s + 1) & 1);
        __syncthreads();
      }
      auto at = [](const float2 (&r)[TN / 2], int j) { return j & 1 ? r[j >> 1].y : r[j >> 1].x; };
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const int m = m0 + row_of(i, ty);
        if (m >= M) continue;
        if constexpr (EPI == kEpiGlu) {
#pragma unroll
          for (int j = 0; j < HN; ++j) {
            const int n = n0 + tx * HN + j;
            if (n >= a.N) continue;
            const size_t row = (size_t)e * a.C + m;
            const float g = at(acc[i], j), u = at(acc[i], HN + j);
            if (pre_out) { pre_out[row * 2 * a.N + n] = g; pre_out[row * 2 * a.N + a.N + n] = u; }
            out[row * a.N + n] = silu_mul<false>(g, u);
          }
        } else {
#pragma unroll
          for (int j = 0; j < TN; ++j) {
            const int n = n0 + col_of(j, tx);
            const float v = at(acc[i], j);
            if (n >= a.N) continue;
            if constexpr (EPI == kEpiDw) {
              float* o = out + ((size_t)e * a.M + m) * a.N + n;
              *o = a.accumulate ? *o + v : v;
            } else if constexpr (EPI == kEpiDact) {
              const size_t row = ((size_t)e * a.C + m) * 2 * a.N;
              float dg, du;
              dact<false>(v, pre_in[row + n], pre_in[row + a.N + n], dg, du);
              out[row + n] = dg; out[row + a.N + n] = du;
            } else {
              out[((size_t)e * a.C + m) * a.N + n] = v;
            }
          }
        }
      }
    }
    first += n_tiles;
  }
  if constexpr (EPI != kEpiDw) {
    const int worker = blockIdx.x * 256 + tid, workers = gridDim.x * 256;
    expert_zero_behind(a, srows, (char*)out, sizeof(float) * (size_t)(EPI == kEpiDact ? 2 * a.N : a.N), 1, worker, workers);
    if (EPI == kEpiGlu && pre_out) expert_zero_behind(a, srows, (char*)pre_out, sizeof(float) * 2 * (size_t)a.N, 1, worker, workers);
  }
}

}  // namespace msr
