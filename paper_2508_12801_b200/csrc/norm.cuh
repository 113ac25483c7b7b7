// Norms before and after a block, fused with its gate and the scaled residual; optionally with combine in front.
//
//   y_i  = combine of the token's expert rows (Eq. 1), or given           rounded to the I/O type
//   n_i  = y_i / rms(y_i) * (offset + w_post)                             rms(v)^2 = mean(v^2) + eps
//   r'_i = res_scale * r_i + gate_(i / rows_per_gate) * n_i               rounded to the I/O type
//   h_i  = r'_i / rms(r'_i) * (offset + w_pre)
//
// Both norms take the rounded value that is also returned, so that the backward pass, which is handed those, forms the
// same statistics again instead of having them stored.  Sums are fp32.
//
// All of it is bound by HBM.  A group of G threads (one CTA) owns a row: V 16-byte vectors per thread, every load of the
// row issued before the first reduction; weights stay packed in registers from row to row.
#pragma once
#include "common.cuh"

namespace msr {

struct NormArgs {
  int T, d, nvec;               // nvec = 16-byte vectors of a row
  int rows_per_gate;            // gate row of token i = i / rows_per_gate (only with a gate)
  float eps, w_offset, res_scale;
  const void *w_post, *gate, *w_pre;   // io type, may be null: that step is left out
};

// Sums of N values over the CTA's threads, the same on every thread and in the same order every time.
template <int N>
__device__ __forceinline__ void group_sum(float (&v)[N], float* red, int warps) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = warp_sum(v[i]);
  if (warps > 1) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    __syncthreads();                       // the last sum's readers are done with red
    if (lane == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) red[warp * N + i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float p = lane < warps ? red[lane * N + i] : 0.f;
      v[i] = warp_sum(p);
    }
  }
}

template <typename T>
__device__ __forceinline__ void unpack_w(const uint4& raw, float offset, float (&w)[Vec16<T>::N]) {
  Vec16<T>::unpack(raw, w);
#pragma unroll
  for (int j = 0; j < Vec16<T>::N; ++j) w[j] += offset;
}
template <typename T> __device__ __forceinline__ uint4 pack16(const float (&f)[Vec16<T>::N]);
template <> __device__ __forceinline__ uint4 pack16<float>(const float (&f)[4]) {
  return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}
template <> __device__ __forceinline__ uint4 pack16<__nv_bfloat16>(const float (&f)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
    w[i] = *reinterpret_cast<uint32_t*>(&h);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// SRC 0: no y (r' = res_scale * r), 1: y given, 2: y combined from the expert buffers
template <typename T, int V, int SRC, int MaxG>
__global__ void __launch_bounds__(MaxG)
norm_fwd_kernel(const T* __restrict__ y_in, const T* __restrict__ src, const int32_t* __restrict__ expert_idx,
                                const int32_t* __restrict__ slot_idx, const float* __restrict__ gate_w, int E, int k, int C,
                                const T* residual, T* __restrict__ y_out, T* r_out, T* __restrict__ h, NormArgs a) {
  constexpr int N = Vec16<T>::N;
  __shared__ float red[32];
  const int G = blockDim.x, warps = G >> 5, lane = threadIdx.x & 31;
  const uint4 zero = make_uint4(0, 0, 0, 0);
  uint4 wpost[V], wpre[V], gat[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int v = threadIdx.x + j * G;
    const bool in = v < a.nvec;
    wpost[j] = (in && a.w_post) ? ldg16((const uint4*)a.w_post + v) : zero;
    wpre[j] = (in && a.w_pre) ? ldg16((const uint4*)a.w_pre + v) : zero;
    gat[j] = zero;
  }
  int gate_row = -1;
  for (int tok = blockIdx.x; tok < a.T; tok += gridDim.x) {
    const size_t row = (size_t)tok * a.d;
    uint4 rv[V], yv[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int v = threadIdx.x + j * G;
      // no __ldg: r_out may be the residual's own buffer (this row is read here before it is written below)
      rv[j] = v < a.nvec ? *reinterpret_cast<const uint4*>(residual + row + (size_t)v * N) : zero;
      if (SRC == 1) yv[j] = v < a.nvec ? ldg16(y_in + row + (size_t)v * N) : zero;
    }
    if (SRC == 2) {
      long long my_off = -1; float my_w = 0.f;
      if (lane < k) {
        const int e = __ldg(expert_idx + (size_t)tok * k + lane), sl = __ldg(slot_idx + (size_t)tok * k + lane);
        const bool valid = e >= 0 && e < E && sl >= 0 && sl < C;   // an empty or surplus pair is neither read nor added
        my_off = valid ? ((long long)e * C + sl) * (long long)a.d : -1;
        my_w = !valid ? 0.f : gate_w ? __ldg(gate_w + (size_t)tok * k + lane) : 1.f;
      }
      long long off[kMaxK]; float wgt[kMaxK];
#pragma unroll
      for (int c = 0; c < kMaxK; ++c) { off[c] = __shfl_sync(0xffffffffu, my_off, c); wgt[c] = __shfl_sync(0xffffffffu, my_w, c); }
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int v = threadIdx.x + j * G;
        uint4 raw[kMaxK];
#pragma unroll
        for (int c = 0; c < kMaxK; ++c)
          if (c < k && off[c] >= 0 && v < a.nvec) raw[c] = ldg16(src + off[c] + (size_t)v * N);
        float acc[N];
#pragma unroll
        for (int i = 0; i < N; ++i) acc[i] = 0.f;
#pragma unroll
        for (int c = 0; c < kMaxK; ++c)
          if (c < k && off[c] >= 0 && v < a.nvec) {
            float x[N];
            Vec16<T>::unpack(raw[c], x);
#pragma unroll
            for (int i = 0; i < N; ++i) acc[i] = fmaf(wgt[c], x[i], acc[i]);
          }
        yv[j] = pack16<T>(acc);
        if (y_out && v < a.nvec) *reinterpret_cast<uint4*>(y_out + row + (size_t)v * N) = yv[j];
      }
    }
    if (SRC && a.gate) {
      const int g = tok / a.rows_per_gate;
      if (g != gate_row) {
        gate_row = g;
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const int v = threadIdx.x + j * G;
          if (v < a.nvec) gat[j] = ldg16((const T*)a.gate + (size_t)g * a.d + (size_t)v * N);
        }
      }
    }
    float inv_y = 1.f;
    if (SRC && a.w_post) {
      float s[1] = {0.f};
#pragma unroll
      for (int j = 0; j < V; ++j) {
        float y[N];
        Vec16<T>::unpack(yv[j], y);
#pragma unroll
        for (int i = 0; i < N; ++i) s[0] = fmaf(y[i], y[i], s[0]);
      }
      group_sum<1>(s, red, warps);
      inv_y = rsqrtf(s[0] / (float)a.d + a.eps);
    }
    float s[1] = {0.f};
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int v = threadIdx.x + j * G;
      float r[N], y[N], w[N], g[N];
      Vec16<T>::unpack(rv[j], r);
      if (SRC) Vec16<T>::unpack(yv[j], y);
      unpack_w<T>(wpost[j], a.w_offset, w);
      Vec16<T>::unpack(gat[j], g);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        float n = 0.f;
        if (SRC) {
          n = y[i];
          if (a.w_post) n = n * inv_y * w[i];
          if (a.gate) n *= g[i];
        }
        r[i] = SRC ? fmaf(a.res_scale, r[i], n) : a.res_scale * r[i];
      }
      rv[j] = pack16<T>(r);
      if (v < a.nvec) {
        if (r_out) *reinterpret_cast<uint4*>(r_out + row + (size_t)v * N) = rv[j];
        Vec16<T>::unpack(rv[j], r);
#pragma unroll
        for (int i = 0; i < N; ++i) s[0] = fmaf(r[i], r[i], s[0]);
      }
    }
    if (h) {
      group_sum<1>(s, red, warps);
      const float inv = rsqrtf(s[0] / (float)a.d + a.eps);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int v = threadIdx.x + j * G;
        float r[N], w[N];
        Vec16<T>::unpack(rv[j], r);
        unpack_w<T>(wpre[j], a.w_offset, w);
#pragma unroll
        for (int i = 0; i < N; ++i) r[i] = r[i] * inv * w[i];
        if (v < a.nvec) Vec16<T>::store(h + row + (size_t)v * N, r);
      }
    }
  }
}

// Backward.  Tokens are cut into units that stay within one gate row; a CTA walks units with a fixed stride and keeps the
// column sums of its rows in registers: those of the two weights over all its units, those of the gate until the unit ends.
// Partial sums go to the workspace (or, where a unit is a whole gate row, straight to dgate) and a second kernel adds them
// in a fixed order, so results repeat bit for bit.
struct NormUnits { int n_units, per_gate, rows; };     // units in all, units of a gate row, rows of a unit

template <typename T, int V, int MaxG>
__global__ void __launch_bounds__(MaxG)
norm_bwd_kernel(const T* dr_out, const T* __restrict__ dh, const T* __restrict__ y,
                                const T* __restrict__ r_out, T* __restrict__ dy, T* dr, float* __restrict__ part_post,
                                float* __restrict__ part_pre, float* __restrict__ part_gate, NormUnits u, NormArgs a) {
  constexpr int N = Vec16<T>::N;
  __shared__ float red[96];
  const int G = blockDim.x, warps = G >> 5;
  const uint4 zero = make_uint4(0, 0, 0, 0);
  const float inv_d = 1.f / (float)a.d;
  uint4 wpost[V], wpre[V], gat[V];
  float apost[V][N], apre[V][N], agate[V][N];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int v = threadIdx.x + j * G;
    const bool in = v < a.nvec;
    wpost[j] = (in && a.w_post) ? ldg16((const uint4*)a.w_post + v) : zero;
    wpre[j] = (in && a.w_pre) ? ldg16((const uint4*)a.w_pre + v) : zero;
    gat[j] = zero;
#pragma unroll
    for (int i = 0; i < N; ++i) apost[j][i] = apre[j][i] = 0.f;
  }
  for (int unit = blockIdx.x; unit < u.n_units; unit += gridDim.x) {
    const int grow = unit / u.per_gate;
    const int gate_end = min((long long)a.T, ((long long)grow + 1) * a.rows_per_gate);
    const int t0 = grow * a.rows_per_gate + (unit - grow * u.per_gate) * u.rows;
    const int t1 = min(gate_end, t0 + u.rows);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int v = threadIdx.x + j * G;
      if (a.gate && v < a.nvec) gat[j] = ldg16((const T*)a.gate + (size_t)grow * a.d + (size_t)v * N);
#pragma unroll
      for (int i = 0; i < N; ++i) agate[j][i] = 0.f;
    }
    for (int tok = t0; tok < t1; ++tok) {
      const size_t row = (size_t)tok * a.d;
      uint4 rdo[V], rdh[V], ry[V], rr[V];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int v = threadIdx.x + j * G;
        const bool in = v < a.nvec;
        const size_t at = row + (size_t)v * N;
        rdo[j] = (in && dr_out) ? *reinterpret_cast<const uint4*>(dr_out + at) : zero;   // dr may be the same buffer
        rdh[j] = (in && dh) ? ldg16(dh + at) : zero;
        rr[j] = (in && dh) ? ldg16(r_out + at) : zero;
        ry[j] = (in && y) ? ldg16(y + at) : zero;
      }
      float s[3] = {0.f, 0.f, 0.f};     // sum r^2, sum dh w r, sum y^2
#pragma unroll
      for (int j = 0; j < V; ++j) {
        float g[N], r[N], yy[N], w[N];
        Vec16<T>::unpack(rdh[j], g); Vec16<T>::unpack(rr[j], r); Vec16<T>::unpack(ry[j], yy);
        unpack_w<T>(wpre[j], a.w_offset, w);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          s[0] = fmaf(r[i], r[i], s[0]);
          s[1] = fmaf(g[i] * w[i], r[i], s[1]);
          s[2] = fmaf(yy[i], yy[i], s[2]);
        }
      }
      group_sum<3>(s, red, warps);
      const float inv_r = rsqrtf(s[0] * inv_d + a.eps), inv_y = rsqrtf(s[2] * inv_d + a.eps);
      const float c_r = s[1] * inv_r * inv_r * inv_d;       // mean(dh w r / rms) / rms
      float b[1] = {0.f};                                   // sum dn w_post y
      float tot[V][N];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int v = threadIdx.x + j * G;
        float o[N], g[N], r[N], w[N], yy[N], gt[N], wp[N], out[N];
        Vec16<T>::unpack(rdo[j], o); Vec16<T>::unpack(rdh[j], g); Vec16<T>::unpack(rr[j], r); Vec16<T>::unpack(ry[j], yy);
        unpack_w<T>(wpre[j], a.w_offset, w); unpack_w<T>(wpost[j], a.w_offset, wp); Vec16<T>::unpack(gat[j], gt);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float t = o[i] + inv_r * (g[i] * w[i] - r[i] * c_r);
          apre[j][i] = fmaf(g[i], r[i] * inv_r, apre[j][i]);
          out[i] = a.res_scale * t;
          const float yn = a.w_post ? yy[i] * inv_y : yy[i];
          agate[j][i] = fmaf(t, a.w_post ? yn * wp[i] : yn, agate[j][i]);
          const float dn = a.gate ? t * gt[i] : t;
          apost[j][i] = fmaf(dn, yn, apost[j][i]);
          tot[j][i] = dn;
          b[0] = fmaf(dn * wp[i], yy[i], b[0]);
        }
        if (v < a.nvec) Vec16<T>::store(dr + row + (size_t)v * N, out);
      }
      if (dy) {
        float c_y = 0.f;
        if (a.w_post) { group_sum<1>(b, red, warps); c_y = b[0] * inv_y * inv_y * inv_d; }
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const int v = threadIdx.x + j * G;
          float yy[N], wp[N], out[N];
          Vec16<T>::unpack(ry[j], yy); unpack_w<T>(wpost[j], a.w_offset, wp);
#pragma unroll
          for (int i = 0; i < N; ++i) out[i] = a.w_post ? inv_y * (tot[j][i] * wp[i] - yy[i] * c_y) : tot[j][i];
          if (v < a.nvec) Vec16<T>::store(dy + row + (size_t)v * N, out);
        }
      }
    }
    if (part_gate)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int v = threadIdx.x + j * G;
        if (v < a.nvec)
#pragma unroll
          for (int i = 0; i < N; ++i) part_gate[(size_t)unit * a.d + (size_t)v * N + i] = agate[j][i];
      }
  }
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int v = threadIdx.x + j * G;
    if (v < a.nvec)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (part_post) part_post[(size_t)blockIdx.x * a.d + (size_t)v * N + i] = apost[j][i];
        if (part_pre) part_pre[(size_t)blockIdx.x * a.d + (size_t)v * N + i] = apre[j][i];
      }
  }
}

// Column sums of up to 2 + gates partial matrices: blockIdx.y picks one (0: w_post, 1: w_pre, 2..: gate rows), a CTA 32
// columns, its 8 warps every eighth row; added in a fixed order.
__global__ void __launch_bounds__(256)
norm_reduce_kernel(const float* __restrict__ part_post, const float* __restrict__ part_pre, const float* __restrict__ part_gate,
                   float* __restrict__ dw_post, float* __restrict__ dw_pre, float* __restrict__ dgate, int rows, int per_gate, int d) {
  __shared__ float sm[8][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
  const int which = blockIdx.y;
  const float* p = which == 0 ? part_post : which == 1 ? part_pre : part_gate;
  float* o = which == 0 ? dw_post : which == 1 ? dw_pre : dgate;
  if (!p || !o) return;
  const size_t r0 = which < 2 ? 0 : (size_t)(which - 2) * per_gate;
  const int n = which < 2 ? rows : per_gate;
  float s = 0.f;
  if (col < d) {
#pragma unroll 4
    for (int r = warp; r < n; r += 8) s += p[(r0 + r) * d + col];
  }
  sm[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && col < d) {
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) t += sm[w][lane];
    o[(which < 2 ? 0 : (size_t)(which - 2) * d) + col] = t;
  }
}

}  // namespace msr
