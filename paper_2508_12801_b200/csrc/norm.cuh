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
// All of it is bound by HBM.  A producer warp streams the rows of the coming tokens into a ring of row buffers in shared
// memory (bulk copies on mbarriers), so the loads never wait for the two reductions a token goes through; a group of G
// threads owns a token at a time, V 16-byte vectors of the row each, weights packed in registers from token to token.
#pragma once
#include "common.cuh"

namespace msr {

struct NormArgs {
  int T, d, nvec;               // nvec = 16-byte vectors of a row
  int rows_per_gate;            // gate row of token i = i / rows_per_gate (only with a gate)
  float eps, w_offset, res_scale;
  const void *w_post, *gate, *w_pre;   // io type, may be null: that step is left out
};

constexpr int kNormSlots = 32, kNormWarps = 16;
struct NormSmem {
  uint64_t full[kNormSlots], empty[kNormSlots];
  float weight[kNormSlots][kMaxK];     // combine weights of the token whose residual row is in this slot
  int count[kNormSlots];               // and how many expert rows follow
  float red[2][3][kNormWarps];
};

// The consumers' side of the ring and their sums.  A wait that gives up leaves ok false: the thread goes on through the
// barriers without waiting or storing, so that all end together.
struct NormGroup {
  NormSmem& sm; const unsigned char* ring; uint32_t row_bytes; int slots, G, warps;
  int s = 0, turn = 0; uint32_t ph = 0; bool ok = true;
  __device__ NormGroup(NormSmem& m, const unsigned char* r, uint32_t b, int n, int g) : sm(m), ring(r), row_bytes(b), slots(n), G(g), warps(g >> 5) {}
  __device__ const uint4* row() {                                  // the next row, once it has landed
    if (ok) ok = mbar_wait_bounded(&sm.full[s], ph);
    return reinterpret_cast<const uint4*>(ring + (size_t)s * row_bytes);
  }
  __device__ void release() {                                      // the row has been read by this warp
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(&sm.empty[s]);
    if (++s == slots) { s = 0; ph ^= 1; }
  }
  // Sums of N values over the group, the same on every thread and in the same order every time.  Two buffers in turn, so one
  // barrier a sum is enough.
  template <int N>
  __device__ void sum(float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = warp_sum(v[i]);
    if (warps == 1) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) sm.red[turn][i][warp] = v[i];
    asm volatile("bar.sync 1, %0;" ::"r"(G) : "memory");
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float t = 0.f;
#pragma unroll
      for (int w = 0; w < kNormWarps; w += 4)
        if (w < warps) {
          const float4 x = *reinterpret_cast<const float4*>(&sm.red[turn][i][w]);
          t += (x.x + x.y) + (x.z + x.w);                          // warps that do not exist left zeros
        }
      v[i] = t;
    }
    turn ^= 1;
  }
};
// The producer's side: lane 0 of its warp.
struct NormFeed {
  NormSmem& sm; unsigned char* ring; uint32_t row_bytes; int slots;
  int s = 0; uint32_t ph = 1; bool ok = true;
  __device__ NormFeed(NormSmem& m, unsigned char* r, uint32_t b, int n) : sm(m), ring(r), row_bytes(b), slots(n) {}
  __device__ bool room() { return ok = ok && mbar_wait_bounded(&sm.empty[s], ph); }
  __device__ void row(const void* src) {
    mbar_expect_tx(&sm.full[s], row_bytes);
    bulk_g2s(ring + (size_t)s * row_bytes, src, row_bytes, &sm.full[s]);
    if (++s == slots) { s = 0; ph ^= 1; }
  }
};
__device__ __forceinline__ void norm_ring_init(NormSmem& sm, int slots, int warps) {
  if (threadIdx.x == 0) {
    for (int i = 0; i < slots; ++i) { mbar_init(&sm.full[i], 1); mbar_init(&sm.empty[i], warps); }
    fence_barrier_init();
  }
  for (int i = threadIdx.x; i < 2 * 3 * kNormWarps; i += blockDim.x) (&sm.red[0][0][0])[i] = 0.f;
  __syncthreads();
}
__device__ __forceinline__ void norm_ring_end(bool ok, unsigned* error_flag) {
  if (!ok && (threadIdx.x & 31) == 0) {
    atomicOr(error_flag, 4u);
    for (int i = 0; i < 1000; ++i) __nanosleep(1000);   // a wait gave up: let the copies that were in flight land
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

// SRC 0: no y (r' = res_scale * r), 1: y given, 2: y combined from the expert buffers.  The last warp is the producer.
template <typename T, int V, int SRC, int MaxG, int Ctas>
__global__ void __launch_bounds__(MaxG + 32, Ctas)
norm_fwd_kernel(const T* y_in, const T* src, const int32_t* __restrict__ expert_idx, const int32_t* __restrict__ slot_idx,
                const float* __restrict__ gate_w, int E, int k, int C, const T* residual, T* __restrict__ y_out, T* r_out,
                T* __restrict__ h, NormArgs a, int slots, unsigned* error_flag) {
  constexpr int N = Vec16<T>::N;
  extern __shared__ __align__(128) unsigned char norm_ring[];
  __shared__ NormSmem sm;
  const int G = blockDim.x - 32, lane = threadIdx.x & 31;
  const uint32_t row_bytes = (uint32_t)a.nvec * 16;
  norm_ring_init(sm, slots, G >> 5);
  if (threadIdx.x >= G) {
    // ---- producer: residual row first, then y or the rows of the token's experts in ascending order -------------------
    NormFeed feed(sm, norm_ring, row_bytes, slots);
    int e = 0, sl = 0; float w = 0.f;
    auto pairs_of = [&](int tok) {
      if (SRC == 2 && lane < k && tok < a.T) {
        e = __ldg(expert_idx + (size_t)tok * k + lane); sl = __ldg(slot_idx + (size_t)tok * k + lane);
        w = gate_w ? __ldg(gate_w + (size_t)tok * k + lane) : 1.f;
      }
    };
    pairs_of(blockIdx.x);
    for (int tok = blockIdx.x; tok < a.T; tok += gridDim.x) {
      // an empty or surplus pair is neither read nor added
      const bool valid = SRC == 2 && lane < k && e >= 0 && e < E && sl >= 0 && sl < C;
      const unsigned mask = __ballot_sync(0xffffffffu, valid);
      const char* at = valid ? reinterpret_cast<const char*>(src) + ((size_t)e * C + sl) * row_bytes : nullptr;
      bool go = true;
      if (lane == 0) go = feed.room();
      go = __shfl_sync(0xffffffffu, go, 0);
      if (!go) break;
      const int first = __shfl_sync(0xffffffffu, feed.s, 0);
      if (SRC == 2) {
        if (valid) sm.weight[first][__popc(mask & ((1u << lane) - 1))] = w;
        if (lane == 0) sm.count[first] = __popc(mask);
        __syncwarp();
        pairs_of(tok + gridDim.x);                                 // the next token's, while this one's rows are on the way
      }
      if (lane == 0) {
        feed.row(residual + (size_t)tok * a.d);
        if (SRC == 1 && feed.room()) feed.row(y_in + (size_t)tok * a.d);
      }
      if (SRC == 2)
        for (unsigned m = mask; m; m &= m - 1) {
          const unsigned long long p = __shfl_sync(0xffffffffu, (unsigned long long)at, __ffs(m) - 1);
          if (lane == 0 && feed.room()) feed.row((const void*)p);
        }
      if (!__shfl_sync(0xffffffffu, feed.ok, 0)) break;
    }
    norm_ring_end(feed.ok || lane != 0, error_flag);
    return;
  }
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
  NormGroup group(sm, norm_ring, row_bytes, slots, G);
  const float inv_d = 1.f / (float)a.d;
  int gate_row = -1;
  for (int tok = blockIdx.x; tok < a.T; tok += gridDim.x) {
    const size_t row = (size_t)tok * a.d;
    uint4 rv[V], yv[V];
    {
      const uint4* p = group.row();
#pragma unroll
      for (int j = 0; j < V; ++j) { const int v = threadIdx.x + j * G; rv[j] = v < a.nvec ? p[v] : zero; }
    }
    if (SRC == 2) {
      const int n = sm.count[group.s];
      float wgt[kMaxK];
#pragma unroll
      for (int c = 0; c < kMaxK; ++c) wgt[c] = sm.weight[group.s][c];
      group.release();
      float acc[V][N];
#pragma unroll
      for (int j = 0; j < V; ++j)
#pragma unroll
        for (int i = 0; i < N; ++i) acc[j][i] = 0.f;
#pragma unroll
      for (int c = 0; c < kMaxK; ++c)
        if (c < n) {
          const uint4* p = group.row();
#pragma unroll
          for (int j = 0; j < V; ++j) {
            const int v = threadIdx.x + j * G;
            float x[N];
            Vec16<T>::unpack(v < a.nvec ? p[v] : zero, x);
#pragma unroll
            for (int i = 0; i < N; ++i) acc[j][i] = fmaf(wgt[c], x[i], acc[j][i]);
          }
          group.release();
        }
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int v = threadIdx.x + j * G;
        yv[j] = pack16<T>(acc[j]);
        if (y_out && v < a.nvec && group.ok) *reinterpret_cast<uint4*>(y_out + row + (size_t)v * N) = yv[j];
      }
    } else {
      group.release();
      if (SRC == 1) {
        const uint4* p = group.row();
#pragma unroll
        for (int j = 0; j < V; ++j) { const int v = threadIdx.x + j * G; yv[j] = v < a.nvec ? p[v] : zero; }
        group.release();
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
      group.sum(s);
      inv_y = rsqrtf(s[0] * inv_d + a.eps);
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
        if (r_out && group.ok) *reinterpret_cast<uint4*>(r_out + row + (size_t)v * N) = rv[j];
        Vec16<T>::unpack(rv[j], r);
#pragma unroll
        for (int i = 0; i < N; ++i) s[0] = fmaf(r[i], r[i], s[0]);
      }
    }
    if (h) {
      group.sum(s);
      const float inv = rsqrtf(s[0] * inv_d + a.eps);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int v = threadIdx.x + j * G;
        float r[N], w[N];
        Vec16<T>::unpack(rv[j], r);
        unpack_w<T>(wpre[j], a.w_offset, w);
#pragma unroll
        for (int i = 0; i < N; ++i) r[i] = r[i] * inv * w[i];
        if (v < a.nvec && group.ok) Vec16<T>::store(h + row + (size_t)v * N, r);
      }
    }
  }
  norm_ring_end(group.ok, error_flag);
}

// Backward.  Tokens are cut into units that stay within one gate row; a CTA walks units with a fixed stride and keeps the
// column sums of its rows in registers: those of the two weights over all its units, those of the gate until the unit ends.
// Partial sums go to the workspace (or, where a unit is a whole gate row, straight to dgate) and a second kernel adds them
// in a fixed order, so results repeat bit for bit.
struct NormUnits { int n_units, per_gate, rows; };     // units in all, units of a gate row, rows of a unit
__device__ __forceinline__ void unit_range(const NormUnits& u, const NormArgs& a, int unit, int& grow, int& t0, int& t1) {
  grow = unit / u.per_gate;
  const long long start = (long long)grow * a.rows_per_gate + (long long)(unit - grow * u.per_gate) * u.rows;
  const long long end = min((long long)a.T, min(((long long)grow + 1) * a.rows_per_gate, start + u.rows));
  t0 = (int)min(start, (long long)a.T); t1 = (int)end;
}

template <typename T, int V, int MaxG, int Ctas>
__global__ void __launch_bounds__(MaxG + 32, Ctas)
norm_bwd_kernel(const T* dr_out, const T* dh, const T* y, const T* r_out, T* __restrict__ dy, T* dr,
                float* __restrict__ part_post, float* __restrict__ part_pre, float* __restrict__ part_gate, NormUnits u, NormArgs a,
                int slots, unsigned* error_flag) {
  constexpr int N = Vec16<T>::N;
  extern __shared__ __align__(128) unsigned char norm_ring[];
  __shared__ NormSmem sm;
  const int G = blockDim.x - 32;
  const uint32_t row_bytes = (uint32_t)a.nvec * 16;
  const uint4 zero = make_uint4(0, 0, 0, 0);
  const float inv_d = 1.f / (float)a.d;
  norm_ring_init(sm, slots, G >> 5);
  int grow, t0, t1;
  if (threadIdx.x >= G) {
    if (threadIdx.x == G) {
      NormFeed feed(sm, norm_ring, row_bytes, slots);
      for (int unit = blockIdx.x; unit < u.n_units && feed.ok; unit += gridDim.x) {
        unit_range(u, a, unit, grow, t0, t1);
        for (int tok = t0; tok < t1 && feed.ok; ++tok) {
          const size_t row = (size_t)tok * a.d;
          if (dh) { if (feed.room()) feed.row(r_out + row); if (feed.room()) feed.row(dh + row); }
          if (y && feed.room()) feed.row(y + row);
          if (dr_out && feed.room()) feed.row(dr_out + row);
        }
      }
      norm_ring_end(feed.ok, error_flag);
    }
    return;
  }
  NormGroup group(sm, norm_ring, row_bytes, slots, G);
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
    unit_range(u, a, unit, grow, t0, t1);
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
      auto take = [&](uint4 (&to)[V], bool given) {
        if (given) {
          const uint4* p = group.row();
#pragma unroll
          for (int j = 0; j < V; ++j) { const int v = threadIdx.x + j * G; to[j] = v < a.nvec ? p[v] : zero; }
          group.release();
        } else {
#pragma unroll
          for (int j = 0; j < V; ++j) to[j] = zero;
        }
      };
      take(rr, dh != nullptr); take(rdh, dh != nullptr); take(ry, y != nullptr); take(rdo, dr_out != nullptr);
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
      group.sum(s);
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
        if (v < a.nvec && group.ok) Vec16<T>::store(dr + row + (size_t)v * N, out);
      }
      if (dy) {
        float c_y = 0.f;
        if (a.w_post) { group.sum(b); c_y = b[0] * inv_y * inv_y * inv_d; }
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const int v = threadIdx.x + j * G;
          float yy[N], wp[N], out[N];
          Vec16<T>::unpack(ry[j], yy); unpack_w<T>(wpost[j], a.w_offset, wp);
#pragma unroll
          for (int i = 0; i < N; ++i) out[i] = a.w_post ? inv_y * (tot[j][i] * wp[i] - yy[i] * c_y) : tot[j][i];
          if (v < a.nvec && group.ok) Vec16<T>::store(dy + row + (size_t)v * N, out);
        }
      }
    }
    if (part_gate)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int v = threadIdx.x + j * G;
        if (v < a.nvec)
#pragma unroll
          for (int i = 0; i < N; i += 4)
            *reinterpret_cast<float4*>(part_gate + (size_t)unit * a.d + (size_t)v * N + i) = make_float4(agate[j][i], agate[j][i + 1], agate[j][i + 2], agate[j][i + 3]);
      }
  }
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int v = threadIdx.x + j * G;
    if (v < a.nvec)
#pragma unroll
      for (int i = 0; i < N; i += 4) {
        const size_t at = (size_t)blockIdx.x * a.d + (size_t)v * N + i;
        if (part_post) *reinterpret_cast<float4*>(part_post + at) = make_float4(apost[j][i], apost[j][i + 1], apost[j][i + 2], apost[j][i + 3]);
        if (part_pre) *reinterpret_cast<float4*>(part_pre + at) = make_float4(apre[j][i], apre[j][i + 1], apre[j][i + 2], apre[j][i + 3]);
      }
  }
  norm_ring_end(group.ok, error_flag);
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
