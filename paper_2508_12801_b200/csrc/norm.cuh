// Norms before and after a block, fused with its gate and the scaled residual; optionally with combine in front.
//
//   y_i  = combine of the token's expert rows (Eq. 1), or given
//   n_i  = y_i / rms(y_i) * (offset + w_post)                             rms(v)^2 = mean(v^2) + eps
//   r'_i = res_scale * r_i + gate_(i / rows_per_gate) * n_i
//   h_i  = r'_i / rms(r'_i) * (offset + w_pre)
//
// A row passes through in fp32: y, r' and h are each rounded once, when they are stored, and the steps behind take the values
// before that.  The backward pass forms the statistics again from the stored rows instead of having them stored too.
//
// All of it is bound by HBM.  A producer warp streams the rows of the coming tokens into a ring of row buffers in shared
// memory (bulk copies on mbarriers), so the loads never wait for the two reductions a token goes through; a group of G
// threads owns a token at a time, V 16-byte vectors of the row each, weights in registers from token to token.
// T 65536, d 4096, bf16: with combine of k 8 930 us (6.9 TB/s where a plain copy, which writes a byte for each that it reads, makes
// 6.54: here nine rows are read for three written), without 350 us (6.1 TB/s), backward 640 us (5.0 TB/s).  The backward is short of
// issue slots and of registers: with the producer's warp a CTA has 17, five of them on one quarter of the SM, which leaves 96
// registers a thread, and its bf16 forms spill (72 bytes at d 4096, 570 at 8192, 1 900 at 16384, where it makes 3.1 and 1.2 TB/s).
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
  float red[2][4][kNormWarps];
};

// The consumers' side of the ring and their sums.  A wait that gives up leaves ok false: the thread goes on through the
// barriers without waiting or storing, so that all end together.
struct NormGroup {
  NormSmem& sm; const unsigned char* ring; uint32_t slot_bytes; int slots, G, warps;
  int s = 0, turn = 0; uint32_t ph = 0; bool ok = true;
  __device__ NormGroup(NormSmem& m, const unsigned char* r, uint32_t b, int n, int g) : sm(m), ring(r), slot_bytes(b), slots(n), G(g), warps(g >> 5) {}
  __device__ const uint4* take() {                                 // the next slot, once its rows have landed
    if (ok) ok = mbar_wait_bounded(&sm.full[s], ph);
    return reinterpret_cast<const uint4*>(ring + (uint32_t)s * slot_bytes);
  }
  // The slot has been read by this warp.  The copy that fills it next is the async proxy's: the fence keeps it behind these ordinary
  // reads, which the barrier alone does not (a load that was still on its way then met the rows of a later token).  It costs the
  // backward 1 to 4 %.
  __device__ void release() {
    fence_proxy_async();
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(&sm.empty[s]);
    if (++s == slots) { s = 0; ph ^= 1; }
  }
  // Sum over the group, the same on every thread and in the same order every time.  Two buffers in turn, so one barrier is
  // enough.
  __device__ float sum(float v) {
    v = warp_sum(v);
    if (warps == 1) return v;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0) sm.red[turn][0][warp] = v;
    asm volatile("bar.sync 1, %0;" ::"r"(G) : "memory");
    v = sm.red[turn][0][lane & (kNormWarps - 1)];                  // warps that do not exist left zeros
#pragma unroll
    for (int o = kNormWarps / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    turn ^= 1;
    return v;
  }
  // Three at once: the butterfly keeps half of the values on either side of the first two exchanges, so that a quarter of the
  // lanes ends up with each of them (6 shuffles instead of 15).
  __device__ void sum3(float& x, float& y, float& z) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const bool hi = lane & 16, odd = lane & 8;
    float p = hi ? z : x, q = hi ? 0.f : y;
    p += __shfl_xor_sync(0xffffffffu, hi ? x : z, 16);
    q += __shfl_xor_sync(0xffffffffu, hi ? y : 0.f, 16);
    float v = odd ? q : p;
    v += __shfl_xor_sync(0xffffffffu, odd ? p : q, 8);
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (warps > 1) {                                               // lane / 8: 0 x, 1 y, 2 z
      if ((lane & 7) == 0) sm.red[turn][lane >> 3][warp] = v;
      asm volatile("bar.sync 1, %0;" ::"r"(G) : "memory");
      const float2 t = *reinterpret_cast<const float2*>(&sm.red[turn][lane >> 3][(lane & 7) * 2]);
      v = t.x + t.y;
#pragma unroll
      for (int o = 4; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
      turn ^= 1;
    }
    x = __shfl_sync(0xffffffffu, v, 0); y = __shfl_sync(0xffffffffu, v, 8); z = __shfl_sync(0xffffffffu, v, 16);
  }
};
// The producer's side: lane 0 of its warp.
struct NormFeed {
  NormSmem& sm; unsigned char* ring; uint32_t slot_bytes; int slots;
  int s = 0; uint32_t ph = 1; bool ok = true;
  __device__ NormFeed(NormSmem& m, unsigned char* r, uint32_t b, int n) : sm(m), ring(r), slot_bytes(b), slots(n) {}
  __device__ bool room() { return ok = ok && mbar_wait_bounded(&sm.empty[s], ph); }
  __device__ void expect(uint32_t bytes) { mbar_expect_tx(&sm.full[s], bytes); }
  __device__ void row(uint32_t at, const void* src, uint32_t bytes) { bulk_g2s(ring + (uint32_t)s * slot_bytes + at, src, bytes, &sm.full[s]); }
  __device__ void next() { if (++s == slots) { s = 0; ph ^= 1; } }
};
__device__ __forceinline__ void norm_ring_init(NormSmem& sm, int slots, int warps) {
  if (threadIdx.x == 0) {
    for (int i = 0; i < slots; ++i) { mbar_init(&sm.full[i], 1); mbar_init(&sm.empty[i], warps); }
    fence_barrier_init();
  }
  for (int i = threadIdx.x; i < 2 * 4 * kNormWarps; i += blockDim.x) (&sm.red[0][0][0])[i] = 0.f;
  __syncthreads();
}
__device__ __forceinline__ void norm_ring_end(bool ok, unsigned* error_flag) {
  if (!ok && (threadIdx.x & 31) == 0) {
    atomicOr(error_flag, 4u);
    for (int i = 0; i < 1000; ++i) __nanosleep(1000);   // a wait gave up: let the copies that were in flight land
  }
}

// ---- pairs of floats: one instruction for two values ----------------------------------------------------------------
// The kernels are short of instruction slots before they are short of bandwidth (a token passes 8 to 48 bytes an element
// through some twenty operations each), so the arithmetic is done on packed pairs.
template <typename T> __device__ __forceinline__ void unpack2(const uint4& v, float2 (&f)[Vec16<T>::N / 2]);
template <> __device__ __forceinline__ void unpack2<float>(const uint4& v, float2 (&f)[2]) {
  f[0] = make_float2(__uint_as_float(v.x), __uint_as_float(v.y)); f[1] = make_float2(__uint_as_float(v.z), __uint_as_float(v.w));
}
template <> __device__ __forceinline__ void unpack2<__nv_bfloat16>(const uint4& v, float2 (&f)[4]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}
template <typename T> __device__ __forceinline__ uint4 pack2(const float2 (&f)[Vec16<T>::N / 2]);
template <> __device__ __forceinline__ uint4 pack2<float>(const float2 (&f)[2]) {
  return make_uint4(__float_as_uint(f[0].x), __float_as_uint(f[0].y), __float_as_uint(f[1].x), __float_as_uint(f[1].y));
}
template <> __device__ __forceinline__ uint4 pack2<__nv_bfloat16>(const float2 (&f)[4]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    __nv_bfloat162 h = __floats2bfloat162_rn(f[i].x, f[i].y);
    w[i] = *reinterpret_cast<uint32_t*>(&h);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// vector v of a weight row (offset added), ones without one
template <typename T>
__device__ __forceinline__ void load_weight(const void* w, size_t v, bool in, float offset, float2 (&f)[Vec16<T>::N / 2]) {
  if (w && in) {
    unpack2<T>(ldg16((const uint4*)w + v), f);
#pragma unroll
    for (int i = 0; i < Vec16<T>::N / 2; ++i) f[i] = add2(f[i], both(offset));
  } else {
#pragma unroll
    for (int i = 0; i < Vec16<T>::N / 2; ++i) f[i] = both(1.f);
  }
}

// SRC 0: no y (r' = res_scale * r), 1: y given, 2: y combined from the expert buffers.  Full: the threads' vectors are exactly
// the row.  The last warp is the producer.  A ring slot holds a token's rows, or one row each where their number varies (SRC 2).
template <typename T, int V, int SRC, bool Full, int MaxG, int Ctas>
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
    constexpr uint32_t kRows = SRC == 1 ? 2 : 1;
    NormFeed feed(sm, norm_ring, row_bytes * kRows, slots);
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
        feed.expect(row_bytes * kRows);
        feed.row(0, residual + (size_t)tok * a.d, row_bytes);
        if (SRC == 1) feed.row(row_bytes, y_in + (size_t)tok * a.d, row_bytes);
        feed.next();
      }
      if (SRC == 2)
        for (unsigned m = mask; m; m &= m - 1) {
          const unsigned long long p = __shfl_sync(0xffffffffu, (unsigned long long)at, __ffs(m) - 1);
          if (lane == 0 && feed.room()) { feed.expect(row_bytes); feed.row(0, (const void*)p, row_bytes); feed.next(); }
        }
      if (!__shfl_sync(0xffffffffu, feed.ok, 0)) break;
    }
    norm_ring_end(feed.ok || lane != 0, error_flag);
    return;
  }
  constexpr int P = N / 2;
  const uint4 zero = make_uint4(0, 0, 0, 0);
  auto mine = [&](int v) { return Full || v < a.nvec; };
  float2 wpre[V][P], gw[V][P];                          // gw: after-norm weight times gate, per gate row
  auto gate_weights = [&](int g) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int v = threadIdx.x + j * G;
      float2 x[P];
      load_weight<T>(a.w_post, v, mine(v), a.w_offset, gw[j]);
      load_weight<T>(a.gate, (size_t)g * a.nvec + v, mine(v), 0.f, x);
#pragma unroll
      for (int i = 0; i < P; ++i) gw[j][i] = mul2(gw[j][i], x[i]);
    }
  };
#pragma unroll
  for (int j = 0; j < V; ++j) load_weight<T>(a.w_pre, threadIdx.x + j * G, mine(threadIdx.x + j * G), a.w_offset, wpre[j]);
  NormGroup group(sm, norm_ring, SRC == 1 ? 2 * row_bytes : row_bytes, slots, G);
  const float inv_d = 1.f / (float)a.d;
  const float2 scale = both(a.res_scale);
  long long gate_end = 0;                               // first token behind the present gate row
  for (int tok = blockIdx.x; tok < a.T; tok += gridDim.x) {
    const size_t row = (size_t)tok * a.d;
    float2 r[V][P], y[V][P];
    {
      const uint4* p = group.take();
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int v = threadIdx.x + j * G;
        unpack2<T>(mine(v) ? p[v] : zero, r[j]);
        if (SRC == 1) unpack2<T>(mine(v) ? p[a.nvec + v] : zero, y[j]);
      }
    }
    if (SRC == 2) {
      const int n = sm.count[group.s];
      float wgt[kMaxK];
#pragma unroll
      for (int c = 0; c < kMaxK; ++c) wgt[c] = sm.weight[group.s][c];
      group.release();
#pragma unroll
      for (int j = 0; j < V; ++j)
#pragma unroll
        for (int i = 0; i < P; ++i) y[j][i] = both(0.f);
#pragma unroll
      for (int c = 0; c < kMaxK; ++c)
        if (c < n) {
          const uint4* p = group.take();
#pragma unroll
          for (int j = 0; j < V; ++j) {
            const int v = threadIdx.x + j * G;
            float2 x[P];
            unpack2<T>(mine(v) ? p[v] : zero, x);
#pragma unroll
            for (int i = 0; i < P; ++i) y[j][i] = fma2(both(wgt[c]), x[i], y[j][i]);
          }
          group.release();
        }
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int v = threadIdx.x + j * G;
        if (y_out && mine(v) && group.ok) __stcs(reinterpret_cast<uint4*>(y_out + row + (size_t)v * N), pack2<T>(y[j]));
      }
    } else {
      group.release();
    }
    if (SRC && tok >= gate_end) {
      const int g = a.gate ? tok / a.rows_per_gate : 0;
      gate_end = a.gate ? ((long long)g + 1) * a.rows_per_gate : a.T;
      gate_weights(g);
    }
    float inv_y = 1.f;
    if (SRC && a.w_post) {
      float2 s = both(0.f);
#pragma unroll
      for (int j = 0; j < V; ++j)
#pragma unroll
        for (int i = 0; i < P; ++i) s = fma2(y[j][i], y[j][i], s);
      inv_y = rsqrtf(group.sum(s.x + s.y) * inv_d + a.eps);
    }
    float2 s = both(0.f);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int v = threadIdx.x + j * G;
#pragma unroll
      for (int i = 0; i < P; ++i) {
        r[j][i] = mul2(scale, r[j][i]);
        if (SRC) r[j][i] = fma2(mul2(y[j][i], both(inv_y)), gw[j][i], r[j][i]);
        s = fma2(r[j][i], r[j][i], s);
      }
      if (r_out && mine(v) && group.ok) __stcs(reinterpret_cast<uint4*>(r_out + row + (size_t)v * N), pack2<T>(r[j]));
    }
    if (h) {
      const float2 inv = both(rsqrtf(group.sum(s.x + s.y) * inv_d + a.eps));
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int v = threadIdx.x + j * G;
#pragma unroll
        for (int i = 0; i < P; ++i) r[j][i] = mul2(mul2(r[j][i], inv), wpre[j][i]);
        if (mine(v) && group.ok) __stcs(reinterpret_cast<uint4*>(h + row + (size_t)v * N), pack2<T>(r[j]));
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

template <typename T, int V, bool Full, int MaxG, int Ctas>
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
  const bool dh_given = dh != nullptr, y_given = y != nullptr, dro_given = dr_out != nullptr;
  // a slot holds the token's rows that are given: r', dh, y, dr'
  const uint32_t at_y = dh_given ? 2 * a.nvec : 0, at_o = at_y + (y_given ? a.nvec : 0), rows = (dh_given ? 2 : 0) + (y_given ? 1 : 0) + (dro_given ? 1 : 0);
  int grow, t0, t1;
  if (threadIdx.x >= G) {
    if (threadIdx.x == G) {
      NormFeed feed(sm, norm_ring, rows * row_bytes, slots);
      for (int unit = blockIdx.x; unit < u.n_units && feed.ok; unit += gridDim.x) {
        unit_range(u, a, unit, grow, t0, t1);
        for (int tok = t0; rows && tok < t1 && feed.room(); ++tok) {
          const size_t row = (size_t)tok * a.d;
          feed.expect(rows * row_bytes);
          if (dh_given) { feed.row(0, r_out + row, row_bytes); feed.row(row_bytes, dh + row, row_bytes); }
          if (y_given) feed.row(at_y * 16, y + row, row_bytes);
          if (dro_given) feed.row(at_o * 16, dr_out + row, row_bytes);
          feed.next();
        }
      }
      norm_ring_end(feed.ok, error_flag);
    }
    return;
  }
  constexpr int P = N / 2;
  NormGroup group(sm, norm_ring, rows * row_bytes, slots, G);
  auto mine = [&](int v) { return Full || v < a.nvec; };
  // Per column only two sums run along the tokens: S = sum dr y / rms(y) (within a gate row: dgate = w_post S, and gate S goes
  // to dw_post, apost, when the unit ends) and dw_pre.
  float2 wpre[V][P], gw[V][P], acc[V][P], apre[V][P], apost[V][P];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    load_weight<T>(a.w_pre, threadIdx.x + j * G, mine(threadIdx.x + j * G), a.w_offset, wpre[j]);
#pragma unroll
    for (int i = 0; i < P; ++i) apost[j][i] = apre[j][i] = both(0.f);
  }
  const float2 scale = both(a.res_scale);
  for (int unit = blockIdx.x; unit < u.n_units; unit += gridDim.x) {
    unit_range(u, a, unit, grow, t0, t1);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int v = threadIdx.x + j * G;
      float2 x[P];
      load_weight<T>(a.w_post, v, mine(v), a.w_offset, gw[j]);
      load_weight<T>(a.gate, (size_t)grow * a.nvec + v, mine(v), 0.f, x);
#pragma unroll
      for (int i = 0; i < P; ++i) { gw[j][i] = mul2(gw[j][i], x[i]); acc[j][i] = both(0.f); }
    }
    for (int tok = t0; tok < t1; ++tok) {
      const size_t row = (size_t)tok * a.d;
      float2 o[V][P], g[V][P], r[V][P], y[V][P];
      auto load = [&](float2 (&to)[V][P], const uint4* p, bool given) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const int v = threadIdx.x + j * G;
          unpack2<T>(given && mine(v) ? p[v] : zero, to[j]);
        }
      };
      if (rows) {
        const uint4* p = group.take();
        load(r, p, dh_given); load(g, p + a.nvec, dh_given); load(y, p + at_y, y_given); load(o, p + at_o, dro_given);
        group.release();
      } else {
        load(r, nullptr, false); load(g, nullptr, false); load(y, nullptr, false); load(o, nullptr, false);
      }
      float2 sr = both(0.f), sg = both(0.f), sy = both(0.f);      // sum r^2, sum dh w r, sum y^2
      float2 pre[V][P];
#pragma unroll
      for (int j = 0; j < V; ++j)
#pragma unroll
        for (int i = 0; i < P; ++i) {
          pre[j][i] = mul2(g[j][i], wpre[j][i]);
          sr = fma2(r[j][i], r[j][i], sr);
          sg = fma2(pre[j][i], r[j][i], sg);
          sy = fma2(y[j][i], y[j][i], sy);
        }
      float s0 = sr.x + sr.y, s1 = sg.x + sg.y, s2 = sy.x + sy.y;
      group.sum3(s0, s1, s2);
      const float inv_r = rsqrtf(s0 * inv_d + a.eps), inv_y = a.w_post ? rsqrtf(s2 * inv_d + a.eps) : 1.f;
      const float2 ir = both(inv_r), iy = both(inv_y), c_r = both(-s1 * inv_r * inv_r * inv_r * inv_d);   // -mean(dh w r / rms) / rms^2
      float2 sb = both(0.f);                                      // sum dn w_post y
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int v = threadIdx.x + j * G;
#pragma unroll
        for (int i = 0; i < P; ++i) {
          const float2 t = fma2(r[j][i], c_r, fma2(pre[j][i], ir, o[j][i]));       // gradient of r'
          apre[j][i] = fma2(mul2(g[j][i], r[j][i]), ir, apre[j][i]);
          acc[j][i] = fma2(mul2(t, y[j][i]), iy, acc[j][i]);
          pre[j][i] = mul2(t, gw[j][i]);                                           // dn w_post
          sb = fma2(pre[j][i], y[j][i], sb);
          o[j][i] = mul2(scale, t);
        }
        if (mine(v) && group.ok) __stcs(reinterpret_cast<uint4*>(dr + row + (size_t)v * N), pack2<T>(o[j]));
      }
      if (y_given) {
        float2 c_y = both(0.f);
        if (a.w_post) c_y = both(-group.sum(sb.x + sb.y) * inv_y * inv_y * inv_y * inv_d);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const int v = threadIdx.x + j * G;
#pragma unroll
          for (int i = 0; i < P; ++i) pre[j][i] = fma2(y[j][i], c_y, mul2(pre[j][i], iy));
          if (mine(v) && group.ok) __stcs(reinterpret_cast<uint4*>(dy + row + (size_t)v * N), pack2<T>(pre[j]));
        }
      }
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int v = threadIdx.x + j * G;
      float2 x[P];
      load_weight<T>(a.gate, (size_t)grow * a.nvec + v, mine(v), 0.f, x);
#pragma unroll
      for (int i = 0; i < P; ++i) apost[j][i] = fma2(acc[j][i], x[i], apost[j][i]);
      if (part_gate && mine(v)) {
        load_weight<T>(a.w_post, v, true, a.w_offset, x);
#pragma unroll
        for (int i = 0; i < P; ++i) *reinterpret_cast<float2*>(part_gate + (size_t)unit * a.d + (size_t)v * N + 2 * i) = mul2(acc[j][i], x[i]);
      }
    }
  }
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int v = threadIdx.x + j * G;
    if (mine(v))
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const size_t at = (size_t)blockIdx.x * a.d + (size_t)v * N + 2 * i;
        if (part_post) *reinterpret_cast<float2*>(part_post + at) = apost[j][i];
        if (part_pre) *reinterpret_cast<float2*>(part_pre + at) = apre[j][i];
      }
  }
  norm_ring_end(group.ok, error_flag);
}

// Column sums of up to 2 + gates partial matrices: blockIdx.y picks one (0: w_post, 1: w_pre, 2..: gate rows), a CTA 32
// columns, its 32 warps every 32nd row; added in a fixed order.  All latency: the rows of a warp are on their way together.
constexpr int kNormReduceWarps = 32;
__global__ void __launch_bounds__(kNormReduceWarps * 32)
norm_reduce_kernel(const float* __restrict__ part_post, const float* __restrict__ part_pre, const float* __restrict__ part_gate,
                   float* __restrict__ dw_post, float* __restrict__ dw_pre, float* __restrict__ dgate, int rows, int per_gate, int d) {
  __shared__ float sm[kNormReduceWarps][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
  const int which = blockIdx.y;
  const float* p = which == 0 ? part_post : which == 1 ? part_pre : part_gate;
  float* o = which == 0 ? dw_post : which == 1 ? dw_pre : dgate;
  if (!p || !o) return;
  const size_t r0 = which < 2 ? 0 : (size_t)(which - 2) * per_gate;
  const int n = which < 2 ? rows : per_gate;
  float s = 0.f;
  if (col < d) {
#pragma unroll 8
    for (int r = warp; r < n; r += kNormReduceWarps) s += p[(r0 + r) * d + col];
  }
  sm[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && col < d) {
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < kNormReduceWarps; ++w) t += sm[w][lane];
    o[(which < 2 ? 0 : (size_t)(which - 2) * d) + col] = t;
  }
}

}  // namespace msr
