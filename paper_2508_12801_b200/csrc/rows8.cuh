// Rows and weights into 8-bit integers.
#pragma once
#include "int8.cuh"

namespace msr {

// ---- rows ----------------------------------------------------------------------------------------------------------------
constexpr int kRows8Warps = 8;

// Largest magnitude of a row's bf16 pairs; NaN wins, then infinity.
__device__ __forceinline__ uint32_t max8(uint32_t a, const uint4& v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    asm("{\n\t.reg .b32 t;\n\tand.b32 t, %1, 0x7fff7fff;\n\tmax.NaN.bf16x2 %0, %0, t;\n\t}" : "+r"(a) : "r"(w[i]));
  }
  return a;
}
__device__ __forceinline__ uint32_t warp_max8(uint32_t a) {                                  // as fp32 bits
  return __reduce_max_sync(0xffffffffu, max(a << 16, a & 0xffff0000u));
}
__device__ __forceinline__ uint4 quant16(const uint4& lo, const uint4& hi, float inv, uint32_t keep) {      // 16 values; keep: 0 or all ones
  const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
  uint32_t o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    o[i] = keep & pack8(round8(__uint_as_float(w[2 * i] << 16), inv), round8(__uint_as_float(w[2 * i] & 0xffff0000u), inv),
                        round8(__uint_as_float(w[2 * i + 1] << 16), inv), round8(__uint_as_float(w[2 * i + 1] & 0xffff0000u), inv));
  return make_uint4(o[0], o[1], o[2], o[3]);
}

// Bound by DRAM: two bytes read and one written a value (dispatch: k written).  Rows of 4096 in expert buffers 6.4 TB/s, of 1024 5.5; dispatch at T 65536,
// d 4096, k 8 460 us, 5.8 TB/s.
// A warp quantises a row of `chunks` 16-element chunks into its `n` destinations.  V: chunks that a lane holds from one pass to the next; 0: any
// number, read twice (the second time from the caches).
template <int V, typename Put>
__device__ __forceinline__ float row8(const uint4* __restrict__ src, int chunks, Put put) {
  const int lane = threadIdx.x & 31;
  uint4 x[V ? V : 1][2];
  uint32_t m = 0;
  if (V) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = lane + 32 * i;
      x[i][0] = x[i][1] = make_uint4(0, 0, 0, 0);
      if (c < chunks) { x[i][0] = __ldcs(src + 2 * c); x[i][1] = __ldcs(src + 2 * c + 1); }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) m = max8(max8(m, x[i][0]), x[i][1]);
  } else {
    for (int c = lane; c < chunks; c += 32) m = max8(max8(m, __ldg(src + 2 * c)), __ldg(src + 2 * c + 1));
  }
  const Step8 s = step8(warp_max8(m));
  const uint32_t keep = s.inv > 0.f ? 0xffffffffu : 0u;
  if (V) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = lane + 32 * i;
      if (c < chunks) put(c, quant16(x[i][0], x[i][1], s.inv, keep));
    }
  } else {
    for (int c = lane; c < chunks; c += 32) put(c, quant16(__ldg(src + 2 * c), __ldg(src + 2 * c + 1), s.inv, keep));
  }
  return s.scale;
}

// Dispatch of token rows as bytes: a row is read and quantised once and written to each of its slots; rows and scales of empty slots
// become zero.
template <int V>
__global__ void __launch_bounds__(kRows8Warps * 32)
dispatch8_kernel(const uint4* __restrict__ src, const int32_t* __restrict__ expert_idx, const int32_t* __restrict__ slot_idx,
                 const int32_t* __restrict__ slot_token, uint4* __restrict__ dst, float* __restrict__ dst_scale, int T, int chunks, int E, int k,
                 int C) {
  const int lane = threadIdx.x & 31;
  const int64_t warp = (int64_t)blockIdx.x * kRows8Warps + (threadIdx.x >> 5), warps = (int64_t)gridDim.x * kRows8Warps;
  for (int64_t tok = warp; tok < T; tok += warps) {
    int64_t my_row = -1;
    if (lane < k) {
      const int e = __ldg(expert_idx + tok * k + lane), s = __ldg(slot_idx + tok * k + lane);
      if (e >= 0 && e < E && s >= 0 && s < C) my_row = (int64_t)e * C + s;
    }
    int64_t row[kMaxK];
#pragma unroll
    for (int c = 0; c < kMaxK; ++c) row[c] = __shfl_sync(0xffffffffu, my_row, c);
    const float scale = row8<V>(src + tok * chunks * 2, chunks, [&](int c, const uint4& q) {
#pragma unroll
      for (int i = 0; i < kMaxK; ++i) if (i < k && row[i] >= 0) __stcs(dst + row[i] * chunks + c, q);
    });
    if (my_row >= 0) dst_scale[my_row] = scale;
  }
  const int64_t slots = (int64_t)E * C;
  for (int64_t base = warp * 32; base < slots; base += warps * 32) {
    const int64_t s = base + lane;
    const bool empty = s < slots && __ldg(slot_token + s) < 0;
    if (empty) dst_scale[s] = 0.f;
    for (uint32_t left = __ballot_sync(0xffffffffu, empty); left; left &= left - 1) {
      uint4* d = dst + (base + __ffs(left) - 1) * chunks;
      for (int c = lane; c < chunks; c += 32) d[c] = make_uint4(0, 0, 0, 0);
    }
  }
}

// Rows of an expert buffer; rows behind the load become zero, their scales too.  load null: all rows are in use (weights).
template <int V>
__global__ void __launch_bounds__(kRows8Warps * 32)
rows8_kernel(const uint4* __restrict__ src, const int32_t* __restrict__ load, uint4* __restrict__ dst, float* __restrict__ dst_scale, int64_t rows,
             int chunks, int C) {
  const int lane = threadIdx.x & 31;
  const int64_t warps = (int64_t)gridDim.x * kRows8Warps;
  for (int64_t r = (int64_t)blockIdx.x * kRows8Warps + (threadIdx.x >> 5); r < rows; r += warps) {
    uint4* d = dst + r * chunks;
    float scale = 0.f;
    if (!load || (int)(r % C) < __ldg(load + r / C)) scale = row8<V>(src + r * chunks * 2, chunks, [&](int c, const uint4& q) { d[c] = q; });
    else for (int c = lane; c < chunks; c += 32) d[c] = make_uint4(0, 0, 0, 0);
    if (lane == 0) dst_scale[r] = scale;
  }
}

// ---- weights [E][d_in][d_out] -> integers [E][d_out][d_in] --------------------------------------------------------------------
// A CTA owns 64 columns of one expert: their largest magnitudes first, then tiles of 64 columns x 128 rows turned round in shared
// memory.  Once per weight, so it only has to be reasonable: the second reading comes from the L2 where a block of columns fits.  E 64, 2048 x 2048
// 413 us, 1.9 TB/s (weights that lie the other way round take rows8_kernel: 129 us, 6.2 TB/s).
constexpr int kTurnCols = 64, kTurnRows = 128;
__global__ void __launch_bounds__(256)
turn8_kernel(const __nv_bfloat16* __restrict__ w, int8_t* __restrict__ q, float* __restrict__ scale, int d_in, int d_out) {
  __shared__ uint32_t part[32][kTurnCols + 1];
  __shared__ float inv[kTurnCols];
  __shared__ __align__(16) uint8_t tile[kTurnCols][kTurnRows + 16];
  const int64_t e = blockIdx.y;
  const int n0 = blockIdx.x * kTurnCols, cv = threadIdx.x & 7, rv = threadIdx.x >> 3;      // eight columns, one row of 32
  const bool in = n0 + cv * 8 < d_out;
  const uint4* src = reinterpret_cast<const uint4*>(w + e * d_in * d_out + n0 + cv * 8);
  const size_t stride = d_out / 8;
  uint32_t m[4] = {};
  if (in)
    for (int r = rv; r < d_in; r += 32) {
      const uint4 v = __ldg(src + r * stride);
      const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) asm("{\n\t.reg .b32 t;\n\tand.b32 t, %1, 0x7fff7fff;\n\tmax.NaN.bf16x2 %0, %0, t;\n\t}" : "+r"(m[i]) : "r"(x[i]));
    }
#pragma unroll
  for (int i = 0; i < 4; ++i) { part[rv][cv * 8 + 2 * i] = m[i] << 16; part[rv][cv * 8 + 2 * i + 1] = m[i] & 0xffff0000u; }
  __syncthreads();
  if (threadIdx.x < kTurnCols) {
    uint32_t a = 0;
    for (int i = 0; i < 32; ++i) a = max(a, part[i][threadIdx.x]);
    const Step8 s = step8(a);
    inv[threadIdx.x] = s.inv;
    if (n0 + threadIdx.x < d_out) scale[e * d_out + n0 + threadIdx.x] = s.scale;
  }
  __syncthreads();
  for (int r0 = 0; r0 < d_in; r0 += kTurnRows) {
    for (int r = rv; r < kTurnRows; r += 32)
      if (in && r0 + r < d_in) {
        float f[8];
        Vec16<__nv_bfloat16>::unpack(__ldg(src + (r0 + r) * stride), f);
#pragma unroll
        for (int i = 0; i < 8; ++i) tile[cv * 8 + i][r] = inv[cv * 8 + i] > 0.f ? (uint8_t)round8(f[i], inv[cv * 8 + i]) : 0;
      }
    __syncthreads();
    for (int i = threadIdx.x; i < kTurnCols * (kTurnRows / 16); i += 256) {
      const int c = i / (kTurnRows / 16), r = i % (kTurnRows / 16) * 16;
      if (n0 + c < d_out && r0 + r < d_in)                             // d_in is a multiple of 16
        *reinterpret_cast<uint4*>(q + (e * d_out + n0 + c) * d_in + r0 + r) = *reinterpret_cast<const uint4*>(&tile[c][r]);
    }
    __syncthreads();
  }
}

}  // namespace msr
