// Routing by top-k: scores, choice of k experts by score + balance bias within the best groups, combine weights; and its backward pass.
//
//   s_e = softmax(l)_e or sigmoid(l_e)        c_e = s_e + b_e
//   a group's value is its largest c, or the sum of its two largest; the best groups stay, the k best c in them are chosen
//   w_c = scale s_c / (sum of the chosen s + 1e-20), or scale s_c
//
// Which of two near values is larger is decided as in 64 bits, for the choice is discrete.  Without a bias the order of s is that of
// l, which fp32 compares exactly.  With one (and for sums of two scores) a row whose last accepted and first refused value lie closer
// than fp32 can tell apart is chosen again in 64 bits, by the whole warp; about one row in 2 000 of 128 experts.
//
// Two forms.  In the usual one eight lanes own a token and a warp four: next to 4 E bytes of logits the instructions count, and what a
// token needs once (sums, maxima, the k rounds) costs a quarter of what it does with a warp per token.  Each lane sorts the values of
// its consecutive experts, keeps the eight largest, and in k rounds the largest heads leave.  Few tokens, which a warp each serves sooner, and groups that are not
// whole lanes, a power of two of them, take the other form, a warp per token with the groups' values in shared memory.
// T 65536, E 128, k 8: 33 us with groups, bias and scores written (a warp per token 49), 19 to 21 without any (31); the bytes take 11 and 6.  300
// instructions a token (580 with a warp for each), issued in 66 to 72 % of the clocks.
#pragma once
#include "common.cuh"

namespace msr {

constexpr int kTopkWarps = 8, kTopkMaxGroups = 32;
constexpr float kTopkEps = 1e-20f;     // in the denominator of the weights: a row whose chosen scores all vanish gets zeros

struct TopkArgs {
  int T, E, k;
  int n_group, topk_group, group_size;
  int group_shift;       // eight lanes a token: a group has 1 << group_shift of them
  int sigmoid, pairs, renorm;
  float scale;
};

// Integers in the order of floats, -0 equal to 0, none of them 0, which stands for "cannot be chosen".  NaN, whatever its sign, is above infinity: a sum
// that is not a number has the one pattern 0x7fffffff.
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float order_value(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }

// m1, m2: the two largest so far, -inf at first; x may be NaN, which counts as nothing (min.NaN hands it to a maximum that drops it)
__device__ __forceinline__ void two_largest(float x, float& m1, float& m2) {
  float low;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(low) : "f"(m1), "f"(x));
  m2 = fmaxf(m2, low);
  m1 = fmaxf(m1, x);
}
// value of a group; inf - inf makes it the last
__device__ __forceinline__ float group_value(float m1, float m2, bool pairs) { return pairs ? fmaxf(m1 + m2, -INFINITY) : m1; }

// How far from v in fp32 the value may lie that 64 bits give: the least it can be for a group that stays, the most for one that goes.  Scores are off by
// 2^-21 and each c by 2^-24 of itself, their sum by 2^-24 more; the terms count and not the sum, in which biases of both signs cancel.  Twice that.
__device__ __forceinline__ float group_bound(float m1, float m2, bool pairs, float v, bool stays) {
  const float err = fmaf(0x1p-22f, fabsf(m1) + (pairs ? fabsf(m2) : 0.f), 0x1p-19f);
  return fabsf(v) == INFINITY ? v : stays ? v - err : v + err;
}

// e^x for x <= 0: 2^t with t = x log2(e) rounded, then what the rounding left of the exponent as a factor 1 + r ln 2.  Off by 2^-22
// (the approximation of 2^t) and some 2^-24 (the products) of itself; below 2^-126 it is 0.  NaN stays NaN.
__device__ __forceinline__ float exp_down(float x) {
  constexpr float log2e = 1.44269504f, rest = 1.92596303e-8f, ln2 = 0.693147181f;      // log2(e) = log2e + rest
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(x) : "f"(x), "f"(-126.f));                       // e^-126 is 0 in fp32
  const float t = x * log2e, r = fmaf(x, rest, fmaf(x, log2e, -t));
  float e;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(t));
  return fmaf(e * ln2, r, e);
}
// sigmoid(l) and 1 - sigmoid(l), both to a few steps of their last bit
__device__ __forceinline__ void sigmoid_pair(float l, float& s, float& rest) {
  const float t = exp_down(-fabsf(l));
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + t));                          // of 1 to 2, to the last bit or so
  const float tr = t * r;
  s = l < 0.f ? tr : r;
  rest = l < 0.f ? r : tr;
}

// Full: rows of exactly 32 VPT experts, moved as vectors.
template <int VPT, bool Full>
__device__ __forceinline__ void topk_load_row(const float* __restrict__ row, int E, int lane, float (&l)[VPT]) {
  const int e0 = lane * VPT;
  if (Full && VPT == 4) {
    const float4 v = __ldg(reinterpret_cast<const float4*>(row) + lane);
    l[0] = v.x; l[1 % VPT] = v.y; l[2 % VPT] = v.z; l[3 % VPT] = v.w;
  } else if (Full && VPT == 2) {
    const float2 v = __ldg(reinterpret_cast<const float2*>(row) + lane);
    l[0] = v.x; l[1 % VPT] = v.y;
  } else {
#pragma unroll
    for (int j = 0; j < VPT; ++j) l[j] = e0 + j < E ? __ldg(row + e0 + j) : 0.f;
  }
}
template <int VPT, bool Full>
__device__ __forceinline__ void topk_store_row(float* __restrict__ row, int E, int lane, const float (&v)[VPT]) {
  const int e0 = lane * VPT;
  if (Full && VPT == 4) reinterpret_cast<float4*>(row)[lane] = make_float4(v[0], v[1 % VPT], v[2 % VPT], v[3 % VPT]);
  else if (Full && VPT == 2) reinterpret_cast<float2*>(row)[lane] = make_float2(v[0], v[1 % VPT]);
  else {
#pragma unroll
    for (int j = 0; j < VPT; ++j) if (e0 + j < E) row[e0 + j] = v[j];
  }
}

// s of the row; for the sigmoid 1 - s too
template <int VPT, bool Full>
__device__ __forceinline__ void topk_scores(const float (&l)[VPT], int E, int lane, bool sigmoid, float (&s)[VPT], float (&rest)[VPT]) {
  const int e0 = lane * VPT;
  if (sigmoid) {
#pragma unroll
    for (int j = 0; j < VPT; ++j) sigmoid_pair(l[j], s[j], rest[j]);
    return;
  }
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < VPT; ++j) if (Full || e0 + j < E) top = max(top, order_key(l[j]));
  const float m = order_value(__reduce_max_sync(0xffffffffu, top));
  float sum = 0.f;
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    s[j] = Full || e0 + j < E ? exp_down(l[j] - m) : 0.f;              // NaN where l is, and in rows whose largest is infinite
    sum += s[j];
  }
  const float inv = 1.f / warp_sum(sum);
#pragma unroll
  for (int j = 0; j < VPT; ++j) s[j] *= inv;
}

// The choice in 64 bits, for rows that fp32 cannot decide.  Returns this lane's chosen experts as bits.  `d`: E doubles of the warp's own.
__device__ __noinline__ uint32_t topk_choose_64(const float* __restrict__ row, const float* __restrict__ bias, TopkArgs a, int vpt, double* d) {
  const int lane = threadIdx.x & 31, e0 = lane * vpt;
  double l[4], v[4];                                                  // four chains side by side: this is a matter of latency
  bool in[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    in[j] = j < vpt && e0 + j < a.E;
    l[j] = in[j] ? (double)__ldg(row + e0 + j) : -INFINITY;
  }
  // a row of one value with one bias (padded tokens, and early training): the lowest groups, and of them the lowest experts
  const double first_l = __shfl_sync(0xffffffffu, l[0], 0);
  const float first_b = bias ? __ldg(bias) : 0.f;
  bool even = true;
#pragma unroll
  for (int j = 0; j < 4; ++j) even = even && (!in[j] || (l[j] == first_l && (!bias || __ldg(bias + e0 + j) == first_b)));
  if (__all_sync(0xffffffffu, even)) {
    uint32_t lowest = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) if (in[j] && e0 + j < a.k) lowest |= 1u << j;
    return lowest;
  }
  if (a.sigmoid) {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = 1.0 / (1.0 + exp(-l[j]));
  } else {
    double m = fmax(fmax(l[0], l[1]), fmax(l[2], l[3])), sum = 0.0;
    for (int o = 16; o > 0; o >>= 1) m = fmax(m, __shfl_xor_sync(0xffffffffu, m, o));
#pragma unroll
    for (int j = 0; j < 4; ++j) { v[j] = exp(l[j] - m); sum += in[j] ? v[j] : 0.0; }
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] /= sum;
  }
  if (bias) {
#pragma unroll
    for (int j = 0; j < 4; ++j) if (in[j]) v[j] += (double)__ldg(bias + e0 + j);
  }
  uint32_t kept = 1u;
  if (a.n_group > 1) {
    auto counts = [](double x) { return x == x ? x : -INFINITY; };    // NaN is nothing in a group's value, and a value of inf - inf the last
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 4; ++j) if (in[j]) d[e0 + j] = counts(v[j]);
    __syncwarp();
    double m1 = -INFINITY, m2 = -INFINITY;
    if (lane < a.n_group) {
#pragma unroll 4
      for (int i = 0; i < a.group_size; ++i) {
        const double x = d[lane * a.group_size + i];
        m2 = fmax(m2, fmin(m1, x)); m1 = fmax(m1, x);
      }
    }
    const double value = counts(a.pairs && a.group_size > 1 ? m1 + m2 : m1);
    int before = 0;
#pragma unroll 4
    for (int g = 0; g < a.n_group; ++g) {
      const double other = __shfl_sync(0xffffffffu, value, g);
      before += other > value || (other == value && g < lane);
    }
    kept = __ballot_sync(0xffffffffu, lane < a.n_group && before < a.topk_group);
  }
  // the experts themselves: without a bias by their logits, as in fp32; NaN ahead of infinity, which no finite value reaches as the largest double
  auto order = [](double x) { return x == x ? fmin(x, 1.7976931348623157e308) : INFINITY; };
  __syncwarp();
#pragma unroll
  for (int j = 0; j < 4; ++j) if (in[j]) { v[j] = order(bias ? v[j] : l[j]); d[e0 + j] = v[j]; }
  __syncwarp();
  int before[4] = {};
  for (uint32_t rest = kept; rest; rest &= rest - 1) {
    const int first = (__ffs(rest) - 1) * a.group_size;
#pragma unroll 4
    for (int i = first; i < first + a.group_size; ++i) {
      const double x = d[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) before[j] += x > v[j] || (x == v[j] && i < e0 + j);
    }
  }
  uint32_t chosen = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) if (in[j] && (kept >> ((e0 + j) / a.group_size) & 1) && before[j] < a.k) chosen |= 1u << j;
  __syncwarp();
  return chosen;
}

// Choice among equal values at the border: the lowest indices of them stay.  Returns this lane's chosen experts as bits.
template <int VPT>
__device__ __noinline__ uint32_t topk_choose_equal(const uint32_t* key, int k) {
  const int lane = threadIdx.x & 31;
  uint32_t left[VPT], last = 0;
#pragma unroll
  for (int j = 0; j < VPT; ++j) left[j] = key[j];
  for (int gone = 0; gone < k;) {                                      // all experts of one value leave together
    uint32_t head = 0;
#pragma unroll
    for (int j = 0; j < VPT; ++j) head = max(head, left[j]);
    last = __reduce_max_sync(0xffffffffu, head);                       // above 0: k experts can be chosen
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      gone += __popc(__ballot_sync(0xffffffffu, left[j] == last));
      if (left[j] == last) left[j] = 0;
    }
  }
  int spare = k, equal = 0;                                            // room for the equal ones; those of lower lanes
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    spare -= __popc(__ballot_sync(0xffffffffu, key[j] > last));
    equal += __popc(__ballot_sync(0xffffffffu, key[j] == last) & ((1u << lane) - 1u));
  }
  uint32_t chosen = 0;
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    if (key[j] > last) chosen |= 1u << j;
    else if (key[j] == last && equal++ < spare) chosen |= 1u << j;
  }
  return chosen;
}

// A warp per token, groups of any size or none.
template <int VPT, bool Full>
__global__ void __launch_bounds__(kTopkWarps * 32)
topk_fwd_scan_kernel(const float* __restrict__ logits, const float* __restrict__ bias, float* __restrict__ scores, int32_t* __restrict__ expert_idx,
                float* __restrict__ gate_w, TopkArgs a) {
  __shared__ __align__(16) double scratch[kTopkWarps][kMaxE];          // 64-bit values of a row; its fp32 values, group by group, before
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, e0 = lane * VPT;
  float* grouped = reinterpret_cast<float*>(scratch[warp]);            // a word between groups, so that lanes = groups read without conflicts
  static_assert(sizeof(double) * kMaxE >= sizeof(float) * (kMaxE + kTopkMaxGroups), "a row and a word per group");
  float b[VPT];
  int group[VPT];
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    b[j] = bias && e0 + j < a.E ? __ldg(bias + e0 + j) : 0.f;
    group[j] = min((e0 + j) / a.group_size, kTopkMaxGroups - 1);
  }
  const bool speaks = lane < a.n_group;                                // a lane per group
  const int64_t step = gridDim.x * kTopkWarps;
  int64_t t = blockIdx.x * kTopkWarps + warp;
  float next[VPT];
  if (t < a.T) topk_load_row<VPT, Full>(logits + t * a.E, a.E, lane, next);
  for (; t < a.T; t += step) {
    float l[VPT], s[VPT], rest[VPT];
#pragma unroll
    for (int j = 0; j < VPT; ++j) l[j] = next[j];
    if (t + step < a.T) topk_load_row<VPT, Full>(logits + (t + step) * a.E, a.E, lane, next);
    topk_scores<VPT, Full>(l, a.E, lane, a.sigmoid, s, rest);
    if (scores) topk_store_row<VPT, Full>(scores + t * a.E, a.E, lane, s);
    float c[VPT];
    uint32_t key[VPT];
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      c[j] = bias ? s[j] + b[j] : l[j];
      key[j] = Full || e0 + j < a.E ? order_key(c[j]) : 0u;
    }
    bool near = false;                                                 // the same in all lanes
    if (a.n_group > 1) {
      // the two largest of each group
      if (!bias && a.pairs) {
#pragma unroll
        for (int j = 0; j < VPT; ++j) c[j] = s[j];
      }
      float m1 = -INFINITY, m2 = -INFINITY;
#pragma unroll
      for (int j = 0; j < VPT; ++j) if (Full || e0 + j < a.E) grouped[e0 + j + group[j]] = c[j];
      __syncwarp();
      if (speaks)
        for (int i = 0; i < a.group_size; ++i) two_largest(grouped[lane * (a.group_size + 1) + i], m1, m2);
      __syncwarp();
      const bool two = a.pairs && a.group_size > 1;
      const float value = group_value(m1, m2, two);
      const uint32_t mine = speaks ? order_key(value) : 0u;
      int before = 0;
      for (int g = 0; g < a.n_group; ++g) before += __shfl_sync(0xffffffffu, mine, g) >= mine + (g >= lane);
      const bool in = speaks && before < a.topk_group;
      if (bias || a.pairs) {
        const uint32_t edge = order_key(group_bound(m1, m2, two, value, in));
        const float low = order_value(__reduce_min_sync(0xffffffffu, in ? edge : 0xffffffffu));
        const float high = order_value(__reduce_max_sync(0xffffffffu, speaks && !in ? edge : 0u));
        near = !(low > high);
      }
      const uint32_t kept = __ballot_sync(0xffffffffu, in);
#pragma unroll
      for (int j = 0; j < VPT; ++j) if (!(kept >> group[j] & 1)) key[j] = 0u;
    }
    // The k-th largest value: lanes keep their own sorted, the largest heads leave.
    uint32_t q[VPT];
#pragma unroll
    for (int j = 0; j < VPT; ++j) q[j] = key[j];
    auto order = [&](int i, int j) { const uint32_t hi = max(q[i], q[j]); q[j] = min(q[i], q[j]); q[i] = hi; };
    if constexpr (VPT == 4) { order(0, 1); order(2, 3); order(0, 2); order(1, 3); order(1, 2); }
    else if constexpr (VPT == 3) { order(0, 1); order(1, 2); order(0, 1); }
    else if constexpr (VPT == 2) order(0, 1);
    uint32_t last = 0;
#pragma unroll 1
    for (int i = 0; i < a.k; ++i) {
      last = __reduce_max_sync(0xffffffffu, q[0]);
      if (q[0] == last) {
#pragma unroll
        for (int j = 0; j + 1 < VPT; ++j) q[j] = q[j + 1];
        q[VPT - 1] = 0;
      }
    }
    uint32_t chosen = 0, at[VPT];                                      // at[j]: the lanes whose j-th expert is chosen
    auto places = [&] {                                                // how many chosen experts lower lanes have
      int n = 0;
#pragma unroll
      for (int j = 0; j < VPT; ++j) n += __popc(at[j] & ((1u << lane) - 1u));
      return n;
    };
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const bool in = key[j] >= last && key[j] != 0u;
      chosen |= (uint32_t)in << j;
      at[j] = __ballot_sync(0xffffffffu, in);
    }
    int place = places();
    const bool equal = __shfl_sync(0xffffffffu, place + __popc(chosen), 31) != a.k;      // equal values left together
    if (bias) {
      // fp32 errors of s: of the exponent |l - m| 2^-24 e^-|l - m|, of exponential, sum and quotient 2^-21 s at most; of the sum with
      // the bias 2^-24 of it.  Twice that between two values, rounded up.
      const uint32_t after = __reduce_max_sync(0xffffffffu, q[0]);
      const float low = order_value(last);
      near = near || equal || (after != 0 && !(low - order_value(after) > 0x1p-19f + 0x1p-22f * fabsf(low)));
    }
    if (near || equal) {
      chosen = near ? topk_choose_64(logits + t * a.E, bias, a, VPT, scratch[warp]) : topk_choose_equal<VPT>(key, a.k);
#pragma unroll
      for (int j = 0; j < VPT; ++j) at[j] = __ballot_sync(0xffffffffu, chosen >> j & 1);
      place = places();
    }
    float f = a.scale;
    if (a.renorm) {
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < VPT; ++j) sum += chosen >> j & 1 ? s[j] : 0.f;
      f = a.scale / (warp_sum(sum) + kTopkEps);
    }
    // ascending: the chosen of lower lanes, then the lane's own
    int32_t* idx = expert_idx + t * a.k;
    float* w = gate_w + t * a.k;
#pragma unroll
    for (int j = 0; j < VPT; ++j)
      if (chosen >> j & 1) {
        idx[place] = e0 + j;
        w[place] = s[j] * f;
        ++place;
      }
  }
}

// ---- eight lanes a token ---------------------------------------------------------------------------------------------------
__device__ __forceinline__ float seg_max(float v) {
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ uint32_t seg_max(uint32_t v) {
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
template <typename T>
__device__ __forceinline__ T seg_sum(T v) {
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ int seg_before(int v, int lane8) {          // sum over the lower lanes of the token
  int incl = v;
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, incl, o, 8);
    if (lane8 >= o) incl += x;
  }
  return incl - v;
}
__device__ __forceinline__ void descend(uint32_t& a, uint32_t& b) { const uint32_t hi = max(a, b); b = min(a, b); a = hi; }
// q[At .. At + N) in descending order
template <int N, int At, int M>
__device__ __forceinline__ void sort_keys(uint32_t (&q)[M]) {
  auto ce = [&](int i, int j) { descend(q[At + i], q[At + j]); };
  if constexpr (N == 2) ce(0, 1);
  else if constexpr (N == 4) { ce(0, 1); ce(2, 3); ce(0, 2); ce(1, 3); ce(1, 2); }
  else {
    static_assert(N == 8, "2, 4 or 8");
    ce(0, 1); ce(2, 3); ce(4, 5); ce(6, 7); ce(0, 2); ce(1, 3); ce(4, 6); ce(5, 7); ce(1, 2); ce(5, 6); ce(0, 4); ce(3, 7); ce(1, 5); ce(2, 6);
    ce(1, 4); ce(3, 6); ce(2, 4); ce(3, 5); ce(3, 4);
  }
}

// V: experts of a lane.  Groups: whether there are any, of whole lanes.  Full: E = 8 V.
template <int V, bool Groups, bool Full>
__global__ void __launch_bounds__(kTopkWarps * 32)
topk_fwd_kernel(const float* __restrict__ logits, const float* __restrict__ bias, float* __restrict__ scores, int32_t* __restrict__ expert_idx,
                float* __restrict__ gate_w, TopkArgs a) {
  constexpr int Q = V < kMaxK ? V : kMaxK;                             // at most k of a lane's experts are chosen
  __shared__ double scratch[kTopkWarps][kMaxE];                        // values of a row that is chosen in 64 bits
  __shared__ uint32_t marks[kTopkWarps][4];                            // and its experts
  constexpr int kPad = V >= 8 ? 4 : 0;                                 // between lanes' parts, so that 16-byte stores do not meet in a bank
  __shared__ __align__(16) float held[kTopkWarps][4][8 * (V + kPad)];  // s of the warp's four tokens
  __shared__ __align__(16) float held_bias[8 * (V + kPad)];            // laid out as they are
  __shared__ int picks[kTopkWarps][4][kMaxK];                          // the chosen of each, ascending
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, lane8 = lane & 7, e0 = lane8 * V;
  const uint32_t seg = 0xffu << (lane & 24);
  const int my_group = lane8 >> a.group_shift;
  const bool speaks = my_group < a.n_group;
  auto there = [&](int j) { return Full || e0 + j < a.E; };
  float* mine_s = held[warp][lane >> 3];
  int* mine_e = picks[warp][lane >> 3];
  auto load = [&](float (&x)[V], const float* p) {
    if constexpr (Full && V % 4 == 0) {
#pragma unroll
      for (int j = 0; j < V; j += 4) {
        const float4 v = __ldg(reinterpret_cast<const float4*>(p + j));
        x[j] = v.x; x[j + 1] = v.y; x[j + 2] = v.z; x[j + 3] = v.w;
      }
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) x[j] = there(j) ? __ldg(p + j) : 0.f;
    }
  };
  for (int e = threadIdx.x; e < 8 * V; e += kTopkWarps * 32) held_bias[e + e / V * kPad] = bias && e < a.E ? __ldg(bias + e) : 0.f;
  __syncthreads();
  const int64_t step = (int64_t)gridDim.x * kTopkWarps * 4, end = (int64_t)a.T - 1;
  float l[V];                                                          // a row; then the next one, on its way during the rounds
  int64_t t0 = ((int64_t)blockIdx.x * kTopkWarps + warp) * 4;
  if (t0 < a.T) load(l, logits + min(t0 + (lane >> 3), end) * a.E + e0);
  for (; t0 < a.T; t0 += step) {
    const int64_t t = min(t0 + (lane >> 3), end);                      // behind the last token: computed again, not written
    const bool valid = t0 + (lane >> 3) < a.T;
    float s[V];
    uint32_t key[V];
    if (a.sigmoid) {
#pragma unroll
      for (int j = 0; j < V; ++j) { float rest; sigmoid_pair(l[j], s[j], rest); }
    } else {
      float m = -INFINITY, sum = 0.f;
#pragma unroll
      for (int j = 0; j < V; ++j) if (there(j)) m = fmaxf(m, l[j]);
      m = seg_max(m);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        s[j] = there(j) ? exp_down(l[j] - m) : 0.f;                    // NaN where l is, and in rows whose largest is infinite
        sum += s[j];
      }
      const float inv = 1.f / seg_sum(sum);
#pragma unroll
      for (int j = 0; j < V; ++j) s[j] *= inv;
    }
#pragma unroll
    for (int j = 0; j < V; j += (V % 4 == 0 ? 4 : 2)) {
      if constexpr (V % 4 == 0) *reinterpret_cast<float4*>(mine_s + e0 + lane8 * kPad + j) = make_float4(s[j], s[j + 1], s[j + 2], s[j + 3]);
      else *reinterpret_cast<float2*>(mine_s + e0 + j) = make_float2(s[j], s[j + 1]);
    }
    if (scores) {
      __syncwarp();
      if constexpr (Full && V >= 4) {
        // from shared memory in whole lines: lane i of a row of V 2 chunks
#pragma unroll
        for (int i = lane; i < 4 * V * 2; i += 32) {
          const int r = i / (V * 2), e = i % (V * 2) * 4;
          if (t0 + r < a.T) *reinterpret_cast<float4*>(scores + (t0 + r) * a.E + e) = *reinterpret_cast<const float4*>(&held[warp][r][e + e / V * kPad]);
        }
      } else {
        for (int r = 0; r < 4 && t0 + r < a.T; ++r)
          for (int e = lane; e < a.E; e += 32) scores[(t0 + r) * a.E + e] = held[warp][r][e + e / V * kPad];
      }
    }
    if (bias) {
#pragma unroll
      for (int j = 0; j < V; ++j) l[j] = s[j] + held_bias[e0 + lane8 * kPad + j];
    }
#pragma unroll
    for (int j = 0; j < V; ++j) key[j] = there(j) ? order_key(l[j]) : 0u;
    bool near = false;                                                 // the same in a token's lanes
    if constexpr (Groups) {
      // the two largest of each group
      float m1 = -INFINITY, m2 = -INFINITY;
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (there(j)) two_largest(!bias && a.pairs ? s[j] : l[j], m1, m2);
      for (int o = 1; o < 1 << a.group_shift; o <<= 1) {
        const float o1 = __shfl_xor_sync(0xffffffffu, m1, o), o2 = __shfl_xor_sync(0xffffffffu, m2, o);
        m2 = fmaxf(fminf(m1, o1), fmaxf(m2, o2));
        m1 = fmaxf(m1, o1);
      }
      const bool two = a.pairs && a.group_size > 1;
      const float value = group_value(m1, m2, two);
      const uint32_t mine = speaks ? order_key(value) : 0u;
      int before = 0;                                                  // lanes of better groups: of equal ones the lower
#pragma unroll
      for (int o = 1; o < 8; ++o) before += __shfl_xor_sync(0xffffffffu, mine, o) >= mine + ((lane8 ^ o) >> a.group_shift >= my_group);
      const bool in = speaks && before < a.topk_group << a.group_shift;
      if (bias || a.pairs) {
        const uint32_t edge = order_key(group_bound(m1, m2, two, value, in));
        const float low = order_value(~seg_max(in ? ~edge : 0u)), high = order_value(seg_max(speaks && !in ? edge : 0u));
        near = !(low > high);
      }
#pragma unroll
      for (int j = 0; j < V; ++j) key[j] = in ? key[j] : 0u;
    }
    if (t0 + step < a.T) load(l, logits + min(t0 + step + (lane >> 3), end) * a.E + e0);
    // The lane's largest in order, then k rounds (or fewer, where equal ones leave together).
    uint32_t q[V];
#pragma unroll
    for (int j = 0; j < V; ++j) q[j] = key[j];
    if constexpr (V == 16) {
      sort_keys<8, 0>(q); sort_keys<8, 8>(q);
#pragma unroll
      for (int j = 0; j < 8; ++j) q[j] = max(q[j], q[15 - j]);         // the eight largest, rising and falling
#pragma unroll
      for (int o = 4; o > 0; o >>= 1)
#pragma unroll
        for (int j = 0; j < 8; ++j) if (!(j & o)) descend(q[j], q[j + o]);
    } else sort_keys<V, 0>(q);
    uint32_t last = 0;                                                 // the k-th largest value
    int gone = 0;
#pragma unroll 1
    for (int i = 0; i < a.k; ++i) {
      const uint32_t m = seg_max(q[0]);
      const bool open = gone < a.k, leaves = open && q[0] == m;
      if (open) last = m;
      gone += __popc(__ballot_sync(0xffffffffu, leaves) & seg);
      if (leaves) {
#pragma unroll
        for (int j = 0; j + 1 < Q; ++j) q[j] = q[j + 1];
        q[Q - 1] = 0;
      }
    }
    uint32_t chosen = 0;
#pragma unroll
    for (int j = 0; j < V; ++j) chosen |= (uint32_t)(key[j] >= last) << j;               // last is above 0: k experts can be chosen
    int place = seg_before(__popc(chosen), lane8);
    const bool equal = __shfl_sync(0xffffffffu, place + __popc(chosen), lane | 7) != a.k;
    if (bias) {
      // fp32 errors of s: of the exponent |l - m| 2^-24 e^-|l - m|, of exponential, sum and quotient 2^-21 s at most; of the sum with
      // the bias 2^-24 of it.  Twice that between two values, rounded up.
      const uint32_t after = seg_max(q[0]);
      const float low = order_value(last);
      const bool blind = V > Q && seg_max((uint32_t)__popc(chosen)) >= Q;              // a lane whose list has run out
      near = near || equal || blind || (after != 0 && !(low - order_value(after) > 0x1p-19f + 0x1p-22f * fabsf(low)));
    }
    if (__any_sync(0xffffffffu, equal || near)) {
      // equal values at the border: the lowest indices of them stay (a token without any keeps its experts)
      int above = 0, same = 0;
#pragma unroll
      for (int j = 0; j < V; ++j) { above += key[j] > last; same += key[j] == last; }
      int room = a.k - seg_sum(above) - seg_before(same, lane8);
#pragma unroll
      for (int j = 0; j < V; ++j) if (key[j] == last && room-- <= 0) chosen &= ~(1u << j);
      // rows that fp32 cannot decide, one by one
      for (uint32_t left = __ballot_sync(0xffffffffu, near && lane8 == 0); left; left &= left - 1) {
        const int first = __ffs(left) - 1, vpt = (a.E + 31) / 32;
        const uint32_t bits = topk_choose_64(logits + min(t0 + (first >> 3), (int64_t)a.T - 1) * a.E, bias, a, vpt, scratch[warp]);
        if (lane < 4) marks[warp][lane] = 0;
        __syncwarp();
        for (int j = 0; j < vpt; ++j) if (bits >> j & 1) atomicOr(&marks[warp][(lane * vpt + j) >> 5], 1u << ((lane * vpt + j) & 31));
        __syncwarp();
        if ((lane & 24) == first) chosen = marks[warp][e0 >> 5] >> (e0 & 31) & (V == 32 ? 0xffffffffu : (1u << V) - 1u);
        __syncwarp();
      }
      place = seg_before(__popc(chosen), lane8);
    }
    // ascending: the chosen of lower lanes, then the lane's own; each of the token's first k lanes then takes one
    for (uint32_t left = chosen; left; left &= left - 1) mine_e[place++] = e0 + __ffs(left) - 1;
    __syncwarp();
    const bool takes = lane8 < a.k;
    const int e = mine_e[takes ? lane8 : 0];
    const float v = takes ? mine_s[e + e / V * kPad] : 0.f;
    const float f = a.renorm ? a.scale / (seg_sum(v) + kTopkEps) : a.scale;
    if (takes && valid) {
      expert_idx[t * a.k + lane8] = e;
      gate_w[t * a.k + lane8] = v * f;
    }
    __syncwarp();
  }
}

// dl from the gradient of the weights and, if given, one of the scores that all tokens share (the balance loss).
//   ds_c = scale / (S + eps) (g_c - sum_j g_j s_j / (S + eps)), S the sum of the chosen s;  without renorm scale g_c
//   softmax: dl = s (ds - sum ds s)      sigmoid: dl = ds s (1 - s)
// Lanes 0 to k - 1 hold the chosen pairs; rows of shared memory carry s to them and ds back.  T 65536, E 128, k 8: 18 us, of 11 by the bytes; 190
// instructions a token, issued in 77 % of the clocks.
template <int VPT, bool Full>
__global__ void __launch_bounds__(kTopkWarps * 32)
topk_bwd_kernel(const float* __restrict__ logits, const int32_t* __restrict__ expert_idx, const float* __restrict__ dgate_w,
                const float* __restrict__ dscores_col, float* __restrict__ dlogits, TopkArgs a) {
  __shared__ __align__(16) float rows[kTopkWarps][2][kMaxE];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, e0 = lane * VPT;
  float* srow = rows[warp][0];
  float* grow = rows[warp][1];
  float col[VPT];
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    col[j] = dscores_col && e0 + j < a.E ? __ldg(dscores_col + e0 + j) : 0.f;
    grow[e0 + j] = 0.f;
  }
  __syncwarp();                                                        // before a first token's gradients: sigmoid without renorm has no other barrier ahead of them
  const int64_t step = gridDim.x * kTopkWarps;
  int64_t t = blockIdx.x * kTopkWarps + warp;
  float next[VPT], next_g = 0.f;
  int next_e = -1;
  auto load = [&](int64_t tok) {
    topk_load_row<VPT, Full>(logits + tok * a.E, a.E, lane, next);
    if (lane < a.k) {
      next_e = __ldg(expert_idx + tok * a.k + lane);
      next_g = __ldg(dgate_w + tok * a.k + lane);
    }
  };
  if (t < a.T) load(t);
  for (; t < a.T; t += step) {
    float l[VPT], s[VPT], rest[VPT];
#pragma unroll
    for (int j = 0; j < VPT; ++j) l[j] = next[j];
    const bool valid = next_e >= 0 && next_e < a.E;                    // an empty pair (-1) has no score and takes no gradient
    const int e = valid ? next_e : 0;
    float g = valid ? a.scale * next_g : 0.f;
    if (t + step < a.T) load(t + step);
    topk_scores<VPT, Full>(l, a.E, lane, a.sigmoid, s, rest);
    float dot = 0.f;                                                   // sum of ds s over the row
    if (a.renorm || !a.sigmoid) {
#pragma unroll
      for (int j = 0; j < VPT; ++j) srow[e0 + j] = s[j];
      __syncwarp();
      const float p = valid ? srow[e] : 0.f;
      auto sum8 = [](float v) {                                        // over lanes 0 to 7: the others hold zeros
        v += __shfl_xor_sync(0xffffffffu, v, 4); v += __shfl_xor_sync(0xffffffffu, v, 2); v += __shfl_xor_sync(0xffffffffu, v, 1);
        return v;
      };
      if (a.renorm) {
        const float inv = 1.f / (sum8(p) + kTopkEps), mean = sum8(g * p) * inv;       // every lane takes part in the sums
        g = valid ? (g - mean) * inv : 0.f;
      }
      if (!a.sigmoid) dot = __shfl_sync(0xffffffffu, sum8(g * p), 0);
    }
    if (!a.sigmoid && dscores_col) {
      float v = 0.f;
#pragma unroll
      for (int j = 0; j < VPT; ++j) if (e0 + j < a.E) v += col[j] * s[j];
      dot += warp_sum(v);
    }
    if (valid) grow[e] = g;
    __syncwarp();
    float o[VPT];
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const float ds = grow[e0 + j] + col[j];
      o[j] = a.sigmoid ? ds * s[j] * rest[j] : s[j] * (ds - dot);
    }
    topk_store_row<VPT, Full>(dlogits + t * a.E, a.E, lane, o);
    __syncwarp();
    if (valid) grow[e] = 0.f;
    __syncwarp();
  }
}

}  // namespace msr
