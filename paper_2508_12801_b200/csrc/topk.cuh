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
// A warp owns a token, a lane VPT consecutive experts (so the lowest lane holds the lowest index and a ballot settles ties).  The k
// largest come out one by one: a warp-wide maximum of order-preserving integers, a ballot, and the owner takes the next of its own.
// The row is read once and what is written is k pairs (and the scores, if they are wanted); next to 4 E bytes of logits the
// instructions count (see the figures at the launch).
#pragma once
#include "common.cuh"

namespace msr {

constexpr int kTopkWarps = 8, kTopkMaxGroups = 32;
constexpr float kTopkEps = 1e-20f;     // in the denominator of the weights: a row whose chosen scores all vanish gets zeros

struct TopkArgs {
  int T, E, k;
  int n_group, topk_group, group_size, group_lanes;      // group_lanes: lanes of a group where that is a power of two, else 0
  int sigmoid, pairs, renorm;
  float scale;
};

// Integers in the order of floats, -0 equal to 0, none of them 0, which stands for "cannot be chosen".  (NaN: first or last by its sign.)
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float order_value(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }

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
  const float t = exp_down(-fabsf(l)), r = __fdividef(1.f, 1.f + t), tr = t * r;
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
  double m = -INFINITY, sum = 0.0;
  if (!a.sigmoid) {
    for (int j = 0; j < vpt; ++j) if (e0 + j < a.E) m = fmax(m, (double)__ldg(row + e0 + j));
    for (int o = 16; o > 0; o >>= 1) m = fmax(m, __shfl_xor_sync(0xffffffffu, m, o));
    for (int j = 0; j < vpt; ++j) if (e0 + j < a.E) sum += exp((double)__ldg(row + e0 + j) - m);
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  }
  auto order = [](double x) { return x == x ? x : -INFINITY; };      // NaN comes last
  __syncwarp();
  for (int j = 0; j < vpt; ++j)
    if (e0 + j < a.E) {
      const double l = (double)__ldg(row + e0 + j);
      const double s = a.sigmoid ? 1.0 / (1.0 + exp(-l)) : exp(l - m) / sum;
      d[e0 + j] = order(bias ? s + (double)__ldg(bias + e0 + j) : s);
    }
  __syncwarp();
  uint32_t kept = 1u;
  if (a.n_group > 1) {
    double m1 = -INFINITY, m2 = -INFINITY;
    if (lane < a.n_group)
      for (int i = 0; i < a.group_size; ++i) {
        const double x = d[lane * a.group_size + i];
        if (x > m1) { m2 = m1; m1 = x; } else if (x > m2) m2 = x;
      }
    const double value = order(a.pairs && a.group_size > 1 ? m1 + m2 : m1);
    int before = 0;
    for (int g = 0; g < a.n_group; ++g) {
      const double other = __shfl_sync(0xffffffffu, value, g);
      before += other > value || (other == value && g < lane);
    }
    kept = __ballot_sync(0xffffffffu, lane < a.n_group && before < a.topk_group);
  }
  if (!bias) {                                          // the experts themselves by their logits, as in fp32
    __syncwarp();
    for (int j = 0; j < vpt; ++j) if (e0 + j < a.E) d[e0 + j] = order((double)__ldg(row + e0 + j));
    __syncwarp();
  }
  uint32_t chosen = 0;
  for (int j = 0; j < vpt; ++j) {
    const int e = e0 + j;
    if (e >= a.E || !(kept >> (e / a.group_size) & 1)) continue;
    int before = 0;
    for (uint32_t rest = kept; rest; rest &= rest - 1) {
      const int first = (__ffs(rest) - 1) * a.group_size;
      for (int i = first; i < first + a.group_size; ++i) before += d[i] > d[e] || (d[i] == d[e] && i < e);
    }
    if (before < a.k) chosen |= 1u << j;
  }
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

// Groups: 0 none; 1 of `group_lanes` lanes each, a power of two; 2 of any size.
template <int VPT, int Groups, bool Full>
__global__ void __launch_bounds__(kTopkWarps * 32)
topk_fwd_kernel(const float* __restrict__ logits, const float* __restrict__ bias, float* __restrict__ scores, int32_t* __restrict__ expert_idx,
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
    group[j] = Groups == 2 ? min((e0 + j) / a.group_size, kTopkMaxGroups - 1) : 0;
  }
  const int group_stride = Groups == 1 ? a.group_lanes : 1;            // lanes that speak for the groups: g * group_stride
  const int my_group = lane / group_stride;
  const bool speaks = my_group < a.n_group;
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
    if (Groups) {
      // the two largest of each group (NaN counts as nothing)
      if (!bias && a.pairs) {
#pragma unroll
        for (int j = 0; j < VPT; ++j) c[j] = s[j];
      }
      float m1 = -INFINITY, m2 = -INFINITY;
      auto take = [&](float x) { m2 = fmaxf(m2, fminf(m1, x)); m1 = fmaxf(m1, x); };
      if (Groups == 1) {
#pragma unroll
        for (int j = 0; j < VPT; ++j) if (Full || e0 + j < a.E) take(c[j]);
        for (int o = 1; o < a.group_lanes; o <<= 1) {
          const float o1 = __shfl_xor_sync(0xffffffffu, m1, o), o2 = __shfl_xor_sync(0xffffffffu, m2, o);
          m2 = fmaxf(fminf(m1, o1), fmaxf(m2, o2));
          m1 = fmaxf(m1, o1);
        }
      } else {
#pragma unroll
        for (int j = 0; j < VPT; ++j) if (Full || e0 + j < a.E) grouped[e0 + j + group[j]] = c[j];
        __syncwarp();
        if (lane < a.n_group)
          for (int i = 0; i < a.group_size; ++i) take(grouped[lane * (a.group_size + 1) + i]);
        __syncwarp();
      }
      const uint32_t mine = speaks ? order_key(a.pairs && a.group_size > 1 ? m1 + m2 : m1) : 0u;
      // the best leave one by one; where equal ones left together, every group counts those before it instead
      uint32_t head = mine, worst = 0;
#pragma unroll 1
      for (int g = 0; g < a.topk_group; ++g) {
        worst = __reduce_max_sync(0xffffffffu, head);
        head = head == worst ? 0u : head;
      }
      bool in = speaks && mine >= worst;
      if (__popc(__ballot_sync(0xffffffffu, in)) != a.topk_group * group_stride) {
        int before = 0;
        for (int g = 0; g < a.n_group; ++g) before += __shfl_sync(0xffffffffu, mine, g * group_stride) >= mine + (g >= my_group);
        in = speaks && before < a.topk_group;
      }
      if (bias || a.pairs) {
        const float low = order_value(__reduce_min_sync(0xffffffffu, in ? mine : 0xffffffffu));
        const float high = order_value(__reduce_max_sync(0xffffffffu, in ? 0u : mine));
        near = !(low - high > 0x1p-18f + 0x1p-21f * fabsf(low));       // two terms, hence twice the bound below
      }
      if (Groups == 1) {
#pragma unroll
        for (int j = 0; j < VPT; ++j) key[j] = in ? key[j] : 0u;
      } else {
        const uint32_t kept = __ballot_sync(0xffffffffu, in);
#pragma unroll
        for (int j = 0; j < VPT; ++j) if (!(kept >> group[j] & 1)) key[j] = 0u;
      }
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

// dl from the gradient of the weights and, if given, one of the scores that all tokens share (the balance loss).
//   ds_c = scale / (S + eps) (g_c - sum_j g_j s_j / (S + eps)), S the sum of the chosen s;  without renorm scale g_c
//   softmax: dl = s (ds - sum ds s)      sigmoid: dl = ds s (1 - s)
// Lanes 0 to k - 1 hold the chosen pairs; rows of shared memory carry s to them and ds back.
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
