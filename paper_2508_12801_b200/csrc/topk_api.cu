// C ABI of routing by top-k (see include/maxscore.h): argument checks and kernel launches on the caller's stream.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "common.cuh"
#include "context.cuh"
#include "topk.cuh"

using namespace msr;

namespace {

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

maxscore_status topk_args(const maxscore_ctx* c, const maxscore_topk* how, TopkArgs* out) {
  if (!c || !how) return MAXSCORE_ERR_INVALID_ARG;
  auto flag = [](int32_t v) { return v == 0 || v == 1; };
  if (!flag(how->score) || !flag(how->group_pairs) || !flag(how->renorm) || !isfinite(how->scale)) return MAXSCORE_ERR_INVALID_ARG;
  TopkArgs a{};
  a.T = c->p.T; a.E = c->p.E; a.k = c->p.k;
  a.n_group = 1; a.topk_group = 1; a.group_size = a.E;
  if (how->n_group < 0) return MAXSCORE_ERR_INVALID_ARG;
  if (how->n_group > 1) {
    if (a.E % how->n_group || how->topk_group < 1 || how->topk_group > how->n_group) return MAXSCORE_ERR_INVALID_ARG;
    if (how->n_group > kTopkMaxGroups) return MAXSCORE_ERR_UNSUPPORTED;
    const int size = a.E / how->n_group;
    if (how->topk_group * size < a.k) return MAXSCORE_ERR_INVALID_ARG;
    if (how->topk_group < how->n_group) { a.n_group = how->n_group; a.topk_group = how->topk_group; a.group_size = size; }
  }
  a.sigmoid = how->score; a.pairs = how->group_pairs; a.renorm = how->renorm; a.scale = how->scale;
  *out = a;
  return MAXSCORE_OK;
}

// tokens: of a warp
int topk_grid(const maxscore_ctx* c, int tokens) {
  const int64_t each = (int64_t)kTopkWarps * tokens;
  return (int)std::min<int64_t>((c->p.T + each - 1) / each, (int64_t)c->sm_count * 8);
}

// experts of a lane: rows of up to 32, 64, 96 and 128; rows of 64 and 128 are moved as vectors
template <typename F>
void topk_by_width(int E, F go) {
  using std::false_type; using std::true_type;
  if (E <= 32) go(std::integral_constant<int, 1>{}, false_type{});
  else if (E < 64) go(std::integral_constant<int, 2>{}, false_type{});
  else if (E == 64) go(std::integral_constant<int, 2>{}, true_type{});
  else if (E <= 96) go(std::integral_constant<int, 3>{}, false_type{});
  else if (E < 128) go(std::integral_constant<int, 4>{}, false_type{});
  else go(std::integral_constant<int, 4>{}, true_type{});
}

}  // namespace

extern "C" {

maxscore_status maxscore_topk_fwd(maxscore_ctx* c, const float* logits, const float* bias, const maxscore_topk* how, float* scores,
                                  int32_t* expert_idx, float* gate_w, void* stream) {
  TopkArgs a;
  maxscore_status s = topk_args(c, how, &a);
  if (s) return s;
  if (!logits || !expert_idx || !gate_w || !aligned16(logits) || !aligned16(scores) || !aligned4(bias) || !aligned4(expert_idx) || !aligned4(gate_w))
    return MAXSCORE_ERR_INVALID_ARG;
  const size_t rows = sizeof(float) * (size_t)a.T * a.E, pairs = sizeof(float) * (size_t)a.T * a.k;
  if (!apart({{scores, rows}, {expert_idx, pairs}, {gate_w, pairs}}, {{logits, rows}, {bias, sizeof(float) * (size_t)a.E}}))
    return MAXSCORE_ERR_INVALID_ARG;
  const int v = a.E <= 16 ? 2 : a.E <= 32 ? 4 : a.E <= 64 ? 8 : 16, lanes = a.group_size / v;       // experts of a lane of eight
  // Eight lanes a token, or a warp where its tokens are resident at once.  us, E 128, k 8 (with groups, bias and scores): T 1 2.7 / 2.2 (3.8 / 2.9),
  // 1024 3.7 / 2.6, 2048 3.8 / 3.0, 4096 3.8 / 4.5, 16384 6.8 / 10.3 (16.5 / 21.0).
  const bool many = c->p.T > 16 * c->sm_count;
  if (many && (a.n_group == 1 || (a.group_size % v == 0 && (lanes & (lanes - 1)) == 0))) {
    while (a.n_group > 1 && 1 << a.group_shift < lanes) ++a.group_shift;
    auto go = [&](auto per_lane, auto whole) {
      constexpr int V = decltype(per_lane)::value;
      constexpr bool F = decltype(whole)::value;
      auto kernel = a.n_group == 1 ? topk_fwd_kernel<V, false, F> : topk_fwd_kernel<V, true, F>;
      kernel<<<topk_grid(c, 4), kTopkWarps * 32, 0, (cudaStream_t)stream>>>(logits, bias, scores, expert_idx, gate_w, a);
    };
    auto by = [&](auto per_lane) { if (a.E == 8 * decltype(per_lane)::value) go(per_lane, std::true_type{}); else go(per_lane, std::false_type{}); };
    if (v == 2) by(std::integral_constant<int, 2>{});
    else if (v == 4) by(std::integral_constant<int, 4>{});
    else if (v == 8) by(std::integral_constant<int, 8>{});
    else by(std::integral_constant<int, 16>{});
  } else {
    topk_by_width(a.E, [&](auto w, auto whole) {
      topk_fwd_scan_kernel<decltype(w)::value, decltype(whole)::value><<<topk_grid(c, 1), kTopkWarps * 32, 0, (cudaStream_t)stream>>>(
          logits, bias, scores, expert_idx, gate_w, a);
    });
  }
  MS_LAUNCH_CHECK("topk_fwd_kernel");
  c->launches += 1;
  return MAXSCORE_OK;
}

maxscore_status maxscore_topk_bwd(maxscore_ctx* c, const float* logits, const int32_t* expert_idx, const float* dgate_w,
                                  const float* dscores_col, const maxscore_topk* how, float* dlogits, void* stream) {
  TopkArgs a;
  maxscore_status s = topk_args(c, how, &a);
  if (s) return s;
  if (!logits || !expert_idx || !dgate_w || !dlogits || !aligned16(logits) || !aligned16(dlogits) || !aligned4(expert_idx) ||
      !aligned4(dgate_w) || !aligned4(dscores_col))
    return MAXSCORE_ERR_INVALID_ARG;
  const size_t rows = sizeof(float) * (size_t)a.T * a.E, pairs = sizeof(float) * (size_t)a.T * a.k;
  if (!apart({{dlogits, rows}}, {{logits, rows}, {expert_idx, pairs}, {dgate_w, pairs}, {dscores_col, sizeof(float) * (size_t)a.E}}))
    return MAXSCORE_ERR_INVALID_ARG;
  topk_by_width(a.E, [&](auto w, auto whole) {
    topk_bwd_kernel<decltype(w)::value, decltype(whole)::value><<<topk_grid(c, 1), kTopkWarps * 32, 0, (cudaStream_t)stream>>>(logits, expert_idx, dgate_w, dscores_col,
                                                                                                      dlogits, a);
  });
  MS_LAUNCH_CHECK("topk_bwd_kernel");
  c->launches += 1;
  return MAXSCORE_OK;
}

}  // extern "C"
