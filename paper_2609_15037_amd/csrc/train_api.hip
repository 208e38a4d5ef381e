// C ABI of the operators beside the projected update: validation and launches. Nothing is allocated,
// nothing synchronises, and no state is kept between calls.
#include <math.h>

#include "../../include/moara.h"
#include "train.h"

namespace {

#define TRAIN_TRY(expr)                                                                            \
  do {                                                                                             \
    const hipError_t e_ = (expr);                                                                  \
    if (e_ != hipSuccess) return moara_fail(MOARA_E_HIP, "%s: %s", #expr, hipGetErrorString(e_));  \
  } while (0)

// A launch has fewer than 2^32 threads: 2^22 workgroups of 512, as many as the largest tensor takes.
constexpr int64_t MAX_COUNT = (int64_t)1 << 33;      // elements of one tensor
constexpr uint32_t MAX_TILES = 1u << 22;             // workgroups of one AdamW launch

bool misaligned(const void* p, int size) { return ((uintptr_t)p & (uintptr_t)(size - 1)) != 0; }

int check_grads(const moara_grad_tensor* t, int32_t n) {
  if (n < 0 || (n > 0 && !t)) return moara_fail(MOARA_E_ARG, "null tensor list");
  for (int i = 0; i < n; ++i) {
    if (t[i].dtype != MOARA_F32 && t[i].dtype != MOARA_BF16) return moara_fail(MOARA_E_ARG, "tensor %d: bad dtype", i);
    if (t[i].count < 0 || t[i].count > MAX_COUNT)
      return moara_fail(MOARA_E_SHAPE, "tensor %d: count %lld", i, (long long)t[i].count);
    if (t[i].grad && misaligned(t[i].grad, t[i].dtype == MOARA_BF16 ? 2 : 4))
      return moara_fail(MOARA_E_ARG, "tensor %d: pointer not aligned to its type", i);
  }
  return MOARA_OK;
}

// The list in launches of at most GRAD_MAX tensors: launch(list) for each.
template <typename F> int each_grad_list(const moara_grad_tensor* t, int32_t n, F launch) {
  GradList l{};
  for (int i = 0; i < n; ++i) {
    if (!t[i].grad || t[i].count == 0) continue;
    if (l.n == GRAD_MAX) {
      TRAIN_TRY(launch(l));
      l = GradList{};
    }
    l.g[l.n] = t[i].grad;
    l.count[l.n] = t[i].count;
    l.start[l.n] = l.tiles;
    if (t[i].dtype == MOARA_BF16) l.bf16[l.n >> 5] |= 1u << (l.n & 31);
    l.tiles += grad_tiles(t[i].count);
    ++l.n;
  }
  if (l.n) TRAIN_TRY(launch(l));
  return MOARA_OK;
}

// Whether the gradients take more than the memory-side cache holds.
bool over_cache(const moara_grad_tensor* t, int32_t n) {
  int64_t bytes = 0;
  for (int i = 0; i < n; ++i)
    if (t[i].grad) bytes += t[i].count * (t[i].dtype == MOARA_BF16 ? 2 : 4);
  return bytes > (int64_t)256 << 20;
}

int check_route(const moara_route_config* c, const void* logits, int64_t tokens, int64_t row_stride) {
  if (!c) return moara_fail(MOARA_E_ARG, "null config");
  if (c->experts < 1 || c->top_k < 1 || c->top_k > c->experts)
    return moara_fail(MOARA_E_ARG, "top_k %d of %d experts", c->top_k, c->experts);
  if (c->groups < 1 || c->top_groups < 1 || c->top_groups > c->groups || c->experts % c->groups)
    return moara_fail(MOARA_E_ARG, "%d of %d groups of %d experts", c->top_groups, c->groups, c->experts);
  if (c->top_k > c->experts / c->groups * c->top_groups)
    return moara_fail(MOARA_E_ARG, "top_k %d exceeds the %d experts of the kept groups", c->top_k,
                      c->experts / c->groups * c->top_groups);
  if (c->group_best != 1 && c->group_best != 2) return moara_fail(MOARA_E_ARG, "group_best must be 1 or 2");
  if (c->score != MOARA_SOFTMAX && c->score != MOARA_SIGMOID) return moara_fail(MOARA_E_ARG, "bad score function");
  if (c->logits_dtype != MOARA_F32 && c->logits_dtype != MOARA_BF16) return moara_fail(MOARA_E_ARG, "bad logits dtype");
  if (!isfinite(c->scale)) return moara_fail(MOARA_E_ARG, "scale is not finite");
  if (c->experts > ROUTE_MAX_EXPERTS || c->top_k > ROUTE_MAX_K || c->groups > ROUTE_MAX_GROUPS)
    return moara_fail(MOARA_E_UNSUPPORTED, "at most %d experts, top_k %d and %d groups", ROUTE_MAX_EXPERTS, ROUTE_MAX_K,
                      ROUTE_MAX_GROUPS);
  if (tokens < 0 || tokens > (int64_t)1 << 40) return moara_fail(MOARA_E_SHAPE, "bad token count");
  if (tokens > 0 && !logits) return moara_fail(MOARA_E_ARG, "null logits");
  if (row_stride < c->experts && tokens > 1) return moara_fail(MOARA_E_SHAPE, "rows overlap: stride %lld", (long long)row_stride);
  if (misaligned(logits, c->logits_dtype == MOARA_BF16 ? 2 : 4))
    return moara_fail(MOARA_E_ARG, "logits not aligned to their type");
  return MOARA_OK;
}

RouteParams route_params(const moara_route_config* c, const void* logits, int64_t tokens, int64_t row_stride) {
  RouteParams p{};
  p.logits = logits;
  p.tokens = tokens;
  p.ld = row_stride;
  p.E = c->experts;
  p.k = c->top_k;
  p.groups = c->groups;
  p.top_groups = c->top_groups;
  p.group_best = c->group_best;
  p.group_size = (uint32_t)(c->experts / c->groups);
  p.group_inv = ((1u << 20) + p.group_size - 1) / p.group_size;
  p.sigmoid = c->score == MOARA_SIGMOID;
  p.renorm = c->renormalise != 0;
  p.bf16 = c->logits_dtype == MOARA_BF16;
  p.scale = c->scale;
  return p;
}

}  // namespace

extern "C" {

int moara_grad_norm(const moara_grad_tensor* tensors, int32_t n, float max_norm, float* out, void* workspace,
                    void* stream) {
  const int rc = check_grads(tensors, n);
  if (rc != MOARA_OK) return rc;
  if (!out || !workspace) return moara_fail(MOARA_E_ARG, "null out or workspace");
  if (misaligned(out, 4) || misaligned(workspace, 8)) return moara_fail(MOARA_E_ARG, "out or workspace not aligned");
  if (!(max_norm > 0)) return moara_fail(MOARA_E_ARG, "max_norm must be positive");
  static_assert(sizeof(double) * NORM_WGS <= MOARA_GRAD_NORM_WORKSPACE, "workspace of moara_grad_norm");
  double* const partial = (double*)workspace;
  const bool once = over_cache(tensors, n);
  uint32_t filled = 0;
  const int rl = each_grad_list(tensors, n, [&](const GradList& l) {
    return launch_grad_norm(l, once, partial, filled, (hipStream_t)stream);
  });
  if (rl != MOARA_OK) return rl;
  TRAIN_TRY(launch_grad_norm_end(partial, filled, max_norm, out, (hipStream_t)stream));
  return MOARA_OK;
}

int moara_grad_scale(const moara_grad_tensor* tensors, int32_t n, const float* coef, void* stream) {
  const int rc = check_grads(tensors, n);
  if (rc != MOARA_OK) return rc;
  if (!coef || misaligned(coef, 4)) return moara_fail(MOARA_E_ARG, "null or misaligned coefficient");
  const bool once = over_cache(tensors, n);
  return each_grad_list(tensors, n, [&](const GradList& l) { return launch_grad_scale(l, once, coef, (hipStream_t)stream); });
}

int moara_adamw_default_config(moara_adamw_config* out) {
  if (!out) return moara_fail(MOARA_E_ARG, "null config");
  out->beta1 = 0.9;
  out->beta2 = 0.999;
  out->eps = 1e-6;
  out->bits = 32;
  out->reserved = 0;
  return MOARA_OK;
}

int moara_adamw_step(const moara_adamw_config* cfg, const moara_adamw_tensor* tensors, int32_t n, const float* clip,
                     uint64_t seed, void* stream) {
  if (!cfg || n < 0 || (n > 0 && !tensors)) return moara_fail(MOARA_E_ARG, "null config or tensor list");
  if (n >= 1 << (64 - ADAMW_PLACE_BIT)) return moara_fail(MOARA_E_ARG, "%d tensors", n);
  if (cfg->bits != 8 && cfg->bits != 32) return moara_fail(MOARA_E_ARG, "moments of %d bits (8 or 32)", cfg->bits);
  if (!(cfg->beta1 >= 0 && cfg->beta1 < 1) || !(cfg->beta2 >= 0 && cfg->beta2 < 1))
    return moara_fail(MOARA_E_ARG, "beta outside [0, 1)");
  if (!(cfg->eps > 0) || !isfinite(cfg->eps)) return moara_fail(MOARA_E_ARG, "eps must be positive");
  if (misaligned(clip, 4)) return moara_fail(MOARA_E_ARG, "clip not aligned");
  const bool q = cfg->bits == 8;
  for (int i = 0; i < n; ++i) {
    const moara_adamw_tensor& t = tensors[i];
    if ((t.param_dtype != MOARA_F32 && t.param_dtype != MOARA_BF16) ||
        (t.grad_dtype != MOARA_F32 && t.grad_dtype != MOARA_BF16))
      return moara_fail(MOARA_E_ARG, "tensor %d: bad dtype", i);
    if (t.count < 0 || t.count > MAX_COUNT)
      return moara_fail(MOARA_E_SHAPE, "tensor %d: count %lld", i, (long long)t.count);
    if (!t.grad || t.count == 0) continue;
    if (!t.param || !t.exp_avg || !t.exp_avg_sq || (q && !t.scales))
      return moara_fail(MOARA_E_ARG, "tensor %d: null parameter or moment", i);
    if (misaligned(t.param, t.param_dtype == MOARA_BF16 ? 2 : 4) || misaligned(t.grad, t.grad_dtype == MOARA_BF16 ? 2 : 4) ||
        (!q && (misaligned(t.exp_avg, 4) || misaligned(t.exp_avg_sq, 4))))
      return moara_fail(MOARA_E_ARG, "tensor %d: pointer not aligned to its type", i);
    if (t.step < 1) return moara_fail(MOARA_E_ARG, "tensor %d: step %lld", i, (long long)t.step);
    if (!isfinite(t.lr) || !isfinite(t.weight_decay)) return moara_fail(MOARA_E_ARG, "tensor %d: lr or decay not finite", i);
  }
  AdamwList l;
  l.clip = clip;
  l.seed = seed;
  l.b1 = (float)cfg->beta1;
  l.c1 = (float)(1 - cfg->beta1);
  l.b2 = (float)cfg->beta2;
  l.c2 = (float)(1 - cfg->beta2);
  l.eps = (float)cfg->eps;
  // tensors of one pair of types share launches, those of one step, rate and decay a set of numbers
  for (int kind = 0; kind < 4; ++kind) {
    uint32_t total = 0;
    int sets = 0;
    l.n = 0;
    auto launch = [&] { return launch_adamw(l, (kind & 1) != 0, (kind & 2) != 0, cfg->bits, total, (hipStream_t)stream); };
    for (int i = 0; i < n; ++i) {
      const moara_adamw_tensor& t = tensors[i];
      if (!t.grad || t.count == 0) continue;
      if ((t.param_dtype == MOARA_BF16 ? 1 : 0) + (t.grad_dtype == MOARA_BF16 ? 2 : 0) != kind) continue;
      const AdamwSet set = {(float)(1 - t.lr * t.weight_decay), (float)(t.lr / (1 - pow(cfg->beta1, (double)t.step))),
                            (float)(1 / (1 - pow(cfg->beta2, (double)t.step)))};
      const uint32_t tiles = adamw_tiles(t.count);
      int at = 0;
      while (at < sets && (l.set[at].decay != set.decay || l.set[at].lr != set.lr || l.set[at].rbc2 != set.rbc2)) ++at;
      if (l.n == ADAMW_MAX || at == ADAMW_SETS || (l.n && total + tiles > MAX_TILES)) {
        TRAIN_TRY(launch());
        total = 0;
        l.n = sets = at = 0;
      }
      if (at == sets) l.set[sets++] = set;
      l.p[l.n] = t.param;
      l.g[l.n] = t.grad;
      l.m[l.n] = t.exp_avg;
      l.v[l.n] = t.exp_avg_sq;
      l.scales[l.n] = (uint8_t*)t.scales;
      l.about[l.n] = (uint64_t)t.count | (uint64_t)at << ADAMW_SET_BIT | (uint64_t)i << ADAMW_PLACE_BIT;
      l.start[l.n++] = total;
      total += tiles;
    }
    if (l.n) TRAIN_TRY(launch());
  }
  return MOARA_OK;
}

int moara_route_default_config(moara_route_config* out) {
  if (!out) return moara_fail(MOARA_E_ARG, "null config");
  *out = moara_route_config{64, 6, 1, 1, 1, MOARA_SOFTMAX, 0, MOARA_F32, 1.0f};
  return MOARA_OK;
}

int moara_route(const moara_route_config* cfg, const void* logits, int64_t tokens, int64_t row_stride, const float* bias,
                const uint8_t* mask, int32_t* out_index, float* out_weight, int64_t* counts, void* stream) {
  const int rc = check_route(cfg, logits, tokens, row_stride);
  if (rc != MOARA_OK) return rc;
  if (tokens == 0) return MOARA_OK;
  if (!out_index || !out_weight) return moara_fail(MOARA_E_ARG, "null output");
  if (misaligned(out_index, 4) || misaligned(out_weight, 4) || misaligned(bias, 4) || misaligned(counts, 8))
    return moara_fail(MOARA_E_ARG, "pointer not aligned to its type");
  RouteParams p = route_params(cfg, logits, tokens, row_stride);
  p.bias = bias;
  p.mask = mask;
  p.index = out_index;
  p.weight = out_weight;
  p.counts = (unsigned long long*)counts;
  TRAIN_TRY(launch_route(p, (hipStream_t)stream));
  return MOARA_OK;
}

int moara_route_backward(const moara_route_config* cfg, const void* logits, int64_t tokens, int64_t row_stride,
                         const int32_t* index, const float* grad_weight, void* out_grad, void* stream) {
  const int rc = check_route(cfg, logits, tokens, row_stride);
  if (rc != MOARA_OK) return rc;
  if (tokens == 0) return MOARA_OK;
  if (!index || !grad_weight || !out_grad) return moara_fail(MOARA_E_ARG, "null index, gradient or output");
  if (misaligned(index, 4) || misaligned(grad_weight, 4) || misaligned(out_grad, cfg->logits_dtype == MOARA_BF16 ? 2 : 4))
    return moara_fail(MOARA_E_ARG, "pointer not aligned to its type");
  RouteParams p = route_params(cfg, logits, tokens, row_stride);
  p.index = const_cast<int32_t*>(index);
  p.weight = const_cast<float*>(grad_weight);
  p.grad = out_grad;
  TRAIN_TRY(launch_route_backward(p, (hipStream_t)stream));
  return MOARA_OK;
}

int moara_route_balance(int32_t experts, int64_t* counts, float* bias, float rate, void* stream) {
  if (experts < 1 || experts > ROUTE_MAX_EXPERTS) return moara_fail(MOARA_E_ARG, "%d experts", experts);
  if (!counts || !bias || misaligned(counts, 8) || misaligned(bias, 4))
    return moara_fail(MOARA_E_ARG, "null or misaligned counts or bias");
  if (!isfinite(rate)) return moara_fail(MOARA_E_ARG, "rate is not finite");
  TRAIN_TRY(launch_route_balance(experts, (long long*)counts, bias, rate, (hipStream_t)stream));
  return MOARA_OK;
}

}  // extern "C"
