// C ABI of the losses: validation and launches. Nothing is allocated, nothing synchronises, and no state is kept
// between calls.
#include <math.h>

#include "../../include/moara.h"
#include "train.h"

namespace {

#define LOSS_TRY(expr)                                                                             \
  do {                                                                                             \
    const hipError_t e_ = (expr);                                                                  \
    if (e_ != hipSuccess) return moara_fail(MOARA_E_HIP, "%s: %s", #expr, hipGetErrorString(e_));  \
  } while (0)

bool misaligned(const void* p, int size) { return ((uintptr_t)p & (uintptr_t)(size - 1)) != 0; }
constexpr int64_t MAX_STRIDE = (int64_t)1 << 44;
int size_of(int32_t dtype) { return dtype == MOARA_BF16 ? 2 : 4; }

int check_packed(Packed& q, const uint8_t* mask, int64_t tokens, const int64_t* offsets, int64_t sequences) {
  if (tokens < 0 || tokens > MAX_LOSS_TOKENS || sequences < 1 || sequences > MAX_SEQUENCES)
    return moara_fail(MOARA_E_SHAPE, "%lld tokens in %lld sequences", (long long)tokens, (long long)sequences);
  if (!offsets && tokens % sequences)
    return moara_fail(MOARA_E_SHAPE, "%lld tokens are no %lld equal sequences", (long long)tokens, (long long)sequences);
  if (misaligned(offsets, 8)) return moara_fail(MOARA_E_ARG, "offsets not aligned to their type");
  q = Packed{offsets, mask, tokens, sequences, offsets ? 0 : tokens / sequences};
  return MOARA_OK;
}

int check_logps(LogpsParams& p, const void* logits, int32_t dtype, int64_t tokens, int64_t vocab, int64_t row_stride,
                int64_t inner, int64_t outer_stride, float scale, const int64_t* labels) {
  if (dtype != MOARA_F32 && dtype != MOARA_BF16) return moara_fail(MOARA_E_ARG, "bad logits dtype");
  if (tokens < 0 || tokens > (int64_t)1 << 40 || vocab < 1 || vocab > (int64_t)1 << 30)
    return moara_fail(MOARA_E_SHAPE, "%lld tokens, vocabulary of %lld", (long long)tokens, (long long)vocab);
  const float log2_scale = (float)(scale * 1.4426950408889634);
  if (!(scale > 0) || !isfinite(log2_scale)) return moara_fail(MOARA_E_ARG, "scale must be positive, below 2.3e38");
  if (tokens == 0) return MOARA_OK;
  if (inner < 1 || (inner > 1 && tokens > 1 && row_stride < vocab) || (inner < tokens && outer_stride < vocab) ||
      row_stride > MAX_STRIDE || outer_stride > MAX_STRIDE)
    return moara_fail(MOARA_E_SHAPE, "rows overlap: strides %lld, %lld of %lld rows", (long long)row_stride,
                      (long long)outer_stride, (long long)inner);
  if (!logits || !labels || misaligned(logits, size_of(dtype)) || misaligned(labels, 8))
    return moara_fail(MOARA_E_ARG, "null or misaligned logits or labels");
  p = LogpsParams{};
  p.logits = logits;
  p.tokens = tokens;
  p.vocab = vocab;
  p.ld = row_stride;
  p.inner = inner;
  p.outer = outer_stride;
  p.labels = labels;
  p.scale = scale;
  p.log2_scale = log2_scale;
  p.bf16 = dtype == MOARA_BF16;
  return MOARA_OK;
}

int check_preference(const Packed& q) {
  if (q.sequences % 2) return moara_fail(MOARA_E_SHAPE, "%lld sequences are no pairs", (long long)q.sequences);
  return MOARA_OK;
}

int check_policy(const moara_policy_config* c, PolicyParams& p, const float* logp, const float* old_logp,
                 const float* ref_logp, const float* advantages, const uint8_t* mask, int64_t tokens, const int64_t* offsets,
                 int64_t sequences) {
  if (!c) return moara_fail(MOARA_E_ARG, "null config");
  if (!(c->clip_low >= 0 && c->clip_low <= 1) || !(c->clip_high >= 0))
    return moara_fail(MOARA_E_ARG, "clipping to [1 - %g, 1 + %g]", c->clip_low, c->clip_high);
  if (!isfinite(c->kl_coef) || !isfinite(c->entropy_coef) || !isfinite(c->divisor) || c->divisor < 0)
    return moara_fail(MOARA_E_ARG, "a coefficient or the divisor is not finite, or the divisor is negative");
  if (c->kl < MOARA_KL_EXP || c->kl > MOARA_KL_SQUARE) return moara_fail(MOARA_E_ARG, "bad kl");
  if (c->reduce != MOARA_MEAN_TOKENS && c->reduce != MOARA_MEAN_SEQUENCES) return moara_fail(MOARA_E_ARG, "bad reduce");
  if (tokens > 0 && c->kl_coef != 0 && !ref_logp) return moara_fail(MOARA_E_ARG, "a KL term needs ref_logp");
  p = PolicyParams{};
  const int rc = check_packed(p.q, mask, tokens, offsets, sequences);
  if (rc != MOARA_OK) return rc;
  if (tokens > 0 && (!logp || !advantages)) return moara_fail(MOARA_E_ARG, "null logp or advantages");
  if (misaligned(logp, 4) || misaligned(old_logp, 4) || misaligned(ref_logp, 4) || misaligned(advantages, 4))
    return moara_fail(MOARA_E_ARG, "pointer not aligned to its type");
  p.logp = logp;
  p.old = old_logp;
  p.ref = ref_logp;
  p.advantages = advantages;
  p.low = log1p(-c->clip_low);
  p.high = log1p(c->clip_high);
  p.at_low = (float)(1 - c->clip_low);
  p.at_high = (float)(1 + c->clip_high);
  p.kl_coef = c->kl_coef;
  p.entropy_coef = c->entropy_coef;
  p.divisor = c->divisor;
  p.kl = c->kl;
  p.by_sequence = c->reduce == MOARA_MEAN_SEQUENCES;
  p.sequence_advantages = c->sequence_advantages != 0;
  return MOARA_OK;
}

int check_balance(const moara_balance_config* c, BalanceParams& p, const void* logits, int64_t tokens, int64_t row_stride,
                  const uint8_t* mask, const int64_t* offsets, int64_t sequences) {
  if (!c) return moara_fail(MOARA_E_ARG, "null config");
  if (c->experts < 1 || c->top_k < 1) return moara_fail(MOARA_E_ARG, "top_k %d of %d experts", c->top_k, c->experts);
  if (c->score != MOARA_SOFTMAX && c->score != MOARA_SIGMOID) return moara_fail(MOARA_E_ARG, "bad score function");
  if (c->logits_dtype != MOARA_F32 && c->logits_dtype != MOARA_BF16) return moara_fail(MOARA_E_ARG, "bad logits dtype");
  if (!isfinite(c->balance_coef) || !isfinite(c->z_coef)) return moara_fail(MOARA_E_ARG, "a coefficient is not finite");
  if (c->experts > ROUTE_MAX_EXPERTS || c->top_k > ROUTE_MAX_K)
    return moara_fail(MOARA_E_UNSUPPORTED, "at most %d experts and top_k %d", ROUTE_MAX_EXPERTS, ROUTE_MAX_K);
  p = BalanceParams{};
  const int rc = check_packed(p.q, mask, tokens, offsets, sequences);
  if (rc != MOARA_OK) return rc;
  if (tokens > 0 && !logits) return moara_fail(MOARA_E_ARG, "null logits");
  if (row_stride < c->experts && tokens > 1) return moara_fail(MOARA_E_SHAPE, "rows overlap: stride %lld", (long long)row_stride);
  if (misaligned(logits, size_of(c->logits_dtype))) return moara_fail(MOARA_E_ARG, "logits not aligned to their type");
  p.logits = logits;
  p.ld = row_stride;
  p.E = c->experts;
  p.k = c->top_k;
  p.sigmoid = c->score == MOARA_SIGMOID;
  p.bf16 = c->logits_dtype == MOARA_BF16;
  p.want_z = c->z_coef != 0;
  p.balance_coef = c->balance_coef;
  p.z_coef = c->z_coef;
  return MOARA_OK;
}

}  // namespace

extern "C" {

int moara_token_logps(const void* logits, int32_t logits_dtype, int64_t tokens, int64_t vocab, int64_t row_stride,
                      int64_t inner, int64_t outer_stride, float scale, const int64_t* labels, float* out_logp,
                      float* out_entropy, float* out_stats, void* stream) {
  LogpsParams p;
  const int rc = check_logps(p, logits, logits_dtype, tokens, vocab, row_stride, inner, outer_stride, scale, labels);
  if (rc != MOARA_OK || tokens == 0) return rc;
  if (!out_logp || !out_stats) return moara_fail(MOARA_E_ARG, "null output");
  if (misaligned(out_logp, 4) || misaligned(out_entropy, 4) || misaligned(out_stats, 16))
    return moara_fail(MOARA_E_ARG, "output not aligned");
  p.logp = out_logp;
  p.entropy = out_entropy;
  p.stats = out_stats;
  LOSS_TRY(launch_logps(p, (hipStream_t)stream));
  return MOARA_OK;
}

int moara_token_logps_backward(const void* logits, int32_t logits_dtype, int64_t tokens, int64_t vocab, int64_t row_stride,
                               int64_t inner, int64_t outer_stride, float scale, const int64_t* labels, const float* stats,
                               const float* grad_logp, const float* entropy, const float* grad_entropy, void* out_grad,
                               int64_t grad_stride, void* stream) {
  LogpsParams p;
  const int rc = check_logps(p, logits, logits_dtype, tokens, vocab, row_stride, inner, outer_stride, scale, labels);
  if (rc != MOARA_OK || tokens == 0) return rc;
  if (!stats || !grad_logp || !out_grad) return moara_fail(MOARA_E_ARG, "null statistics, gradient or output");
  if (grad_entropy && !entropy) return moara_fail(MOARA_E_ARG, "the entropies' gradient needs the entropies");
  if ((grad_stride < vocab && tokens > 1) || grad_stride > MAX_STRIDE) return moara_fail(MOARA_E_SHAPE, "rows overlap: stride %lld", (long long)grad_stride);
  if (misaligned(stats, 16) || misaligned(grad_logp, 4) || misaligned(entropy, 4) || misaligned(grad_entropy, 4) ||
      misaligned(out_grad, size_of(logits_dtype)))
    return moara_fail(MOARA_E_ARG, "pointer not aligned");
  p.stats = const_cast<float*>(stats);
  p.logp = const_cast<float*>(grad_logp);
  p.entropy = const_cast<float*>(entropy);
  p.grad_entropy = grad_entropy;
  p.grad = out_grad;
  p.grad_ld = grad_stride;
  LOSS_TRY(launch_logps_backward(p, (hipStream_t)stream));
  return MOARA_OK;
}

int moara_preference_default_config(moara_preference_config* out) {
  if (!out) return moara_fail(MOARA_E_ARG, "null config");
  *out = moara_preference_config{0.1, 0, 0, MOARA_PREF_SIGMOID, 0};
  return MOARA_OK;
}

int moara_preference_loss(const moara_preference_config* cfg, const float* logp, const float* ref_logp, const uint8_t* mask,
                          int64_t tokens, const int64_t* offsets, int64_t sequences, float* out, float* out_loss,
                          float* out_rewards, float* out_slope, void* workspace, void* stream) {
  if (!cfg) return moara_fail(MOARA_E_ARG, "null config");
  if (!(cfg->beta > 0) || !isfinite(cfg->beta)) return moara_fail(MOARA_E_ARG, "beta must be positive");
  if (cfg->kind < MOARA_PREF_SIGMOID || cfg->kind > MOARA_PREF_SQUARE) return moara_fail(MOARA_E_ARG, "bad kind");
  if (!isfinite(cfg->margin) || (cfg->margin != 0 && cfg->kind == MOARA_PREF_SQUARE))
    return moara_fail(MOARA_E_ARG, "a margin that is not finite, or of the square");
  if (!(cfg->smoothing >= 0 && cfg->smoothing <= 1) || (cfg->smoothing != 0 && cfg->kind != MOARA_PREF_SIGMOID))
    return moara_fail(MOARA_E_ARG, "smoothing %g of kind %d", cfg->smoothing, cfg->kind);
  PreferenceParams p{};
  int rc = check_packed(p.q, mask, tokens, offsets, sequences);
  if (rc == MOARA_OK) rc = check_preference(p.q);
  if (rc != MOARA_OK) return rc;
  if (tokens > 0 && !logp) return moara_fail(MOARA_E_ARG, "null logp");
  if (!out || !out_rewards || !out_slope || (!workspace && MOARA_LOSS_WORKSPACE(tokens, sequences) > 0))
    return moara_fail(MOARA_E_ARG, "null output or workspace");
  if (misaligned(logp, 4) || misaligned(ref_logp, 4) || misaligned(out, 4) || misaligned(out_loss, 4) || misaligned(out_rewards, 4) ||
      misaligned(out_slope, 4) || misaligned(workspace, 8))
    return moara_fail(MOARA_E_ARG, "pointer not aligned");
  p.logp = logp;
  p.ref = ref_logp;
  p.beta = cfg->beta;
  p.margin = cfg->margin;
  p.smoothing = cfg->smoothing;
  p.kind = cfg->kind;
  p.average = cfg->average != 0;
  p.out = out;
  p.loss = out_loss;
  p.rewards = out_rewards;
  p.slope = out_slope;
  p.sums = (double*)workspace;
  LOSS_TRY(launch_preference(p, (hipStream_t)stream));
  return MOARA_OK;
}

int moara_preference_loss_backward(const float* slope, const float* grad_loss, const uint8_t* mask, int64_t tokens,
                                   const int64_t* offsets, int64_t sequences, float* out_grad, void* stream) {
  Packed q;
  int rc = check_packed(q, mask, tokens, offsets, sequences);
  if (rc == MOARA_OK) rc = check_preference(q);
  if (rc != MOARA_OK || tokens == 0) return rc;
  if (!slope || !grad_loss || !out_grad || misaligned(slope, 4) || misaligned(grad_loss, 4) || misaligned(out_grad, 4))
    return moara_fail(MOARA_E_ARG, "null or misaligned slope, gradient or output");
  LOSS_TRY(launch_preference_backward(q, slope, grad_loss, out_grad, (hipStream_t)stream));
  return MOARA_OK;
}

int moara_policy_default_config(moara_policy_config* out) {
  if (!out) return moara_fail(MOARA_E_ARG, "null config");
  *out = moara_policy_config{0.2, 0.2, 0, 0, 0, MOARA_KL_EXP, MOARA_MEAN_TOKENS, 0, 0};
  return MOARA_OK;
}

int moara_policy_loss(const moara_policy_config* cfg, const float* logp, const float* old_logp, const float* ref_logp,
                      const float* entropy, const float* advantages, const uint8_t* mask, int64_t tokens,
                      const int64_t* offsets, int64_t sequences, float* out, float* out_loss, float* out_weight,
                      void* workspace, void* stream) {
  PolicyParams p;
  const int rc = check_policy(cfg, p, logp, old_logp, ref_logp, advantages, mask, tokens, offsets, sequences);
  if (rc != MOARA_OK) return rc;
  if (tokens > 0 && cfg->entropy_coef != 0 && !entropy) return moara_fail(MOARA_E_ARG, "an entropy term needs entropy");
  if (!out || !out_weight || (!workspace && MOARA_LOSS_WORKSPACE(tokens, sequences) > 0))
    return moara_fail(MOARA_E_ARG, "null output or workspace");
  if (misaligned(entropy, 4) || misaligned(out, 4) || misaligned(out_loss, 4) || misaligned(out_weight, 4) || misaligned(workspace, 8))
    return moara_fail(MOARA_E_ARG, "pointer not aligned");
  p.entropy = entropy;
  p.out = out;
  p.loss = out_loss;
  p.weight = out_weight;
  p.sums = (double*)workspace;
  LOSS_TRY(launch_policy(p, (hipStream_t)stream));
  return MOARA_OK;
}

int moara_policy_loss_backward(const moara_policy_config* cfg, const float* logp, const float* old_logp, const float* ref_logp,
                               const float* advantages, const uint8_t* mask, int64_t tokens, const int64_t* offsets,
                               int64_t sequences, const float* weight, const float* grad_loss, float* out_grad_logp,
                               float* out_grad_entropy, void* stream) {
  PolicyParams p;
  const int rc = check_policy(cfg, p, logp, old_logp, ref_logp, advantages, mask, tokens, offsets, sequences);
  if (rc != MOARA_OK || tokens == 0) return rc;
  if (!weight || !grad_loss || !out_grad_logp) return moara_fail(MOARA_E_ARG, "null weight, gradient or output");
  if (misaligned(weight, 4) || misaligned(grad_loss, 4) || misaligned(out_grad_logp, 4) || misaligned(out_grad_entropy, 4))
    return moara_fail(MOARA_E_ARG, "pointer not aligned to its type");
  p.weight = const_cast<float*>(weight);
  p.grad_loss = grad_loss;
  p.grad_logp = out_grad_logp;
  p.grad_entropy = out_grad_entropy;
  LOSS_TRY(launch_policy_backward(p, (hipStream_t)stream));
  return MOARA_OK;
}

int moara_balance_default_config(moara_balance_config* out) {
  if (!out) return moara_fail(MOARA_E_ARG, "null config");
  *out = moara_balance_config{64, 6, MOARA_SOFTMAX, MOARA_F32, 0.01, 0};
  return MOARA_OK;
}

int moara_balance_loss(const moara_balance_config* cfg, const void* logits, int64_t tokens, int64_t row_stride,
                       const int32_t* index, const uint8_t* mask, const int64_t* offsets, int64_t sequences,
                       const int64_t* load, float* out, float* out_loss, int64_t* out_counts, float* out_slope, void* workspace,
                       void* stream) {
  BalanceParams p;
  const int rc = check_balance(cfg, p, logits, tokens, row_stride, mask, offsets, sequences);
  if (rc != MOARA_OK) return rc;
  if (tokens > 0 && !index) return moara_fail(MOARA_E_ARG, "null index");
  if (!out || !out_counts || !out_slope || !workspace) return moara_fail(MOARA_E_ARG, "null output or workspace");
  if (misaligned(index, 4) || misaligned(load, 8) || misaligned(out, 4) || misaligned(out_loss, 4) || misaligned(out_counts, 8) ||
      misaligned(out_slope, 4) || misaligned(workspace, 8))
    return moara_fail(MOARA_E_ARG, "pointer not aligned");
  p.index = index;
  p.load = load;
  p.out = out;
  p.loss = out_loss;
  p.counts = (long long*)out_counts;
  p.slope = out_slope;
  p.workspace = workspace;
  LOSS_TRY(launch_balance(p, (hipStream_t)stream));
  return MOARA_OK;
}

int moara_balance_loss_backward(const moara_balance_config* cfg, const void* logits, int64_t tokens, int64_t row_stride,
                                const uint8_t* mask, const int64_t* offsets, int64_t sequences, const float* slope,
                                const float* grad_loss, void* out_grad, void* stream) {
  BalanceParams p;
  const int rc = check_balance(cfg, p, logits, tokens, row_stride, mask, offsets, sequences);
  if (rc != MOARA_OK || tokens == 0) return rc;
  if (!slope || !grad_loss || !out_grad) return moara_fail(MOARA_E_ARG, "null slope, gradient or output");
  if (misaligned(slope, 4) || misaligned(grad_loss, 4) || misaligned(out_grad, size_of(cfg->logits_dtype)))
    return moara_fail(MOARA_E_ARG, "pointer not aligned to its type");
  p.slope = const_cast<float*>(slope);
  p.grad_loss = grad_loss;
  p.grad = out_grad;
  LOSS_TRY(launch_balance_backward(p, (hipStream_t)stream));
  return MOARA_OK;
}

}  // extern "C"
