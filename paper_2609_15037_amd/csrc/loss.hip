// Losses over packed sequences of tokens' log-probabilities: pairs of responses, and a clipped policy. Both sum
// over a sequence's tokens, so their forward pass is two steps: a wave sums a cell (tokens of one sequence within
// one tile) in 64 bits, then one workgroup adds up each sequence's cells, in order, and forms the loss.
#include "packed.h"

namespace {

constexpr int END_THREADS = 1024;

// e^q - q - 1. The three cancel near 0: there its series, q^2 (1/2 + q/6 + ..), to 1e-9 of its value at |q| = 1/2.
__device__ __forceinline__ float exp_excess(float q) {
  if (fabsf(q) < 0.5f) {
    float s = 1.f / 3628800.f;
    s = fmaf(s, q, 1.f / 362880.f);
    s = fmaf(s, q, 1.f / 40320.f);
    s = fmaf(s, q, 1.f / 5040.f);
    s = fmaf(s, q, 1.f / 720.f);
    s = fmaf(s, q, 1.f / 120.f);
    s = fmaf(s, q, 1.f / 24.f);
    s = fmaf(s, q, 1.f / 6.f);
    s = fmaf(s, q, 0.5f);
    return s * q * q;
  }
  return expf(q) - 1.f - q;
}

// Lanes of a sequence in the second step: as many as there are for each.
__device__ __forceinline__ int lanes_of_each(int64_t groups) {
  int lanes = 64;
  while (lanes > 1 && groups * lanes > END_THREADS) lanes >>= 1;
  return lanes;
}
// Sum over `lanes` neighbouring lanes.
__device__ __forceinline__ double over_lanes(double x, int lanes) {
  for (int o = lanes >> 1; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}

// ---------------------------------------------------------------- pairs of responses
__device__ __forceinline__ void preference_cell(const PreferenceParams& p, int64_t i) {
  const Cell c = cell_at(p.q, i, LOSS_CELL);
  double sum = 0, n = 0;
#pragma unroll 4
  for (int64_t t = c.begin + (threadIdx.x & 63); t < c.end; t += 64) {
    const bool on = !p.q.mask || p.q.mask[t];
    const double d = (double)p.logp[t] - (p.ref ? (double)p.ref[t] : 0.0);
    sum += on ? d : 0.0;
    n += on ? 1.0 : 0.0;
  }
  sum = wave_sum_d(sum);
  n = wave_sum_d(n);
  if ((threadIdx.x & 63) == 0) {
    p.sums[2 * i] = sum;
    p.sums[2 * i + 1] = n;
  }
}

__device__ __forceinline__ double log1p_exp(double z) { return fmax(z, 0.0) + log1p(exp(-fabs(z))); }

__device__ __forceinline__ void preference_end(const PreferenceParams& p) {
  __shared__ double part[END_THREADS / 64];
  const int64_t pairs = p.q.sequences / 2;
  const int lanes = lanes_of_each(pairs), lane = threadIdx.x & (lanes - 1);
  double loss = 0, ahead = 0, margin = 0, live = 0;
  for (int64_t pair = threadIdx.x / lanes; pair < pairs; pair += END_THREADS / lanes) {
    double d[2], n[2];
    for (int k = 0; k < 2; ++k) {
      int64_t first, last;
      cells_of(p.q, 2 * pair + k, LOSS_CELL, first, last);
      double s = 0, m = 0;
      for (int64_t i = first + lane; i < last; i += lanes) {
        s += p.sums[2 * i];
        m += p.sums[2 * i + 1];
      }
      d[k] = over_lanes(s, lanes);
      n[k] = over_lanes(m, lanes);
    }
    if (lane) continue;
    const double per0 = p.average && n[0] > 0 ? 1 / n[0] : 1, per1 = p.average && n[1] > 0 ? 1 / n[1] : 1;
    d[0] *= per0;
    d[1] *= per1;
    const double h = d[0] - d[1], z = p.beta * h - p.margin;
    double l, dl;               // the loss and its derivative by h
    if (p.kind == 0) {
      l = (1 - p.smoothing) * log1p_exp(-z) + p.smoothing * log1p_exp(z);
      dl = p.beta * (p.smoothing - 1 / (1 + exp(z)));
    } else if (p.kind == 1) {
      l = z < 1 ? 1 - z : z != z ? z : 0;
      dl = z < 1 ? -p.beta : 0;
    } else {
      l = (h - 0.5 / p.beta) * (h - 0.5 / p.beta);
      dl = 2 * (h - 0.5 / p.beta);
    }
    p.rewards[2 * pair] = (float)(p.beta * d[0]);
    p.rewards[2 * pair + 1] = (float)(p.beta * d[1]);
    const bool on = n[0] + n[1] > 0;
    p.slope[2 * pair] = on ? (float)(dl * per0) : 0.f;
    p.slope[2 * pair + 1] = on ? (float)(-dl * per1) : 0.f;
    if (on) {
      loss += l;
      ahead += h > 0 ? 1 : 0;
      margin += p.beta * h;
      live += 1;
    }
  }
  loss = group_sum<END_THREADS>(loss, part);
  ahead = group_sum<END_THREADS>(ahead, part);
  margin = group_sum<END_THREADS>(margin, part);
  live = group_sum<END_THREADS>(live, part);
  const double share = live > 0 ? 1 / live : 0;
  for (int64_t pair = threadIdx.x / lanes; pair < pairs; pair += END_THREADS / lanes) {
    if (lane) continue;         // the thread that wrote them
    p.slope[2 * pair] = (float)(p.slope[2 * pair] * share);
    p.slope[2 * pair + 1] = (float)(p.slope[2 * pair + 1] * share);
  }
  if (threadIdx.x == 0) {
    p.out[0] = (float)(loss * share);
    p.out[1] = (float)(ahead * share);
    p.out[2] = (float)(margin * share);
  }
}

__global__ __launch_bounds__(256) void k_preference_cells(PreferenceParams p, int64_t cells) {
  const int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (i < cells) preference_cell(p, i);
}
__global__ __launch_bounds__(END_THREADS) void k_preference_end(PreferenceParams p) { preference_end(p); }

// A token's gradient is its sequence's slope: written once, nothing but the mask is read for it.
__global__ __launch_bounds__(256) void k_preference_backward(Packed q, const float* __restrict__ slope,
                                                             const float* __restrict__ grad_loss, float* __restrict__ grad,
                                                             int64_t cells) {
  const int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (i >= cells) return;
  const int lane = threadIdx.x & 63;
  const Cell c = cell_at(q, i, LOSS_CELL);
  const float g = c.seq >= 0 ? slope[c.seq] * *grad_loss : 0.f;
  for (int64_t t = c.begin + lane; t < c.end; t += 64) grad[t] = !q.mask || q.mask[t] ? g : 0.f;
  for (int64_t t = c.fill0 + lane; t < c.fill1; t += 64) grad[t] = 0.f;
  for (int64_t t = c.fill2 + lane; t < c.fill3; t += 64) grad[t] = 0.f;
}

// ---------------------------------------------------------------- clipped policy
// A token's terms. d and the comparison with the bounds are 64 bits: a ratio next to a bound falls on the side
// that the difference of the two fp32 log-probabilities says.
struct Token { float gain, slope, kl, dkl, excess; bool clipped; };
__device__ __forceinline__ Token policy_token(const PolicyParams& p, float logp, float old, float ref, float a) {
  Token t;
  const double d = p.old ? (double)logp - (double)old : 0.0;
  const float ratio = expf((float)d);
  const bool up = d > p.high && a > 0, down = d < p.low && a < 0;
  t.clipped = up || down;
  t.gain = (up ? p.at_high : down ? p.at_low : ratio) * a;
  t.slope = t.clipped ? 0.f : -ratio * a;
  t.excess = p.old ? exp_excess((float)d) : 0.f;
  t.kl = t.dkl = 0.f;
  if (p.ref) {
    const float q = (float)((double)ref - (double)logp);
    t.kl = p.kl == 0 ? exp_excess(q) : p.kl == 1 ? -q : 0.5f * q * q;
    t.dkl = p.kl == 0 ? -expm1f(q) : p.kl == 1 ? 1.f : -q;
  }
  return t;
}

__device__ __forceinline__ void policy_cell(const PolicyParams& p, int64_t i) {
  const Cell c = cell_at(p.q, i, LOSS_CELL);
  double sum[POLICY_SUMS] = {};
  const float each = p.sequence_advantages && c.seq >= 0 ? p.advantages[c.seq] : 0.f;
#pragma unroll 2
  for (int64_t t = c.begin + (threadIdx.x & 63); t < c.end; t += 64) {
    const bool on = !p.q.mask || p.q.mask[t];
    const Token x = policy_token(p, p.logp[t], p.old ? p.old[t] : 0.f, p.ref ? p.ref[t] : 0.f,
                                 p.sequence_advantages ? each : p.advantages[t]);
    const float entropy = p.entropy ? p.entropy[t] : 0.f;
    if (on) {
      sum[0] += 1;
      sum[1] -= (double)x.gain;
      sum[2] += (double)x.kl;
      sum[3] += (double)entropy;
      sum[4] += x.clipped ? 1 : 0;
      sum[5] += (double)x.excess;
    }
  }
#pragma unroll
  for (int k = 0; k < POLICY_SUMS; ++k) {
    const double s = wave_sum_d(sum[k]);
    if ((threadIdx.x & 63) == 0) p.sums[POLICY_SUMS * i + k] = s;
  }
}

__device__ __forceinline__ void policy_end(const PolicyParams& p) {
  __shared__ double part[END_THREADS / 64];
  const int64_t S = p.q.sequences;
  const int lanes = lanes_of_each(S), lane = threadIdx.x & (lanes - 1);
  double sum[POLICY_SUMS] = {}, live = 0;
  for (int64_t s = threadIdx.x / lanes; s < S; s += END_THREADS / lanes) {
    int64_t first, last;
    cells_of(p.q, s, LOSS_CELL, first, last);
    double own[POLICY_SUMS] = {};
    for (int64_t i = first + lane; i < last; i += lanes)
#pragma unroll
      for (int k = 0; k < POLICY_SUMS; ++k) own[k] += p.sums[POLICY_SUMS * i + k];
#pragma unroll
    for (int k = 0; k < POLICY_SUMS; ++k) own[k] = over_lanes(own[k], lanes);
    if (lane) continue;
    const double per = !p.by_sequence ? 1 : own[0] > 0 ? 1 / own[0] : 0;
    live += own[0] > 0 ? 1 : 0;
    sum[0] += own[0];
#pragma unroll
    for (int k = 1; k < POLICY_SUMS; ++k) sum[k] += own[k] * per;
    p.weight[s] = own[0] > 0 ? (float)per : 0.f;
  }
  live = group_sum<END_THREADS>(live, part);
#pragma unroll
  for (int k = 0; k < POLICY_SUMS; ++k) sum[k] = group_sum<END_THREADS>(sum[k], part);
  const double over = p.divisor > 0 ? p.divisor : p.by_sequence ? live : sum[0], share = over > 0 ? 1 / over : 0;
  for (int64_t s = threadIdx.x / lanes; s < S; s += END_THREADS / lanes)
    if (!lane) p.weight[s] = (float)(p.weight[s] * share);      // the thread that wrote it
  if (threadIdx.x == 0) {
    const double policy = sum[1] * share, kl = sum[2] * share, entropy = sum[3] * share;
    p.out[0] = (float)(policy + (p.ref ? p.kl_coef * kl : 0) - (p.entropy ? p.entropy_coef * entropy : 0));
    p.out[1] = (float)policy;
    p.out[2] = (float)kl;
    p.out[3] = (float)entropy;
    p.out[4] = (float)(sum[4] * share);
    p.out[5] = (float)(sum[5] * share);
  }
}

__global__ __launch_bounds__(256) void k_policy_cells(PolicyParams p, int64_t cells) {
  const int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (i < cells) policy_cell(p, i);
}
__global__ __launch_bounds__(END_THREADS) void k_policy_end(PolicyParams p) { policy_end(p); }

__global__ __launch_bounds__(256) void k_policy_backward(PolicyParams p, int64_t cells) {
  const int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (i >= cells) return;
  const int lane = threadIdx.x & 63;
  const Cell c = cell_at(p.q, i, LOSS_CELL);
  const float each = p.sequence_advantages && c.seq >= 0 ? p.advantages[c.seq] : 0.f;
  const float w = c.seq >= 0 ? p.weight[c.seq] * *p.grad_loss : 0.f;
  const float kl_coef = (float)p.kl_coef, bonus = -(float)p.entropy_coef * w;
#pragma unroll 2
  for (int64_t t = c.begin + lane; t < c.end; t += 64) {
    const bool on = !p.q.mask || p.q.mask[t];
    const Token x = policy_token(p, p.logp[t], p.old ? p.old[t] : 0.f, p.ref ? p.ref[t] : 0.f,
                                 p.sequence_advantages ? each : p.advantages[t]);
    p.grad_logp[t] = on ? (x.slope + (p.ref ? kl_coef * x.dkl : 0.f)) * w : 0.f;
    if (p.grad_entropy) p.grad_entropy[t] = on ? bonus : 0.f;
  }
  auto clear = [&](int64_t from, int64_t to) {
    for (int64_t t = from + lane; t < to; t += 64) {
      p.grad_logp[t] = 0.f;
      if (p.grad_entropy) p.grad_entropy[t] = 0.f;
    }
  };
  clear(c.fill0, c.fill1);
  clear(c.fill2, c.fill3);
}

}  // namespace

#define ON_CELLS(kernel, q, st, ...)                                                                                   \
  do {                                                                                                                 \
    const int64_t cells = cells_of_all(q, LOSS_CELL);                                                                  \
    if (cells > 0) hipLaunchKernelGGL(kernel, dim3((uint32_t)((cells + 3) / 4)), dim3(256), 0, st, __VA_ARGS__, cells); \
  } while (0)

hipError_t launch_preference(const PreferenceParams& p, hipStream_t st) {
  ON_CELLS(k_preference_cells, p.q, st, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_preference_end, dim3(1), dim3(END_THREADS), 0, st, p);
  return hipGetLastError();
}
hipError_t launch_preference_backward(const Packed& q, const float* slope, const float* grad_loss, float* grad, hipStream_t st) {
  ON_CELLS(k_preference_backward, q, st, q, slope, grad_loss, grad);
  return hipGetLastError();
}
hipError_t launch_policy(const PolicyParams& p, hipStream_t st) {
  ON_CELLS(k_policy_cells, p.q, st, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_policy_end, dim3(1), dim3(END_THREADS), 0, st, p);
  return hipGetLastError();
}
hipError_t launch_policy_backward(const PolicyParams& p, hipStream_t st) {
  ON_CELLS(k_policy_backward, p.q, st, p);
  return hipGetLastError();
}
