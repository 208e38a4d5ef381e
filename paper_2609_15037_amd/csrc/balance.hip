// Load-balancing loss of expert routing, its counts and its gradient. Forward: a workgroup sums the scores and counts
// the experts of a cell's tokens, a second launch adds up each sequence's cells and forms its loss, and where there
// are several sequences a third one their mean. Backward: the scores again, and a row of the gradient for each token.
#include <float.h>

#include "lanes.h"
#include "packed.h"

namespace {

constexpr int THREADS = 256, END_THREADS = 1024;

// What a cell leaves in the workspace, experts padded to an even number: its scores' sums, its counts, z and its tokens.
struct CellSums {
  char* at;
  int E;
  __device__ __forceinline__ int64_t size() const { return 8 * (int64_t)((E + 1) & ~1) + 16; }
  __device__ __forceinline__ double* about(int64_t i) const { return (double*)(at + i * size()); }       // z, tokens
  __device__ __forceinline__ float* scores(int64_t i) const { return (float*)(about(i) + 2); }
  __device__ __forceinline__ uint32_t* counts(int64_t i) const { return (uint32_t*)(scores(i) + ((E + 1) & ~1)); }
};
// What a sequence leaves: its balance, whether it has tokens, z, its tokens.
__device__ __forceinline__ double* about_sequences(const BalanceParams& p, int64_t cells) {
  return (double*)((char*)p.workspace + cells * CellSums{nullptr, p.E}.size());
}

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896340736f); }

// A token's scores (of a sigmoid over their sum, which exists where they underflow) and, for the gradient, 1 - sigmoid;
// with z the softmax and the logits' log-sum-exp. False where it has no scores.
template <int LANES, int V, bool BACKWARD>
__device__ __forceinline__ bool token_scores(const float (&l)[V], int sigmoid, int want_z, float (&s)[V], float (&rest)[V],
                                             float (&soft)[V], float& lse) {
  float top = l[0], sum = 0;
#pragma unroll
  for (int j = 1; j < V; ++j) top = fmaxf(top, l[j]);
  top = max_of<LANES>(top);
  lse = 0;
  if (sigmoid) {
    const float shift = fminf(top, 0.f);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float q = exp_of(-fabsf(l[j])), r = 1.f / (1.f + q);
      s[j] = exp_of(fminf(l[j], 0.f) - shift) * r;
      if (BACKWARD) rest[j] = l[j] > 0 ? q * r : r;
      sum += s[j];
    }
    sum = sum_of<LANES>(sum);
    const bool there = sum > 0;         // not NaN, not a row of -infinity
    const float y = 1.f / sum;
#pragma unroll
    for (int j = 0; j < V; ++j) s[j] *= y;
    if (want_z) {
      float total = 0;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        soft[j] = exp_of(l[j] - top);
        total += soft[j];
      }
      total = sum_of<LANES>(total);
      lse = top + logf(total);
      if (BACKWARD) {
        const float w = 1.f / total;
#pragma unroll
        for (int j = 0; j < V; ++j) soft[j] *= w;
      }
    }
    return there;
  }
#pragma unroll
  for (int j = 0; j < V; ++j) {
    s[j] = exp_of(l[j] - top);
    sum += s[j];
  }
  sum = sum_of<LANES>(sum);
  const bool there = sum > 0;           // not NaN: a row of -infinity, one with a NaN or +infinity
  const float y = 1.f / sum;
#pragma unroll
  for (int j = 0; j < V; ++j) s[j] *= y;
  if (want_z) lse = top + logf(sum);
  return there;
}

template <int LANES, int V> __device__ __forceinline__ void fetch(const BalanceParams& p, int64_t t, int lane, float (&l)[V]) {
#pragma unroll
  for (int j = 0; j < V; j += 4) {
    const int e = expert_of<LANES>(j, lane);
    load4(p.logits, p.bf16, t * p.ld + e, p.E - e, l + j);
  }
}

template <int LANES, int V> __global__ __launch_bounds__(THREADS) void k_balance(BalanceParams p, int tile) {
  constexpr int TOK = THREADS / LANES;
  __shared__ float red[TOK * LANES * V];
  __shared__ uint32_t hist[LANES * V];
  __shared__ double part[THREADS / 64];
  const int lane = threadIdx.x % LANES, slot = threadIdx.x / LANES;
  const int64_t i = blockIdx.x;
  const Cell c = cell_at(p.q, i, tile);
  for (int e = threadIdx.x; e < LANES * V; e += THREADS) hist[e] = 0;
  __syncthreads();
  float sum[V] = {};
  double z = 0, n = 0;
  for (int64_t t0 = c.begin; t0 < c.end; t0 += TOK) {
    const int64_t t = t0 + slot;
    const bool in = t < c.end;
    float l[V], s[V], rest[V], soft[V], lse;
    fetch<LANES, V>(p, in ? t : t0, lane, l);
    const bool there = token_scores<LANES, V, false>(l, p.sigmoid, p.want_z, s, rest, soft, lse);
    const bool on = in && there && !(p.q.mask && !p.q.mask[t]);
    if (!on) continue;
#pragma unroll
    for (int j = 0; j < V; ++j) sum[j] += s[j];
    if (lane == 0) {
      n += 1;
      z += (double)lse * (double)lse;
    }
    for (int j = lane; j < p.k; j += LANES) {
      const int e = p.index[t * p.k + j];
      if (e >= 0 && e < p.E) atomicAdd(&hist[e], 1u);
    }
  }
#pragma unroll
  for (int j = 0; j < V; ++j) red[slot * (LANES * V) + expert_of<LANES>(j, lane)] = sum[j];
  z = group_sum<THREADS>(z, part);
  n = group_sum<THREADS>(n, part);
  __syncthreads();
  const CellSums w = {(char*)p.workspace, p.E};
  for (int e = threadIdx.x; e < p.E; e += THREADS) {
    float x = 0;
#pragma unroll 4
    for (int k = 0; k < TOK; ++k) x += red[k * (LANES * V) + e];
    w.scores(i)[e] = x;
    w.counts(i)[e] = hist[e];
  }
  if (threadIdx.x == 0) {
    w.about(i)[0] = z;
    w.about(i)[1] = n;
  }
}

// out and the factors of the gradient, from the sums over the sequences.
__device__ __forceinline__ void balance_out(const BalanceParams& p, double balance, double live, double z, double n) {
  const double each = live > 0 ? 1 / live : 0, per = n > 0 ? 1 / n : 0;
  p.out[0] = (float)(p.balance_coef * balance * each + p.z_coef * z * per);
  p.out[1] = (float)(balance * each);
  p.out[2] = (float)(z * per);
  float* tail = p.slope + p.q.sequences * p.E;
  tail[0] = (float)(p.balance_coef * each);
  tail[1] = (float)(2 * p.z_coef * per);
}

// One workgroup for each sequence: threads take an expert and every so many-th cell.
__global__ __launch_bounds__(END_THREADS) void k_balance_end(BalanceParams p, int tile, int64_t cells) {
  __shared__ double score[END_THREADS];
  __shared__ long long count[END_THREADS];
  __shared__ double part[END_THREADS / 64];
  const int64_t s = blockIdx.x;
  const CellSums w = {(char*)p.workspace, p.E};
  int64_t first, last;
  cells_of(p.q, s, tile, first, last);
  int width = 64;
  while (width < p.E) width *= 2;
  const int e = threadIdx.x & (width - 1), row = threadIdx.x / width, rows = END_THREADS / width;
  double x = 0;
  long long c = 0;
  if (e < p.E) {
#pragma unroll 4
    for (int64_t i = first + row; i < last; i += rows) {
      x += (double)w.scores(i)[e];
      c += w.counts(i)[e];
    }
  }
  double z = 0, n = 0;
  for (int64_t i = first + threadIdx.x; i < last; i += END_THREADS) {
    z += w.about(i)[0];
    n += w.about(i)[1];
  }
  z = group_sum<END_THREADS>(z, part);
  n = group_sum<END_THREADS>(n, part);
  score[threadIdx.x] = x;
  count[threadIdx.x] = c;
  __syncthreads();
  const bool mine = row == 0 && e < p.E;
  x = 0;
  c = 0;
  if (mine) {
    for (int k = 0; k < rows; ++k) {
      x += score[k * width + e];
      c += count[k * width + e];
    }
    p.counts[s * p.E + e] = c;
    if (p.load) c = p.load[e];
  }
  const double total = group_sum<END_THREADS>(mine ? (double)c : 0.0, part);
  // f less its mean, 1: scores sum to 1, so a constant has no gradient, and nothing cancels where the load is even
  const double f = total > 0 ? p.E * (double)c / total : 0, per = n > 0 ? 1 / n : 0;
  const double balance = group_sum<END_THREADS>(mine ? f * x * per : 0.0, part);
  if (mine) p.slope[s * p.E + e] = total > 0 ? (float)((f - 1) * per) : 0.f;
  if (threadIdx.x) return;
  if (p.q.sequences == 1) {
    balance_out(p, balance, n > 0 ? 1 : 0, z, n);
  } else {
    double* a = about_sequences(p, cells) + 4 * s;
    a[0] = balance;
    a[1] = n > 0 ? 1 : 0;
    a[2] = z;
    a[3] = n;
  }
}
__global__ __launch_bounds__(END_THREADS) void k_balance_out(BalanceParams p, int64_t cells) {
  __shared__ double part[END_THREADS / 64];
  const double* a = about_sequences(p, cells);
  double sum[4] = {};
  for (int64_t s = threadIdx.x; s < p.q.sequences; s += END_THREADS)
#pragma unroll
    for (int k = 0; k < 4; ++k) sum[k] += a[4 * s + k];
#pragma unroll
  for (int k = 0; k < 4; ++k) sum[k] = group_sum<END_THREADS>(sum[k], part);
  if (threadIdx.x == 0) balance_out(p, sum[0], sum[1], sum[2], sum[3]);
}

template <int LANES, int V> __global__ __launch_bounds__(THREADS) void k_balance_backward(BalanceParams p, int tile) {
  constexpr int TOK = THREADS / LANES;
  const int lane = threadIdx.x % LANES, slot = threadIdx.x / LANES;
  const Cell c = cell_at(p.q, blockIdx.x, tile);
  const float* tail = p.slope + p.q.sequences * p.E;
  const float g = *p.grad_loss, a = g * tail[0], b = g * tail[1];
  float f[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int e = expert_of<LANES>(j, lane);
    f[j] = c.seq >= 0 && e < p.E ? p.slope[c.seq * p.E + e] * a : 0.f;
  }
  for (int64_t t0 = c.begin; t0 < c.end; t0 += TOK) {
    const int64_t t = t0 + slot;
    const bool in = t < c.end;
    float l[V], s[V], rest[V], soft[V], lse;
    fetch<LANES, V>(p, in ? t : t0, lane, l);
    const bool there = token_scores<LANES, V, true>(l, p.sigmoid, p.want_z, s, rest, soft, lse);
    const bool on = in && there && !(p.q.mask && !p.q.mask[t]);
    float mean = 0;
#pragma unroll
    for (int j = 0; j < V; ++j) mean = fmaf(f[j], s[j], mean);
    mean = sum_of<LANES>(mean);
    if (!in) continue;
    float x[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      float d = s[j] * (f[j] - mean);
      if (p.sigmoid) d *= rest[j];
      if (p.want_z) d = fmaf(b * lse, p.sigmoid ? soft[j] : s[j], d);
      x[j] = on ? d : 0.f;
    }
#pragma unroll
    for (int j = 0; j < V; j += 4) {
      const int e = expert_of<LANES>(j, lane);
      store4(p.grad, p.bf16, t * p.E + e, p.E - e, x + j);
    }
  }
  auto clear = [&](int64_t from, int64_t to) {
    const float zero[4] = {};
    for (int64_t t = from + slot; t < to; t += TOK)
#pragma unroll
      for (int j = 0; j < V; j += 4) {
        const int e = expert_of<LANES>(j, lane);
        store4(p.grad, p.bf16, t * p.E + e, p.E - e, zero);
      }
  };
  clear(c.fill0, c.fill1);
  clear(c.fill2, c.fill3);
}

// Tokens of a tile: enough for 256 workgroups, a multiple of what one takes at a time.
int tile_of(const BalanceParams& p) {
  int64_t tile = BALANCE_LEAST_TILE;
  while (tile * 256 < p.q.tokens && tile < 1 << 20) tile *= 2;
  return (int)tile;
}

}  // namespace

#define BALANCE_ON(kernel, ...)                                                                                       \
  do {                                                                                                                \
    const dim3 g((uint32_t)cells), b(THREADS);                                                                        \
    if (p.E <= 32) hipLaunchKernelGGL((kernel<8, 4>), g, b, 0, st, __VA_ARGS__);                                      \
    else if (p.E <= 64) hipLaunchKernelGGL((kernel<16, 4>), g, b, 0, st, __VA_ARGS__);                                \
    else if (p.E <= 128) hipLaunchKernelGGL((kernel<16, 8>), g, b, 0, st, __VA_ARGS__);                               \
    else if (p.E <= 256) hipLaunchKernelGGL((kernel<16, 16>), g, b, 0, st, __VA_ARGS__);                              \
    else if (p.E <= 512) hipLaunchKernelGGL((kernel<32, 16>), g, b, 0, st, __VA_ARGS__);                              \
    else hipLaunchKernelGGL((kernel<64, 16>), g, b, 0, st, __VA_ARGS__);                                              \
  } while (0)

hipError_t launch_balance(const BalanceParams& p, hipStream_t st) {
  const int tile = tile_of(p);
  const int64_t cells = cells_of_all(p.q, tile);
  if (cells > 0) BALANCE_ON(k_balance, p, tile);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_balance_end, dim3((uint32_t)p.q.sequences), dim3(END_THREADS), 0, st, p, tile, cells);
  e = hipGetLastError();
  if (e != hipSuccess || p.q.sequences == 1) return e;
  hipLaunchKernelGGL(k_balance_out, dim3(1), dim3(END_THREADS), 0, st, p, cells);
  return hipGetLastError();
}

hipError_t launch_balance_backward(const BalanceParams& p, hipStream_t st) {
  const int tile = tile_of(p);
  const int64_t cells = cells_of_all(p.q, tile);
  if (cells > 0) BALANCE_ON(k_balance_backward, p, tile);
  return hipGetLastError();
}
