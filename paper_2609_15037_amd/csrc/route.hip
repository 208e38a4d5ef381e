// Routing of tokens to experts: scores, selection (groups, top-k), weights, their gradient, and the step
// of the balancing bias.
#include <float.h>

#include "train.h"

namespace {

typedef uint16_t u16x4u __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));

// ---- reductions over the LANES (16 or 64) lanes of a token; every lane gets the result. Sixteen lanes are
// one row of the cross-lane data path: neighbours, neighbouring pairs, mirrored halves and rows.
template <int CTRL> __device__ __forceinline__ uint32_t dpp(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, false);
}
template <int CTRL> __device__ __forceinline__ float dpp(float x) {
  return __uint_as_float(dpp<CTRL>(__float_as_uint(x)));
}
template <int CTRL> __device__ __forceinline__ double dpp(double x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  return __builtin_bit_cast(double, (uint64_t)dpp<CTRL>((uint32_t)(b >> 32)) << 32 | dpp<CTRL>((uint32_t)b));
}
template <int LANES, typename T, typename F> __device__ __forceinline__ T reduce(T x, F f) {
  x = f(x, dpp<0xB1>(x));     // lane ^ 1
  x = f(x, dpp<0x4E>(x));     // lane ^ 2
  x = f(x, dpp<0x141>(x));    // mirrored within eight lanes
  x = f(x, dpp<0x140>(x));    // mirrored within sixteen
  if (LANES == 64) {
    x = f(x, (T)__shfl_xor(x, 16, 64));
    x = f(x, (T)__shfl_xor(x, 32, 64));
  }
  return x;
}
template <int LANES> __device__ __forceinline__ float sum_of(float x) {
  return reduce<LANES>(x, [](float a, float b) { return a + b; });
}
template <int LANES> __device__ __forceinline__ double sum_of(double x) {
  return reduce<LANES>(x, [](double a, double b) { return a + b; });
}
template <int LANES> __device__ __forceinline__ float max_of(float x) {
  return reduce<LANES>(x, [](float a, float b) { return fmaxf(a, b); });
}
template <int LANES> __device__ __forceinline__ uint32_t max_of(uint32_t x) {
  return reduce<LANES>(x, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
template <int LANES> __device__ __forceinline__ uint32_t min_of(uint32_t x) {
  return reduce<LANES>(x, [](uint32_t a, uint32_t b) { return a < b ? a : b; });
}

// Four lanes' worth of a row: experts e0 .. e0 + 3 of which those below E exist (the others read -inf).
__device__ __forceinline__ void load4(const float* q, int n, float* x) {
  if (n >= 4) {
    const f32x4u a = *reinterpret_cast<const f32x4u*>(q);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = a[j];
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = j < n ? q[j] : -__builtin_inff();
  }
}
__device__ __forceinline__ void load4(const bf16* q, int n, float* x) {
  if (n >= 4) {
    const u16x4u a = *reinterpret_cast<const u16x4u*>(q);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = __uint_as_float((uint32_t)a[j] << 16);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = j < n ? bf2f(q[j]) : -__builtin_inff();
  }
}
__device__ __forceinline__ void store4(float* q, int n, const float* x) {
  if (n >= 4) {
    *reinterpret_cast<f32x4u*>(q) = f32x4u{x[0], x[1], x[2], x[3]};
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) if (j < n) q[j] = x[j];
  }
}
__device__ __forceinline__ void store4(bf16* q, int n, const float* x) {
  if (n >= 4) {
    u16x4u a;
#pragma unroll
    for (int j = 0; j < 4; ++j) a[j] = __builtin_bit_cast(uint16_t, f2bf(x[j]));
    *reinterpret_cast<u16x4u*>(q) = a;
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) if (j < n) q[j] = f2bf(x[j]);
  }
}
template <typename T> __device__ __forceinline__ float to_f32(T x) { return (float)x; }

// Expert of a lane's value j: groups of four consecutive experts are dealt to the lanes in turn, so that
// a load of the row is contiguous; a lane's experts ascend with j.
template <int LANES> __device__ __forceinline__ int expert_of(int j, int lane) {
  return (j >> 2) * (4 * LANES) + lane * 4 + (j & 3);
}

// Floats as unsigned integers of the same order; 0 is left for what cannot be chosen (-inf, NaN, none).
__device__ __forceinline__ uint32_t order_key(float c) {
  if (!(c > -__builtin_inff())) return 0;
  const uint32_t b = __float_as_uint(c + 0.f);     // -0 counts as 0
  return (int)b < 0 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float((int)k < 0 ? k & 0x7FFFFFFFu : ~k);
}

// The score of a logit; top and total: the row's largest logit and its sum of exponentials (softmax). The
// sum is taken in 64 bits: an expert's score must not depend on the order of the others.
struct Row { float top, total; };
__device__ __forceinline__ float score(float l, const Row& r, int sigmoid) {
  return sigmoid ? 1.f / (1.f + expf(-l)) : expf(l - r.top) / r.total;
}
template <int LANES, int V> __device__ __forceinline__ Row softmax_row(const float (&l)[V]) {
  Row r;
  float top = l[0];
#pragma unroll
  for (int j = 1; j < V; ++j) top = fmaxf(top, l[j]);
  r.top = max_of<LANES>(top);
  double sum = 0;
#pragma unroll
  for (int j = 0; j < V; ++j) sum += (double)expf(l[j] - r.top);
  r.total = (float)sum_of<LANES>(sum);
  return r;
}

// u_j of the chosen experts, one a lane (lanes without one: there = false): the score itself, or its share
// of the chosen ones' sum, from the logits less their largest, so that shares exist where scores underflow
// (the sigmoid as exp(min(l, 0)) / (1 + exp(-|l|))). No share where every chosen logit is -inf.
template <int LANES> __device__ __forceinline__ float chosen_share(float l, bool there, const Row& r, const RouteParams& p) {
  if (!p.renorm) return there ? score(l, r, p.sigmoid) : 0.f;
  const float x = p.sigmoid ? fminf(l, 0.f) : l;
  const float top = max_of<LANES>(there ? x : -FLT_MAX);
  float u = there ? expf(x - fmaxf(top, -FLT_MAX)) : 0.f;
  if (p.sigmoid) u /= 1.f + expf(-fabsf(l));
  const float total = sum_of<LANES>(u);
  return total > 0.f ? u / total : 0.f;
}

// LANES lanes take one token, V experts each. A workgroup walks over its tokens and counts the experts'
// tokens in LDS; whole numbers, so the order of the atomic additions does not change them.
template <typename T, int LANES, int V, bool GROUPS>
__global__ __launch_bounds__(256) void k_route(RouteParams p) {
  constexpr int TOK = 256 / LANES;      // tokens of a workgroup at a time
  __shared__ uint32_t hist[LANES * V];
  __shared__ uint32_t rowkey[GROUPS ? TOK * LANES * V : 1];
  __shared__ uint32_t groupkey[GROUPS ? TOK * ROUTE_MAX_GROUPS : 1];
  const int lane = threadIdx.x % LANES, slot = threadIdx.x / LANES;
  if (p.counts)
    for (int e = threadIdx.x; e < LANES * V; e += 256) hist[e] = 0;
  __syncthreads();
  for (int64_t t0 = (int64_t)blockIdx.x * TOK; t0 < p.tokens; t0 += (int64_t)gridDim.x * TOK) {
    const int64_t t = t0 + slot;
    const bool live = t < p.tokens && !(p.mask && !p.mask[t]);
    const T* row = (const T*)p.logits + (t < p.tokens ? t : 0) * p.ld;
    float l[V];
#pragma unroll
    for (int j = 0; j < V; j += 4) load4(row + expert_of<LANES>(j, lane), p.E - expert_of<LANES>(j, lane), l + j);
    Row r = {0.f, 1.f};
    if (!p.sigmoid) r = softmax_row<LANES, V>(l);
    uint32_t key[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int e = expert_of<LANES>(j, lane);
      float c = score(l[j], r, p.sigmoid);
      if (p.bias && e < p.E) c += p.bias[e];
      key[j] = live && e < p.E ? order_key(c) : 0u;
    }
    if (GROUPS) {
      uint32_t* rk = rowkey + slot * (LANES * V);
      uint32_t* gk = groupkey + slot * ROUTE_MAX_GROUPS;
      __syncthreads();
#pragma unroll
      for (int j = 0; j < V; ++j) rk[expert_of<LANES>(j, lane)] = key[j];
      __syncthreads();
      for (int g = lane; g < p.groups; g += LANES) {
        uint32_t best = 0, next = 0;
        for (uint32_t q = 0; q < p.group_size; ++q) {
          const uint32_t k = rk[g * p.group_size + q];
          next = max(next, min(best, k));
          best = max(best, k);
        }
        // the sum of the two best (what cannot be chosen adds nothing), or the best
        gk[g] = p.group_best == 2 && next ? order_key(key_value(best) + key_value(next)) : best;
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int e = expert_of<LANES>(j, lane);
        if (e < p.E && key[j]) {
          const int g = (int)(((uint32_t)e * p.group_inv) >> 20);
          const uint32_t mine = gk[g];
          int rank = 0;
          for (int q = 0; q < p.groups; ++q) rank += gk[q] > mine || (gk[q] == mine && q < g);
          if (rank >= p.top_groups) key[j] = 0;
        }
      }
    }
    int chosen = -1;      // of lane i < k: the token's i-th expert
    for (int i = 0; i < p.k; ++i) {
      uint32_t best = 0, at = 0xFFFFFFFFu;
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (key[j] > best) { best = key[j]; at = (uint32_t)expert_of<LANES>(j, lane); }
      const uint32_t top = max_of<LANES>(best);
      at = min_of<LANES>(top && best == top ? at : 0xFFFFFFFFu);
#pragma unroll
      for (int j = 0; j < V; ++j)
        if ((uint32_t)expert_of<LANES>(j, lane) == at) key[j] = 0;
      if (lane == i) chosen = (int)at;
    }
    const bool there = chosen >= 0;
    const float u = chosen_share<LANES>(there ? to_f32(row[chosen]) : 0.f, there, r, p);
    if (lane < p.k && t < p.tokens) {
      p.index[t * p.k + lane] = chosen;
      p.weight[t * p.k + lane] = u * p.scale;
      if (p.counts && there) atomicAdd(&hist[chosen], 1u);
    }
  }
  if (!p.counts) return;
  __syncthreads();
  for (int e = threadIdx.x; e < p.E; e += 256)
    if (hist[e]) atomicAdd(&p.counts[e], (unsigned long long)hist[e]);
}

// Gradient of the weights -> gradient of the logits. With u_j the chosen experts' shares and s their scores:
// renormalised, t_j = u_j (dw_j - sum dw u) and d l_j = t_j, times 1 - s_j for the sigmoid (the softmax's own
// sum vanishes); else t_j = dw_j s_j, times 1 - s_j for the sigmoid, and d l_e = t_e - s_e sum t for the softmax,
// the only form that needs the whole row.
template <typename T, int LANES, int V>
__global__ __launch_bounds__(256) void k_route_backward(RouteParams p) {
  constexpr int TOK = 256 / LANES;
  __shared__ float out[TOK * LANES * V];
  const int lane = threadIdx.x % LANES, slot = threadIdx.x / LANES;
  const bool whole = !p.sigmoid && !p.renorm;
  for (int64_t t0 = (int64_t)blockIdx.x * TOK; t0 < p.tokens; t0 += (int64_t)gridDim.x * TOK) {
    const int64_t t = t0 + slot;
    const bool in = t < p.tokens;
    const T* row = (const T*)p.logits + (in ? t : 0) * p.ld;
    const int chosen = in && lane < p.k ? p.index[t * p.k + lane] : -1;
    const bool there = chosen >= 0 && chosen < p.E;
    const float dw = there ? p.weight[t * p.k + lane] : 0.f;
    const float lc = there ? to_f32(row[chosen]) : 0.f;
    float l[V];
    Row r = {0.f, 1.f};
    if (whole) {
#pragma unroll
      for (int j = 0; j < V; j += 4) load4(row + expert_of<LANES>(j, lane), p.E - expert_of<LANES>(j, lane), l + j);
      r = softmax_row<LANES, V>(l);
    }
    const float u = chosen_share<LANES>(lc, there, r, p);
    const float mean = p.renorm ? sum_of<LANES>(dw * u) : 0.f;
    float d = there ? p.scale * u * (dw - mean) : 0.f;
    if (p.sigmoid) d *= 1.f / (1.f + expf(lc));
    const float total = whole ? sum_of<LANES>(d) : 0.f;
    const bool any = max_of<LANES>((uint32_t)there) != 0;
    float* o = out + slot * (LANES * V);
    __syncthreads();
#pragma unroll
    for (int j = 0; j < V; ++j)
      o[expert_of<LANES>(j, lane)] = whole && any ? -score(l[j], r, 0) * total : 0.f;
    __syncthreads();
    if (there) o[chosen] += d;
    __syncthreads();
    if (in) {
      T* q = (T*)p.grad + t * p.E;
#pragma unroll
      for (int j = 0; j < V; j += 4) {
        const int e = expert_of<LANES>(j, lane);
        store4(q + e, p.E - e, o + e);
      }
    }
  }
}

// bias += rate sign(mean of the counts - count), then the counts start again from zero.
__global__ __launch_bounds__(256) void k_route_balance(int E, long long* __restrict__ counts, float* __restrict__ bias,
                                                       float rate) {
  __shared__ long long part[4];
  long long sum = 0;
  for (int e = threadIdx.x; e < E; e += 256) sum += counts[e];
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
  __syncthreads();
  sum = part[0] + part[1] + part[2] + part[3];
  for (int e = threadIdx.x; e < E; e += 256) {
    const long long d = sum - counts[e] * E;
    bias[e] += d > 0 ? rate : d < 0 ? -rate : 0.f;
    counts[e] = 0;
  }
}

template <typename T> hipError_t route(const RouteParams& p, bool backward, hipStream_t st) {
  const bool wide = p.k > 16 || p.E > 256;
  const int tok = wide ? 4 : 16;
  const int64_t wgs = (p.tokens + tok - 1) / tok;
  const dim3 g((uint32_t)(wgs < 1024 ? wgs : 1024)), b(256);
#define ROUTE(LANES, V)                                                                               \
  do {                                                                                                \
    if (backward) hipLaunchKernelGGL((k_route_backward<T, LANES, V>), g, b, 0, st, p);                \
    else if (p.groups > 1) hipLaunchKernelGGL((k_route<T, LANES, V, true>), g, b, 0, st, p);          \
    else hipLaunchKernelGGL((k_route<T, LANES, V, false>), g, b, 0, st, p);                           \
  } while (0)
  if (!wide && p.E <= 64) ROUTE(16, 4);
  else if (!wide && p.E <= 128) ROUTE(16, 8);
  else if (!wide) ROUTE(16, 16);
  else if (p.E <= 256) ROUTE(64, 4);
  else if (p.E <= 512) ROUTE(64, 8);
  else ROUTE(64, 16);
#undef ROUTE
  return hipGetLastError();
}

}  // namespace

hipError_t launch_route(const RouteParams& p, hipStream_t st) {
  return p.bf16 ? route<bf16>(p, false, st) : route<float>(p, false, st);
}
hipError_t launch_route_backward(const RouteParams& p, hipStream_t st) {
  return p.bf16 ? route<bf16>(p, true, st) : route<float>(p, true, st);
}
hipError_t launch_route_balance(int E, long long* counts, float* bias, float rate, hipStream_t st) {
  hipLaunchKernelGGL(k_route_balance, dim3(1), dim3(256), 0, st, E, counts, bias, rate);
  return hipGetLastError();
}
