// Log-probabilities (and entropies) of given tokens under logits tokens x vocab, and the gradient of the logits.
// Forward: one pass over a row with the running maximum and sum of the exponentials; backward: one pass more, which
// writes the gradient. Both are bound by memory.
#include <float.h>

#include "train.h"

namespace {

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.693147180559945309417f;
// Exponents of 2 below this have no weight in any sum; a bound keeps -inf out of products with 0.
constexpr float LEAST = -200.f;

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef uint16_t u16x8u __attribute__((ext_vector_type(8), aligned(2)));
// Sixteen bytes a lane: 4 fp32 or 8 bf16, of any alignment; `left` of them exist, the others are -inf and not written.
__device__ __forceinline__ void load(const float* q, int left, float (&x)[4]) {
  if (left >= 4) {
    const f32x4u a = *reinterpret_cast<const f32x4u*>(q);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = a[j];
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = j < left ? q[j] : -__builtin_inff();
  }
}
__device__ __forceinline__ void load(const bf16* q, int left, float (&x)[8]) {
  if (left >= 8) {
    const u16x8u a = *reinterpret_cast<const u16x8u*>(q);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = __uint_as_float((uint32_t)a[j] << 16);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = j < left ? bf2f(q[j]) : -__builtin_inff();
  }
}
__device__ __forceinline__ void store(float* q, int left, const float (&x)[4]) {
  if (left >= 4) {
    *reinterpret_cast<f32x4u*>(q) = f32x4u{x[0], x[1], x[2], x[3]};
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) if (j < left) q[j] = x[j];
  }
}
__device__ __forceinline__ void store(bf16* q, int left, const float (&x)[8]) {
  if (left >= 8) {
    u16x8u a;
#pragma unroll
    for (int j = 0; j < 8; ++j) a[j] = __builtin_bit_cast(uint16_t, f2bf(x[j]));
    *reinterpret_cast<u16x8u*>(q) = a;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) if (j < left) q[j] = f2bf(x[j]);
  }
}
__device__ __forceinline__ float value(const float* q) { return *q; }
__device__ __forceinline__ float value(const bf16* q) { return bf2f(*q); }

template <typename T> __device__ __forceinline__ const T* row_of(const LogpsParams& p, int64_t r) {
  const T* q = (const T*)p.logits;
  return p.inner >= p.tokens ? q + r * p.ld : q + (r / p.inner) * p.outer + (r % p.inner) * p.ld;
}

// Part of a row without its label: the largest logit, the sum of e = 2^((x - top) k) and of e (x - top) k.
struct Part {
  float top;
  double sum, bits;
};
__device__ __forceinline__ Part joined(const Part& a, const Part& b, float k, bool entropy) {
  const float top = fmaxf(a.top, b.top);
  const float da = fmaxf((a.top - top) * k, LEAST), db = fmaxf((b.top - top) * k, LEAST);
  const double fa = exp2f(da), fb = exp2f(db);
  Part r = {top, a.sum * fa + b.sum * fb, 0};
  if (entropy) r.bits = fa * (a.bits + da * a.sum) + fb * (b.bits + db * b.sum);
  return r;
}

// THREADS threads take a row. The label is left out of the sum, which is then small where the label has nearly all of
// the probability: log p = a - log1p(sum + (e_label - 1)) with a = scale (x_label - top) keeps its relative accuracy.
template <typename T, int THREADS, bool ENTROPY>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void k_logps(LogpsParams p) {
  constexpr int N = 16 / sizeof(T), U = 4, BLOCK = THREADS < 256 ? 256 : THREADS, ROWS = BLOCK / THREADS;
  __shared__ Part parts[THREADS / 64];
  const int lane = threadIdx.x % THREADS;
  const float k = p.log2_scale;
  for (int64_t r = (int64_t)blockIdx.x * ROWS + threadIdx.x / THREADS; r < p.tokens; r += (int64_t)gridDim.x * ROWS) {
    const int64_t label = p.labels[r];
    if (label < 0 || label >= p.vocab) {
      if (lane == 0) {
        p.logp[r] = 0.f;
        if (ENTROPY) p.entropy[r] = 0.f;
        reinterpret_cast<float4*>(p.stats)[r] = float4{0.f, 0.f, 0.f, 0.f};
      }
      continue;
    }
    const T* row = row_of<T>(p, r);
    const int V = (int)p.vocab, own = (int)label;
    const float xl = value(row + own);
    float top = -FLT_MAX, sum = 0, bits = 0;
    for (int base = N * lane; base < V; base += N * THREADS * U) {
      float x[U][N];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int e = base + u * N * THREADS;
        load(row + e, V - e, x[u]);
      }
      float most = top;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int at = own - (base + u * N * THREADS);
        if ((unsigned)at < (unsigned)N)
#pragma unroll
          for (int j = 0; j < N; ++j) x[u][j] = j == at ? -__builtin_inff() : x[u][j];
#pragma unroll
        for (int j = 0; j < N; ++j) most = fmaxf(most, x[u][j]);
      }
      const float d = fmaxf((top - most) * k, LEAST), f = exp2f(d);
      if (ENTROPY) bits = f * (bits + d * sum);
      sum *= f;
      top = most;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const float t = (x[u][j] - top) * k, e = __builtin_amdgcn_exp2f(t);
          sum += e;
          if (ENTROPY) bits = fmaf(e, fmaxf(t, LEAST), bits);
        }
    }
    Part a = {top, sum, bits};
    for (int o = 32; o > 0; o >>= 1)
      a = joined(a, Part{__shfl_xor(a.top, o, 64), __shfl_xor(a.sum, o, 64), __shfl_xor(a.bits, o, 64)}, k, ENTROPY);
    if (THREADS > 64) {
      __syncthreads();          // the last row's have been read
      if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = a;
      __syncthreads();
      a = parts[0];
      for (int i = 1; i < THREADS / 64; ++i) a = joined(a, parts[i], k, ENTROPY);
    }
    if (lane == 0) {
      const float last = fmaxf(a.top, xl);
      a = joined(a, Part{last, 0, 0}, k, ENTROPY);
      const float el = exp2f((xl - last) * k);
      const double total = a.sum + (double)el;
      const float log = log1pf((float)(a.sum + ((double)el - 1)));
      const float logp = (xl - last) * p.scale - log;
      p.logp[r] = logp;
      if (ENTROPY)
        p.entropy[r] = (float)((a.sum * log - (double)LN2 * a.bits) / total - (el > 0 ? (double)el / total * logp : 0));
      reinterpret_cast<float4*>(p.stats)[r] = float4{last, log * LOG2E, (float)(a.sum / total), logp};
    }
  }
}

// 2^((x - top) k - log2 sum) is p; a workgroup takes U vectors a lane of a row. The label's own value has 1 - p and
// log p from the forward pass.
template <typename T, bool ENTROPY> __global__ __launch_bounds__(256) void k_logps_backward(LogpsParams p, int parts) {
  constexpr int N = 16 / sizeof(T), U = 4, SPAN = 256 * N * U;
  const int64_t units = p.tokens * parts;
  for (int64_t i = blockIdx.x; i < units; i += gridDim.x) {
    const int64_t r = i / parts;
    const int base = (int)(i - r * parts) * SPAN + N * threadIdx.x, V = (int)p.vocab;
    T* out = (T*)p.grad + r * p.grad_ld;
    const int64_t label = p.labels[r];
    const float g = p.logp[r], h = ENTROPY ? p.grad_entropy[r] : 0.f;
    if (label < 0 || label >= p.vocab || (g == 0 && h == 0)) {
      float zero[N] = {};
#pragma unroll
      for (int u = 0; u < U; ++u) store(out + base + u * N * 256, V - (base + u * N * 256), zero);
      continue;
    }
    const T* row = row_of<T>(p, r);
    const float4 s = reinterpret_cast<const float4*>(p.stats)[r];
    const float H = ENTROPY ? p.entropy[r] : 0.f, k = p.log2_scale;
    const float c0 = -p.scale * fmaf(h, H, g), c1 = -p.scale * h * LN2;
    float x[U][N];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int e = base + u * N * 256;
      load(row + e, V - e, x[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int e = base + u * N * 256, at = (int)label - e;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float t = fmaf(x[u][j] - s.x, k, -s.y), q = __builtin_amdgcn_exp2f(t);
        x[u][j] = ENTROPY ? q * fmaf(c1, fmaxf(t, LEAST), c0) : q * c0;
      }
      if ((unsigned)at < (unsigned)N) {
        // scale (g (1 - p) - h p (log p + H)); p log p is 0 where p is
        const float q = exp2f(s.w * LOG2E), b = ENTROPY && q > 0 ? h * q * (s.w + H) : 0.f;
        const float y = p.scale * (g * s.z - b);
#pragma unroll
        for (int j = 0; j < N; ++j) x[u][j] = j == at ? y : x[u][j];
      }
      store(out + e, V - e, x[u]);
    }
  }
}

constexpr int64_t MOST_GROUPS = 1 << 22;        // workgroups of a launch: fewer than 2^32 threads

template <typename T, int THREADS> void forward(const LogpsParams& p, hipStream_t st) {
  constexpr int block = THREADS < 256 ? 256 : THREADS, rows = block / THREADS;
  const int64_t n = (p.tokens + rows - 1) / rows;
  const dim3 g((uint32_t)(n < MOST_GROUPS ? n : MOST_GROUPS)), b(block);
  if (p.entropy) hipLaunchKernelGGL((k_logps<T, THREADS, true>), g, b, 0, st, p);
  else hipLaunchKernelGGL((k_logps<T, THREADS, false>), g, b, 0, st, p);
}
template <typename T> void backward(const LogpsParams& p, hipStream_t st) {
  constexpr int span = 256 * 4 * (16 / sizeof(T));
  const int parts = (int)((p.vocab + span - 1) / span);
  const int64_t n = p.tokens * parts;
  const dim3 g((uint32_t)(n < MOST_GROUPS ? n : MOST_GROUPS)), b(256);
  if (p.grad_entropy) hipLaunchKernelGGL((k_logps_backward<T, true>), g, b, 0, st, p, parts);
  else hipLaunchKernelGGL((k_logps_backward<T, false>), g, b, 0, st, p, parts);
}

}  // namespace

hipError_t launch_logps(const LogpsParams& p, hipStream_t st) {
  const bool small = p.vocab <= 2048;
  if (p.bf16) small ? forward<bf16, 64>(p, st) : forward<bf16, 256>(p, st);
  else small ? forward<float, 64>(p, st) : forward<float, 256>(p, st);
  return hipGetLastError();
}

hipError_t launch_logps_backward(const LogpsParams& p, hipStream_t st) {
  if (p.bf16) backward<bf16>(p, st); else backward<float>(p, st);
  return hipGetLastError();
}
