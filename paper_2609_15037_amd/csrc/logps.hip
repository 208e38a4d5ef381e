// Log-probabilities (and entropies) of given tokens under logits tokens x vocab, and the gradient of the logits.
// Forward: one pass over a row with the running maximum and sum of the exponentials; backward: one pass more, which
// writes the gradient. Both are bound by memory.
#include <float.h>

#include <type_traits>

#include "lanes.h"
#include "train.h"

namespace {

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.693147180559945309417f;
// Exponents of 2 below this have no weight in any sum; a bound keeps -inf out of products with 0.
constexpr float LEAST = -200.f;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4h __attribute__((ext_vector_type(4), aligned(2)));
// Sixteen bytes a lane, 4 fp32 or 8 bf16, of any alignment; ONCE: past the caches. A vector is loaded as it is and taken
// apart later: taken apart where it may not exist, each load would be waited for before the next.
template <bool ONCE> __device__ __forceinline__ u32x4 load(const float* q) {
  return GET(ONCE, reinterpret_cast<const u32x4u*>(q));
}
template <bool ONCE> __device__ __forceinline__ u32x4 load(const bf16* q) {
  return GET(ONCE, reinterpret_cast<const u32x4h*>(q));
}
template <typename T> __device__ __forceinline__ u32x4 nothing() {      // -inf
  const uint32_t x = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;
  return u32x4{x, x, x, x};
}
__device__ __forceinline__ void apart(const u32x4& a, float (&x)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = __uint_as_float(a[j]);
}
__device__ __forceinline__ void apart(const u32x4& a, float (&x)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(j & 1 ? a[j / 2] & 0xFFFF0000u : a[j / 2] << 16);
}
template <bool ONCE> __device__ __forceinline__ void store(float* q, const float (&x)[4]) {
  u32x4u a;
#pragma unroll
  for (int j = 0; j < 4; ++j) a[j] = __float_as_uint(x[j]);
  PUT(ONCE, reinterpret_cast<u32x4u*>(q), a);
}
template <bool ONCE> __device__ __forceinline__ void store(bf16* q, const float (&x)[8]) {
  u32x4h a;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    a[j] = (uint32_t)__builtin_bit_cast(uint16_t, f2bf(x[2 * j + 1])) << 16 | __builtin_bit_cast(uint16_t, f2bf(x[2 * j]));
  PUT(ONCE, reinterpret_cast<u32x4h*>(q), a);
}
__device__ __forceinline__ void store1(float* q, float x) { *q = x; }
__device__ __forceinline__ void store1(bf16* q, float x) { *q = f2bf(x); }
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
// The parts that LANES neighbouring lanes hold, put together in each of them.
template <int LANES, bool ENTROPY> __device__ __forceinline__ Part together(const Part& a, float k) {
  Part r = {max_of<LANES>(a.top), 0, 0};
  const float d = fmaxf((a.top - r.top) * k, LEAST);
  const double f = __builtin_amdgcn_exp2f(d);
  r.sum = sum_of<LANES>(f * a.sum);
  if (ENTROPY) r.bits = sum_of<LANES>(f * fma((double)d, a.sum, a.bits));
  return r;
}

// THREADS threads take a row. The label is left out of the sum, which is then small where the label has nearly all of
// the probability: log p = a - log1p(sum + (e_label - 1)) with a = scale (x_label - top) keeps its relative accuracy.
// A lane's sum is fp32, rescaled when its maximum grows (once for U vectors), the lanes' are joined in 64 bits. Of its last
// turn a wave skips the vectors that it has nothing of (2039 x 50021 fp32 on 512 threads 75 us with them, 67 without). Bound
// by reads; with a label in every row, two sets of logits in turn: 4096 x 131072 bf16 1.07 GB in 163 us, 6.6 TB/s, with entropies
// 191, 5.6; fp32 2.1 GB in 340 us, 6.3 TB/s; 2039 x 50021 fp32 with entropies, rows 50048 apart, 408 MB in 76 us, 5.4 TB/s (a tenth
// without a label: 58). 8 x 32000 4.7 us, a launch and the latencies of a row. One vector more in flight for each lane, a fetch ahead of the next turn,
// or registers held down for more waves (64: 120 us instead of 96 at 8192 x 32000) gained nothing.
template <typename T, int THREADS, int U, bool ENTROPY, bool ONCE>
__global__ __launch_bounds__(THREADS <= 64 ? 256 : THREADS) void k_logps(LogpsParams p) {
  constexpr int N = 16 / sizeof(T), BLOCK = THREADS <= 64 ? 256 : THREADS, ROWS = BLOCK / THREADS;
  constexpr int WAVES = THREADS < 64 ? 1 : THREADS / 64, LANES = THREADS < 64 ? THREADS : 64;
  __shared__ Part parts[2][WAVES];
  const int lane = threadIdx.x % THREADS, first = THREADS > 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x & -64) : 0;
  const float k = p.log2_scale;
  int turn = 0;
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
    // U vectors a lane; in the last ones (whole: false) those that there are, and of the row's last V % N elements one a lane
    auto take = [&](int at, auto whole) {
      constexpr bool WHOLE = decltype(whole)::value;
      const int base = at + N * lane;
      // whether the wave has any of its u-th vectors
      auto some = [&](int u) { return WHOLE || at + N * (first + u * THREADS) < V; };
      u32x4 raw[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int e = base + u * N * THREADS;
        if (!WHOLE) raw[u] = nothing<T>();
        if (WHOLE || e + N <= V) raw[u] = load<ONCE>(row + e);
      }
      const int rag = (V & -N) + lane;
      const float more = !WHOLE && rag < V && rag != own ? value(row + rag) : -__builtin_inff();
      float x[U][N];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (some(u)) apart(raw[u], x[u]);
      const unsigned hit = own - base;
      if (hit < N * THREADS * U && hit % (N * THREADS) < N)
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int j = 0; j < N; ++j) x[u][j] = hit == u * N * THREADS + j ? -__builtin_inff() : x[u][j];
      float most = WHOLE ? top : fmaxf(top, more);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (some(u))
#pragma unroll
          for (int j = 0; j < N; ++j) most = fmaxf(most, x[u][j]);
      const float d = fmaxf((top - most) * k, LEAST), f = __builtin_amdgcn_exp2f(d);
      if (ENTROPY) bits = f * fmaf(d, sum, bits);
      sum *= f;
      top = most;
      auto add = [&](float y) {
        const float t = (y - top) * k, e = __builtin_amdgcn_exp2f(t);
        sum += e;
        if (ENTROPY) bits = fmaf(e, fmaxf(t, LEAST), bits);
      };
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (some(u))
#pragma unroll
          for (int j = 0; j < N; ++j) add(x[u][j]);
      if (!WHOLE) add(more);
    };
    int at = 0;
    for (; at + N * THREADS * U <= V; at += N * THREADS * U) take(at, std::true_type{});
    if (at < V) take(at, std::false_type{});
    Part a = together<LANES, ENTROPY>(Part{top, sum, bits}, k);
    if (WAVES > 1) {
      // one barrier a row: the next row's parts go to the other half, and the first wave has read this one's when it
      // comes to the next barrier
      if ((threadIdx.x & 63) == 0) parts[turn][threadIdx.x >> 6] = a;
      __syncthreads();
      const int wave = threadIdx.x >> 6, i = threadIdx.x & 15;
      a = i < WAVES ? parts[turn][i] : Part{-FLT_MAX, 0, 0};
      turn ^= 1;
      if (wave) continue;
      a = together<16, ENTROPY>(a, k);
    }
    if (lane == 0) {
      const float last = fmaxf(a.top, xl), d = fmaxf((a.top - last) * k, LEAST);
      const double f = __builtin_amdgcn_exp2f(d), el = __builtin_amdgcn_exp2f((xl - last) * k);
      if (ENTROPY) a.bits = f * fma((double)d, a.sum, a.bits);
      a.sum *= f;
      const double total = a.sum + el;
      const float log = log1pf((float)(a.sum + (el - 1)));
      const float logp = (xl - last) * p.scale - log;
      p.logp[r] = logp;
      if (ENTROPY)
        p.entropy[r] = (float)((a.sum * log - (double)LN2 * a.bits) / total - (el > 0 ? el / total * logp : 0));
      reinterpret_cast<float4*>(p.stats)[r] = float4{last, log * LOG2E, (float)(a.sum / total), logp};
    }
  }
}

// 2^((x - top) k - log2 sum) is p; GROUP threads take U vectors a lane of a row. The label's own value has 1 - p and
// log p from the forward pass: no difference of values near 1. Parts of rows, not rows, so that a large vocabulary's few rows
// fill the GPU. The gradient is rounded once, to its type. Bound by memory; every row with a label and a gradient: 4096 x 131072
// bf16 2.15 GB in 345 us, 6.2 TB/s, with entropies 359, 6.0; fp32 4.3 GB in 734, 5.9; 2039 x 50021 fp32 with entropies 816 MB in
// 150 us, 5.4 TB/s.
template <typename T, int GROUP, bool ENTROPY, bool ONCE_IN, bool ONCE_OUT>
__global__ __launch_bounds__(256) void k_logps_backward(LogpsParams p, uint32_t parts) {
  constexpr int N = 16 / sizeof(T), U = 4, SPAN = GROUP * N * U, GROUPS = 256 / GROUP;
  const int lane = threadIdx.x % GROUP, first = GROUP > 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x & -64) : 0;
  const int64_t units = p.tokens * parts;
  for (int64_t i = (int64_t)blockIdx.x * GROUPS + threadIdx.x / GROUP; i < units; i += (int64_t)gridDim.x * GROUPS) {
    const int64_t r = parts == 1 ? i : i <= 0xFFFFFFFF ? (uint32_t)i / parts : i / parts;
    const int at = (int)(i - r * parts) * SPAN, base = at + N * lane, V = (int)p.vocab;
    const bool whole = at + SPAN <= V;
    const int rag = (V & -N) + lane;             // of the row's last V % N elements one a lane
    T* out = (T*)p.grad + r * p.grad_ld;
    const int64_t label = p.labels[r];
    const float g = p.logp[r], h = ENTROPY ? p.grad_entropy[r] : 0.f;
    if (label < 0 || label >= p.vocab || (g == 0 && h == 0)) {
      const float zero[N] = {};
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (whole || base + u * N * GROUP + N <= V) store<ONCE_OUT>(out + base + u * N * GROUP, zero);
      if (!whole && rag < V) store1(out + rag, 0.f);
      continue;
    }
    const T* row = row_of<T>(p, r);
    u32x4 raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int e = base + u * N * GROUP;
      raw[u] = nothing<T>();
      if (whole || e + N <= V) raw[u] = load<ONCE_IN>(row + e);
    }
    const float more = !whole && rag < V ? value(row + rag) : 0.f;
    const float4 s = reinterpret_cast<const float4*>(p.stats)[r];
    const float H = ENTROPY ? p.entropy[r] : 0.f, k = p.log2_scale;
    const float c0 = -p.scale * fmaf(h, H, g), c1 = -p.scale * h * LN2;
    auto slope = [&](float x) {
      const float t = fmaf(x - s.x, k, -s.y), q = __builtin_amdgcn_exp2f(t);
      return ENTROPY ? q * fmaf(c1, fmaxf(t, LEAST), c0) : q * c0;
    };
    // scale (g (1 - p) - h p (log p + H)); p log p is 0 where p is
    auto own = [&] {
      const float q = exp2f(s.w * LOG2E), b = ENTROPY && q > 0 ? h * q * (s.w + H) : 0.f;
      return p.scale * (g * s.z - b);
    };
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!whole && at + N * (first + u * GROUP) >= V) break;         // nothing for the whole wave
      const int e = base + u * N * GROUP;
      float x[N];
      apart(raw[u], x);
#pragma unroll
      for (int j = 0; j < N; ++j) x[j] = slope(x[j]);
      const unsigned hit = (int)label - e;
      if (hit < N) {
        const float y = own();
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] = hit == j ? y : x[j];
      }
      if (whole || e + N <= V) store<ONCE_OUT>(out + e, x);
    }
    if (!whole && rag < V) store1(out + rag, rag == label ? own() : slope(more));
  }
}

// Logits that are well over the memory-side cache (256 MiB) go past the caches, gradients where both are. Rows of 32000 bf16,
// both ways one after another, us, through the caches and past them: 250 MiB 122 and 134, 280 MiB 141 and 150, 300 MiB 160 and
// 160, 330 MiB 186 and 176, 420 MiB 236 and 219; 8192 x 32000 96 + 208 and 84 + 173. Gradients only past them: 183 MiB 95 and
// 99 through, 122 MiB 67 either way.
constexpr double CACHE = 300 << 20;
template <typename T> double bytes_of(const LogpsParams& p) { return (double)p.tokens * (double)p.vocab * sizeof(T); }
constexpr int64_t MOST_GROUPS = 1 << 21;        // workgroups of a launch: fewer than 2^32 threads

template <typename T, int THREADS, int U, bool ONCE> void forward(const LogpsParams& p, hipStream_t st) {
  constexpr int block = THREADS <= 64 ? 256 : THREADS, rows = block / THREADS;
  const int64_t n = (p.tokens + rows - 1) / rows;
  const dim3 g((uint32_t)(n < MOST_GROUPS ? n : MOST_GROUPS)), b(block);
  if (p.entropy) hipLaunchKernelGGL((k_logps<T, THREADS, U, true, ONCE>), g, b, 0, st, p);
  else hipLaunchKernelGGL((k_logps<T, THREADS, U, false, ONCE>), g, b, 0, st, p);
}
template <typename T, int THREADS, int U> void forward(const LogpsParams& p, hipStream_t st) {
  if (bytes_of<T>(p) > CACHE) forward<T, THREADS, U, true>(p, st); else forward<T, THREADS, U, false>(p, st);
}
template <typename T, int GROUP, bool ONCE_IN, bool ONCE_OUT> void backward(const LogpsParams& p, hipStream_t st) {
  constexpr int span = GROUP * 4 * (16 / sizeof(T)), groups = 256 / GROUP;
  const uint32_t parts = (uint32_t)((p.vocab + span - 1) / span);
  const int64_t n = (p.tokens * parts + groups - 1) / groups;
  const dim3 g((uint32_t)(n < MOST_GROUPS ? n : MOST_GROUPS)), b(256);
  if (p.grad_entropy) hipLaunchKernelGGL((k_logps_backward<T, GROUP, true, ONCE_IN, ONCE_OUT>), g, b, 0, st, p, parts);
  else hipLaunchKernelGGL((k_logps_backward<T, GROUP, false, ONCE_IN, ONCE_OUT>), g, b, 0, st, p, parts);
}
template <typename T, int GROUP> void backward(const LogpsParams& p, hipStream_t st) {
  const double bytes = bytes_of<T>(p);
  if (bytes > CACHE) backward<T, GROUP, true, true>(p, st);
  else if (2 * bytes > CACHE) backward<T, GROUP, false, true>(p, st);
  else backward<T, GROUP, false, false>(p, st);
}

}  // namespace

// Threads of a row: a turn of all of them takes 4 vectors each, and what a row's last turn lacks is lost. Many rows, us, on
// 64, 256, 512 and 1024 threads: bf16 16384 x 3000 21, 37, 75 and 127; 16384 x 9000 52, 65, 97 and 174; 8192 x 20000 61, 56, 77
// and 107; 4096 x 65536 102, 87, 85 and 96; 4096 x 100000 139, 140, 135 and 145; fp32 16384 x 4096 45, 41, 60 and 128; 8192 x
// 20000 102, 101, 98 and 127; 4096 x 131072 329, 323, 318 and 314. Few rows: bf16 64 x 4096 4.2, 3.8, 3.7 and 3.9; 1024 x 4096
// 4.2, 4.9, 6.6 and 9.8; 1024 x 8192 5.7, 5.2, 7.0 and 10.6; 256, 512 and 1024 threads: 256 x 50021 7.7, 6.8 and 6.9; 300 x
// 50021 10.0, 10.6 and 12.1. 65536 x 512 15 on 16 lanes, 44 on a wave.
hipError_t launch_logps(const LogpsParams& p, hipStream_t st) {
  const int64_t vectors = (p.vocab + (p.bf16 ? 7 : 3)) / (p.bf16 ? 8 : 4);
#define LOGPS(THREADS, U) p.bf16 ? forward<bf16, THREADS, U>(p, st) : forward<float, THREADS, U>(p, st)
  if (vectors <= 128) LOGPS(16, 2);
  else if (p.tokens <= 256 && vectors >= 1280) LOGPS(512, 4);
  else if ((p.tokens > 512 && vectors <= 512) || (p.tokens >= 2048 && vectors <= 1280)) LOGPS(64, 4);
  else if (vectors <= (p.bf16 ? 8192 : 4096)) LOGPS(256, 4);
  else LOGPS(512, 4);
#undef LOGPS
  return hipGetLastError();
}

// Threads of a row's part. bf16, us: 65536 x 512 22 on 16 lanes, 35 on a wave, 114 on 256 threads; on a wave and on 256 threads:
// 16384 x 2100 26 and 31, x 9000 103 and 129, 8192 x 32000 186 and 181, 4096 x 131072 342 and 339; fp32 16384 x 5000 111 and 133,
// 8192 x 16384 175 and 169.
hipError_t launch_logps_backward(const LogpsParams& p, hipStream_t st) {
  const int64_t vectors = (p.vocab + (p.bf16 ? 7 : 3)) / (p.bf16 ? 8 : 4);
#define LOGPS(GROUP) p.bf16 ? backward<bf16, GROUP>(p, st) : backward<float, GROUP>(p, st)
  if (vectors <= 128) LOGPS(16);
  else if (vectors <= 2048) LOGPS(64);
  else LOGPS(256);
#undef LOGPS
  return hipGetLastError();
}
