// Norm of all gradients, clipping, and AdamW over lists of tensors. All are bound by memory: each
// element is read once (and written once), and tensors of any number and size share a launch.
#include "train.h"

namespace {

typedef uint16_t u16x8u __attribute__((ext_vector_type(8), aligned(2)));
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2u __attribute__((ext_vector_type(2), aligned(1)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// Eight consecutive elements of any alignment (the hardware takes unaligned vector accesses);
// `left` of them exist, the others read as zero and are not written.
__device__ __forceinline__ void load8(const float* q, int64_t left, float (&x)[8]) {
  if (left >= 8) {
    const f32x4u a = *reinterpret_cast<const f32x4u*>(q), b = *reinterpret_cast<const f32x4u*>(q + 4);
#pragma unroll
    for (int j = 0; j < 4; ++j) { x[j] = a[j]; x[4 + j] = b[j]; }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = j < left ? q[j] : 0.f;
  }
}
__device__ __forceinline__ void load8(const bf16* q, int64_t left, float (&x)[8]) {
  if (left >= 8) {
    const u16x8u a = *reinterpret_cast<const u16x8u*>(q);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = __uint_as_float((uint32_t)a[j] << 16);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = j < left ? bf2f(q[j]) : 0.f;
  }
}
__device__ __forceinline__ void store8(float* q, int64_t left, const float (&x)[8]) {
  if (left >= 8) {
    *reinterpret_cast<f32x4u*>(q) = f32x4u{x[0], x[1], x[2], x[3]};
    *reinterpret_cast<f32x4u*>(q + 4) = f32x4u{x[4], x[5], x[6], x[7]};
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) if (j < left) q[j] = x[j];
  }
}
__device__ __forceinline__ void store8(bf16* q, int64_t left, const float (&x)[8]) {
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

// Index of the tensor a tile belongs to: the last one that starts at or before it.
template <typename F>
__device__ __forceinline__ int find_tensor(int n, uint32_t t, F start) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (start(mid) <= t) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// ---------------------------------------------------------------- norm and clipping
constexpr int GRAD_TILE = 8192;

__device__ __forceinline__ double block_sum(double x) {
  __shared__ double part[4];
  x = wave_sum_d(x);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
  __syncthreads();
  return (part[0] + part[1]) + (part[2] + part[3]);
}

template <typename T>
__device__ __forceinline__ void tile_squares(const T* g, int64_t left, double& sum) {
  for (int e = 8 * threadIdx.x; e < GRAD_TILE && e < left; e += 8 * 256) {
    float x[8];
    load8(g + e, left - e, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) sum = fma((double)x[j], (double)x[j], sum);
  }
}

// Squares are summed in 64 bits (no overflow or underflow of a square of a 32-bit gradient), in an
// order that depends on the list of tensors alone. Workgroup b takes the tiles b, b + NORM_WGS, ...
__global__ __launch_bounds__(256) void k_grad_norm(GradList L, double* __restrict__ partial, int first) {
  double sum = 0;
  for (uint32_t t = blockIdx.x; t < L.tiles; t += gridDim.x) {
    const int i = find_tensor(L.n, t, [&](int j) { return L.start[j]; });
    const int64_t e0 = (int64_t)(t - L.start[i]) * GRAD_TILE, left = L.count[i] - e0;
    if ((L.bf16[i >> 5] >> (i & 31)) & 1) tile_squares((const bf16*)L.g[i] + e0, left, sum);
    else tile_squares((const float*)L.g[i] + e0, left, sum);
  }
  sum = block_sum(sum);
  if (threadIdx.x == 0) partial[blockIdx.x] = first ? sum : partial[blockIdx.x] + sum;
}

// The norm and the coefficient that clips it to max_norm; NaN where the norm is not finite.
__global__ __launch_bounds__(256) void k_grad_norm_end(const double* __restrict__ partial, float max_norm,
                                                       float* __restrict__ out) {
  double sum = 0;
#pragma unroll
  for (int j = 0; j < NORM_WGS / 256; ++j) sum += partial[j * 256 + threadIdx.x];
  sum = block_sum(sum);
  if (threadIdx.x) return;
  const float norm = (float)sqrt(sum);
  out[0] = norm;
  out[1] = isfinite(norm) ? fminf(1.f, max_norm / (norm + 1e-6f)) : __builtin_nanf("");
}

template <typename T>
__device__ __forceinline__ void tile_scale(T* g, int64_t left, float c) {
  for (int e = 8 * threadIdx.x; e < GRAD_TILE && e < left; e += 8 * 256) {
    float x[8];
    load8(g + e, left - e, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = c == c ? x[j] * c : 0.f;
    store8(g + e, left - e, x);
  }
}

__global__ __launch_bounds__(256) void k_grad_scale(GradList L, const float* __restrict__ coef) {
  const float c = *coef;
  if (c == 1.f) return;
  for (uint32_t t = blockIdx.x; t < L.tiles; t += gridDim.x) {
    const int i = find_tensor(L.n, t, [&](int j) { return L.start[j]; });
    const int64_t e0 = (int64_t)(t - L.start[i]) * GRAD_TILE, left = L.count[i] - e0;
    if ((L.bf16[i >> 5] >> (i & 31)) & 1) tile_scale((bf16*)L.g[i] + e0, left, c);
    else tile_scale((float*)L.g[i] + e0, left, c);
  }
}

// ---------------------------------------------------------------- AdamW
constexpr int ADAMW_TILE = 2048;

// Moments of one element. The products and sums are rounded one by one (no fused multiply-adds): the
// 8-bit codes, whose rounding is a comparison, must not depend on which products are fused.
__device__ __forceinline__ void moments(float g, float& m, float& v, const AdamwList& L) {
#pragma clang fp contract(off)
  m = m * L.b1 + g * L.c1;
  v = v * L.b2 + (g * g) * L.c2;
}
__device__ __forceinline__ float updated(float p, float m, float v, const AdamwTensor& T, float eps) {
  return p * T.decay - T.lr * (m / (sqrtf(v * T.rbc2) + eps));
}

template <typename PT, typename GT>
__global__ __launch_bounds__(256) void k_adamw32(AdamwList L) {
  const uint32_t t = blockIdx.x;
  const int i = find_tensor(L.n, t, [&](int j) { return L.t[j].start; });
  const AdamwTensor& T = L.t[i];
  const float clip = L.clip ? *L.clip : 1.f;
  const int64_t e = (int64_t)(t - T.start) * ADAMW_TILE + 8 * threadIdx.x, left = T.count - e;
  if (left <= 0 || !(clip == clip)) return;
  float p[8], g[8], m[8], v[8];
  load8((const PT*)T.p + e, left, p);
  load8((const GT*)T.g + e, left, g);
  load8((const float*)T.m + e, left, m);
  load8((const float*)T.v + e, left, v);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    moments(g[j] * clip, m[j], v[j], L);
    p[j] = updated(p[j], m[j], v[j], T, L.eps);
  }
  store8((PT*)T.p + e, left, p);
  store8((float*)T.m + e, left, m);
  store8((float*)T.v + e, left, v);
}

// ---- 8-bit moments: blocks of 32 elements (four lanes of eight), a biased exponent for each moment.
constexpr uint32_t MIX_A = 0x9E3779B1u, MIX_B = 0x6A09E667u, MIX_C = 0xB7E15163u;

// 32 random bits for the elements 2c and 2c + 1 of a tensor.
__device__ __forceinline__ uint32_t random32(uint64_t c, uint32_t k0, uint32_t k1) {
  uint32_t x = (uint32_t)c + (uint32_t)(c >> 32) * MIX_C + k0;
  x = ((x ^ (x >> 16)) * MIX_A) ^ k1;
  x = (x ^ (x >> 15)) * MIX_B;
  return x ^ (x >> 16);
}

// Largest value over the four lanes of a block.
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, false));   // lane ^ 1
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, false));   // lane ^ 2
}

constexpr uint32_t INF_BITS = 0x7F800000u;

// Bits of the largest finite magnitude of a block.
__device__ __forceinline__ uint32_t block_top(const float (&x)[8]) {
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t b = __float_as_uint(x[j]) & 0x7FFFFFFFu;
    top = max(top, b < INF_BITS ? b : 0u);
  }
  return quad_max(top);
}
// Its exponent, one more where the significand is over 1.75: the codes' largest value is 1.75 2^e.
__device__ __forceinline__ int block_exponent(uint32_t top, int least) {
  return min(max((int)((top + 0x1FFFFFu) >> 23), least), 254);
}
__device__ __forceinline__ float two_to(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

template <typename PT, typename GT>
__global__ __launch_bounds__(256) void k_adamw8(AdamwList L) {
  const uint32_t t = blockIdx.x;
  const int i = find_tensor(L.n, t, [&](int j) { return L.t[j].start; });
  const AdamwTensor& T = L.t[i];
  const float clip = L.clip ? *L.clip : 1.f;
  if (!(clip == clip)) return;
  const int64_t e = (int64_t)(t - T.start) * ADAMW_TILE + 8 * threadIdx.x, left = T.count - e;
  float p[8], g[8], m[8], v[8];
  uint8_t* const mq = (uint8_t*)T.m + e;
  uint8_t* const vq = (uint8_t*)T.v + e;
  uint8_t* const sq = T.scales + (e >> 5) * 2;
  u32x2u mc = {0, 0}, vc = {0, 0};
  int em = 18, ev = 35;
#pragma unroll
  for (int j = 0; j < 8; ++j) p[j] = g[j] = 0.f;
  if (left > 0) {
    load8((const PT*)T.p + e, left, p);
    load8((const GT*)T.g + e, left, g);
    if (left >= 8) {
      mc = *reinterpret_cast<const u32x2u*>(mq);
      vc = *reinterpret_cast<const u32x2u*>(vq);
    } else {
      for (int j = 0; j < 8; ++j)
        if (j < left) {
          mc[j >> 2] |= (uint32_t)mq[j] << (8 * (j & 3));
          vc[j >> 2] |= (uint32_t)vq[j] << (8 * (j & 3));
        }
    }
    em = sq[0];
    ev = sq[1];
  }
  {
    const float s = two_to(em - 135);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)mc[h], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)mc[h], true);
      m[4 * h] = a[0] * s; m[4 * h + 1] = a[1] * s; m[4 * h + 2] = b[0] * s; m[4 * h + 3] = b[1] * s;
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t c = (vc[j >> 2] >> (8 * (j & 3))) & 255u;
    // a code's bits at the top of a 32-bit float's exponent and fraction are its value times 2^(31 - ev)
    v[j] = c == 255u ? __builtin_nanf("") : __builtin_amdgcn_ldexpf(__uint_as_float(c << 20), ev - 31);
    moments(g[j] * clip, m[j], v[j], L);
    p[j] = updated(p[j], m[j], v[j], T, L.eps);
  }
  em = block_exponent(block_top(m), 18);
  ev = block_exponent(block_top(v), 35);
  if (left <= 0) return;
  store8((PT*)T.p + e, left, p);
  uint32_t co[8], cv[8];
  const float sm = two_to(135 - em);
#pragma unroll
  for (int j = 0; j < 8; j += 2) {
    const float a = fminf(fmaxf(m[j] * sm, -448.f), 448.f), b = fminf(fmaxf(m[j + 1] * sm, -448.f), 448.f);
    const uint32_t w = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    co[j] = isfinite(m[j]) ? w & 255u : 0x7Fu;
    co[j + 1] = isfinite(m[j + 1]) ? (w >> 8) & 255u : 0x7Fu;
    const uint32_t r = random32((uint64_t)(e + j) >> 1, T.key0, T.key1);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const float x = v[j + q];
      const uint32_t b20 = __float_as_uint(__builtin_amdgcn_ldexpf(x, 31 - ev)) + ((q ? r >> 16 : r & 0xFFFFu) << 4);
      const uint32_t c = min(max(b20 >> 20, x > 0.f ? 1u : 0u), 254u);
      cv[j + q] = isfinite(x) ? c : 255u;
    }
  }
  if (left >= 8) {
    u32x2u a, b;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      a[h] = co[4 * h] | co[4 * h + 1] << 8 | co[4 * h + 2] << 16 | co[4 * h + 3] << 24;
      b[h] = cv[4 * h] | cv[4 * h + 1] << 8 | cv[4 * h + 2] << 16 | cv[4 * h + 3] << 24;
    }
    *reinterpret_cast<u32x2u*>(mq) = a;
    *reinterpret_cast<u32x2u*>(vq) = b;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) { mq[j] = (uint8_t)co[j]; vq[j] = (uint8_t)cv[j]; }
  }
  if ((threadIdx.x & 3) == 0) { sq[0] = (uint8_t)em; sq[1] = (uint8_t)ev; }
}

}  // namespace

uint32_t grad_tiles(int64_t count) { return (uint32_t)((count + GRAD_TILE - 1) / GRAD_TILE); }
uint32_t adamw_tiles(int64_t count) { return (uint32_t)((count + ADAMW_TILE - 1) / ADAMW_TILE); }

hipError_t launch_grad_norm(const GradList& l, double* partial, bool first, hipStream_t st) {
  hipLaunchKernelGGL(k_grad_norm, dim3(NORM_WGS), dim3(256), 0, st, l, partial, (int)first);
  return hipGetLastError();
}

hipError_t launch_grad_norm_end(const double* partial, float max_norm, float* out, hipStream_t st) {
  hipLaunchKernelGGL(k_grad_norm_end, dim3(1), dim3(256), 0, st, partial, max_norm, out);
  return hipGetLastError();
}

hipError_t launch_grad_scale(const GradList& l, const float* coef, hipStream_t st) {
  hipLaunchKernelGGL(k_grad_scale, dim3(l.tiles < 2048 ? l.tiles : 2048), dim3(256), 0, st, l, coef);
  return hipGetLastError();
}

hipError_t launch_adamw(const AdamwList& l, bool p_bf16, bool g_bf16, int bits, uint32_t total, hipStream_t st) {
  const dim3 g(total), b(256);
#define ADAMW(P, G)                                                        \
  do {                                                                     \
    if (bits == 8) hipLaunchKernelGGL((k_adamw8<P, G>), g, b, 0, st, l);   \
    else hipLaunchKernelGGL((k_adamw32<P, G>), g, b, 0, st, l);            \
  } while (0)
  if (p_bf16 && g_bf16) ADAMW(bf16, bf16);
  else if (p_bf16) ADAMW(bf16, float);
  else if (g_bf16) ADAMW(float, bf16);
  else ADAMW(float, float);
#undef ADAMW
  return hipGetLastError();
}
