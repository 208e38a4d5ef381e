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
constexpr int CHUNK = 8 * 256;        // elements a workgroup takes at a time, eight a thread

// Moments of one element. The products and sums are rounded one by one (no fused multiply-adds): the
// 8-bit codes, whose rounding is a comparison, must not depend on which products are fused.
__device__ __forceinline__ void moments(float g, float& m, float& v, const AdamwList& L) {
#pragma clang fp contract(off)
  m = m * L.b1 + g * L.c1;
  v = v * L.b2 + (g * g) * L.c2;
}
// The hardware's root and reciprocal (1 ulp each) for the update: it is rounded into a parameter many
// times its size. The smallest normal number under the root keeps its argument out of the subnormals,
// which the instruction takes for zero (1e-19 beside eps).
__device__ __forceinline__ float updated(float p, float m, float v, const AdamwTensor& T, float eps) {
  const float root = __builtin_amdgcn_sqrtf(fmaf(v, T.rbc2, 0x1p-126f)) + eps;
  return fmaf(-T.lr, m * __builtin_amdgcn_rcpf(root), p * T.decay);
}

template <typename PT, typename GT>
__device__ __forceinline__ void chunk32(const AdamwTensor& T, const AdamwList& L, float clip, int64_t e, int64_t left) {
  if (left <= 0) return;
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

template <typename PT, typename GT>
__global__ __launch_bounds__(256) void k_adamw32(AdamwList L) {
  const uint32_t t = blockIdx.x;
  const int i = find_tensor(L.n, t, [&](int j) { return L.t[j].start; });
  const AdamwTensor& T = L.t[i];
  const float clip = L.clip ? *L.clip : 1.f;
  if (!(clip == clip)) return;
  const int64_t e0 = (int64_t)(t - T.start) * CHUNK;
  const int64_t e = e0 + 8 * threadIdx.x;
  if (T.count - e0 >= CHUNK) chunk32<PT, GT>(T, L, clip, e, CHUNK);
  else chunk32<PT, GT>(T, L, clip, e, T.count - e);
}

// ---- 8-bit moments: blocks of 32 elements (four lanes of eight), a biased exponent for each moment.
constexpr uint32_t MIX_A = 0x9E3779B1u, MIX_B = 0x6A09E667u, MIX_C = 0xB7E15163u;

// 32 random bits for the elements 2c and 2c + 1 of a tensor. base: key0 and the index's upper half mixed.
__device__ __forceinline__ uint32_t random32(uint32_t c, uint32_t base, uint32_t k1) {
  uint32_t x = c + base;
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
constexpr uint32_t TOP_BITS = 0x7F600000u;     // 1.75 2^127: larger values do not fit the largest exponent

// The exponent of a block's largest magnitude, one more where the significand is over 1.75: the codes'
// largest value is 1.75 2^e.
__device__ __forceinline__ int block_exponent(uint32_t top, int least) {
  return max((int)((top + 0x1FFFFFu) >> 23), least);
}
__device__ __forceinline__ float two_to(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Codes of blocks with values that are not finite, or too large for the largest exponent: the exponents
// are those of the finite values.
__device__ __forceinline__ void encode_any(const float (&m)[8], const float (&v)[8], const uint32_t (&r)[4],
                                           uint32_t (&co)[2], uint32_t (&cv)[2], int& em, int& ev) {
  uint32_t tm = 0, tv = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t a = __float_as_uint(m[j]) & 0x7FFFFFFFu, b = __float_as_uint(v[j]) & 0x7FFFFFFFu;
    tm = max(tm, a < INF_BITS ? a : 0u);
    tv = max(tv, b < INF_BITS ? b : 0u);
  }
  em = min(block_exponent(quad_max(tm), 18), 254);
  ev = min(block_exponent(quad_max(tv), 35), 254);
  co[0] = co[1] = cv[0] = cv[1] = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float y = fminf(fmaxf(m[j] * two_to(135 - em), -448.f), 448.f);
    const uint32_t a = isfinite(m[j]) ? (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y, y, 0, false) & 255u : 0x7Fu;
    const uint32_t y20 = __float_as_uint(__builtin_amdgcn_ldexpf(v[j], 31 - ev)) + (((r[j >> 1] >> (16 * (j & 1))) & 0xFFFFu) << 4);
    const uint32_t b = isfinite(v[j]) ? min(max(y20 >> 20, v[j] > 0.f ? 1u : 0u), 254u) : 255u;
    co[j >> 2] |= a << (8 * (j & 3));
    cv[j >> 2] |= b << (8 * (j & 3));
  }
}

template <typename PT, typename GT>
__device__ __forceinline__ void chunk8(const AdamwTensor& T, const AdamwList& L, float clip, int64_t e, int64_t left) {
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
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < left) {
          mc[j >> 2] |= (uint32_t)mq[j] << (8 * (j & 3));
          vc[j >> 2] |= (uint32_t)vq[j] << (8 * (j & 3));
        }
    }
    em = sq[0];
    ev = sq[1];
  }
  const float s = two_to(max(em, 18) - 135);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)mc[h], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)mc[h], true);
    m[4 * h] = a[0] * s; m[4 * h + 1] = a[1] * s; m[4 * h + 2] = b[0] * s; m[4 * h + 3] = b[1] * s;
  }
  uint32_t tc = 0, tv = 0;
  float tm = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    // a code's bits below the sign and three bits of a 32-bit float are its value times 2^(31 - ev)
    const int sh = 20 - 8 * (j & 3);
    const uint32_t c = (sh >= 0 ? vc[j >> 2] << (sh & 31) : vc[j >> 2] >> (-sh & 31)) & 0x0FF00000u;
    tc = max(tc, c);
    v[j] = __builtin_amdgcn_ldexpf(__uint_as_float(c), ev - 31);
    moments(g[j] * clip, m[j], v[j], L);
    p[j] = updated(p[j], m[j], v[j], T, L.eps);
    tm = fmaxf(tm, fabsf(m[j]));
    tv = max(tv, __float_as_uint(v[j]));
  }
  const uint32_t qm = quad_max(__float_as_uint(tm));
  const uint32_t qv = quad_max(tc == 0x0FF00000u ? 0xFFFFFFFFu : tv);
  uint32_t r[4];
  const uint64_t c0 = (uint64_t)e >> 1;
  const uint32_t base = (uint32_t)(c0 >> 32) * MIX_C + T.key0;
#pragma unroll
  for (int j = 0; j < 4; ++j) r[j] = random32((uint32_t)c0 + j, base, T.key1);
  uint32_t co[2], cv[2];
  if (max(qm, qv) <= TOP_BITS) {
    em = block_exponent(qm, 18);
    ev = block_exponent(qv, 35);
    const float sm = two_to(135 - em);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      co[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(m[4 * h] * sm, m[4 * h + 1] * sm, 0, false);
      co[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(m[4 * h + 2] * sm, m[4 * h + 3] * sm, (int)co[h], true);
      uint32_t c[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float x = v[4 * h + j];
        const uint32_t rr = r[2 * h + (j >> 1)], r16 = j & 1 ? rr >> 16 : rr & 0xFFFFu;
        const uint32_t y = __float_as_uint(__builtin_amdgcn_ldexpf(x, 31 - ev)) + (r16 << 4);
        c[j] = max(y >> 20, min(__float_as_uint(x), 1u));      // not 0 where x is above 0
      }
      cv[h] = c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (((vc[j >> 2] >> (8 * (j & 3))) & 255u) == 255u) v[j] = p[j] = __builtin_nanf("");
    encode_any(m, v, r, co, cv, em, ev);
  }
  if (left <= 0) return;
  store8((PT*)T.p + e, left, p);
  if (left >= 8) {
    *reinterpret_cast<u32x2u*>(mq) = u32x2u{co[0], co[1]};
    *reinterpret_cast<u32x2u*>(vq) = u32x2u{cv[0], cv[1]};
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) {
        mq[j] = (uint8_t)(co[j >> 2] >> (8 * (j & 3)));
        vq[j] = (uint8_t)(cv[j >> 2] >> (8 * (j & 3)));
      }
  }
  if ((threadIdx.x & 3) == 0) { sq[0] = (uint8_t)em; sq[1] = (uint8_t)ev; }
}

template <typename PT, typename GT>
__global__ __launch_bounds__(256) void k_adamw8(AdamwList L) {
  const uint32_t t = blockIdx.x;
  const int i = find_tensor(L.n, t, [&](int j) { return L.t[j].start; });
  const AdamwTensor& T = L.t[i];
  const float clip = L.clip ? *L.clip : 1.f;
  if (!(clip == clip)) return;
  const int64_t e0 = (int64_t)(t - T.start) * CHUNK;
  const int64_t e = e0 + 8 * threadIdx.x;
  if (T.count - e0 >= CHUNK) chunk8<PT, GT>(T, L, clip, e, CHUNK);
  else chunk8<PT, GT>(T, L, clip, e, T.count - e);
}

}  // namespace

uint32_t grad_tiles(int64_t count) { return (uint32_t)((count + GRAD_TILE - 1) / GRAD_TILE); }
uint32_t adamw_tiles(int64_t count) { return (uint32_t)((count + CHUNK - 1) / CHUNK); }

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
