// Norm of all gradients, clipping, and AdamW over lists of tensors. All are bound by memory: each
// element is read once (and written once), and tensors of any number and size share a launch.
#include "train.h"

namespace {

// Vectors of any alignment (the hardware takes unaligned vector accesses). A lane's 16 bytes and the next
// lane's are neighbours in every access: lanes that took 32 consecutive bytes of fp32 in two halves
// touched each line twice (32-bit AdamW over 66 M elements 254 us instead of 227 side by side).
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32u __attribute__((aligned(1)));
typedef uint16_t u16u __attribute__((aligned(1)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// N consecutive elements (4, or 8 of bf16); `left` of them exist, the others read as zero and are not written. ONCE: the line is
// not needed again soon.
template <bool ONCE, int N> __device__ __forceinline__ void load(const float* q, int64_t left, float (&x)[N]) {
  static_assert(N == 4);
  if (left >= N) {
    const f32x4u a = GET(ONCE, reinterpret_cast<const f32x4u*>(q));
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = a[j];
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = j < left ? q[j] : 0.f;
  }
}
template <bool ONCE, int N> __device__ __forceinline__ void load(const bf16* q, int64_t left, float (&x)[N]) {
  typedef uint16_t vec __attribute__((ext_vector_type(N), aligned(2)));
  if (left >= N) {
    const vec a = GET(ONCE, reinterpret_cast<const vec*>(q));
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = __uint_as_float((uint32_t)a[j] << 16);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = j < left ? bf2f(q[j]) : 0.f;
  }
}
template <bool ONCE, int N> __device__ __forceinline__ void store(float* q, int64_t left, const float (&x)[N]) {
  static_assert(N == 4);
  if (left >= N) {
    PUT(ONCE, reinterpret_cast<f32x4u*>(q), (f32x4u{x[0], x[1], x[2], x[3]}));
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) if (j < left) q[j] = x[j];
  }
}
template <bool ONCE, int N> __device__ __forceinline__ void store(bf16* q, int64_t left, const float (&x)[N]) {
  typedef uint16_t vec __attribute__((ext_vector_type(N), aligned(2)));
  if (left >= N) {
    vec a;
#pragma unroll
    for (int j = 0; j < N; ++j) a[j] = __builtin_bit_cast(uint16_t, f2bf(x[j]));
    PUT(ONCE, reinterpret_cast<vec*>(q), a);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) if (j < left) q[j] = f2bf(x[j]);
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

// f(values, pointer, how many exist) for 16 bytes a lane over a tile.
template <bool ONCE, typename T, typename F>
__device__ __forceinline__ void each_of_tile(T* g, int64_t left, F f) {
  constexpr int N = 16 / sizeof(T);
  if (left >= GRAD_TILE) {
#pragma unroll 4
    for (int e = N * threadIdx.x; e < GRAD_TILE; e += N * 256) {
      float x[N];
      load<ONCE>(g + e, N, x);
      f(x, g + e, (int64_t)N);
    }
  } else {
    for (int e = N * threadIdx.x; e < left; e += N * 256) {
      float x[N];
      load<ONCE>(g + e, left - e, x);
      f(x, g + e, left - e);
    }
  }
}
// A workgroup's tiles: its own, and every gridDim.x-th after it.
template <bool ONCE, typename F>
__device__ __forceinline__ void each_tile(const GradList& L, F f) {
  for (uint32_t t = blockIdx.x; t < L.tiles; t += gridDim.x) {
    const int i = find_tensor(L.n, t, [&](int j) { return L.start[j]; });
    const int64_t e0 = (int64_t)(t - L.start[i]) * GRAD_TILE, left = L.count[i] - e0;
    if ((L.bf16[i >> 5] >> (i & 31)) & 1) each_of_tile<ONCE>((bf16*)L.g[i] + e0, left, f);
    else each_of_tile<ONCE>((float*)L.g[i] + e0, left, f);
  }
}

__device__ __forceinline__ double block_sum(double x) {
  __shared__ double part[4];
  x = wave_sum_d(x);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
  __syncthreads();
  return (part[0] + part[1]) + (part[2] + part[3]);
}

// Squares are summed in 64 bits (no overflow or underflow of a square of a 32-bit gradient), in an
// order that depends on the list of tensors alone: the workgroups' sums go to the workspace, a second
// launch adds them up. (The last workgroup to arrive could: the fences of 1024 arrivals took 20 us, those
// of 97 as long as the second launch.)
// 1.62 GB of bf16 gradients: 237 us, 6.8 TB/s (the copy rate of this card is 5.4, a library sum's 5.6).
template <bool ONCE>
__global__ __launch_bounds__(256) void k_grad_norm(GradList L, double* __restrict__ partial, uint32_t filled) {
  double sum = 0;
  each_tile<ONCE>(L, [&](const auto& x, const void*, int64_t) {
#pragma unroll
    for (float v : x) sum = fma((double)v, (double)v, sum);
  });
  sum = block_sum(sum);
  if (threadIdx.x == 0) partial[blockIdx.x] = blockIdx.x < filled ? partial[blockIdx.x] + sum : sum;
}

// The norm and the coefficient that clips it to max_norm; NaN where the norm is not finite.
__global__ __launch_bounds__(256) void k_grad_norm_end(const double* __restrict__ partial, uint32_t filled, float max_norm,
                                                       float* __restrict__ out) {
  double sum = 0;
#pragma unroll
  for (int j = 0; j < NORM_WGS / 256; ++j) {
    const uint32_t b = j * 256 + threadIdx.x;
    sum += b < filled ? partial[b] : 0.0;
  }
  sum = block_sum(sum);
  if (threadIdx.x) return;
  const float norm = (float)sqrt(sum);
  out[0] = norm;
  out[1] = isfinite(norm) ? fminf(1.f, max_norm / (norm + 1e-6f)) : __builtin_nanf("");
}

template <bool ONCE>
__global__ __launch_bounds__(256) void k_grad_scale(GradList L, const float* __restrict__ coef) {
  const float c = *coef;
  if (c == 1.f) return;
  each_tile<ONCE>(L, [&](auto& x, auto* q, int64_t left) {
#pragma unroll
    for (float& v : x) v = c == c ? v * c : 0.f;
    store<ONCE>(q, left, x);
  });
}

// ---------------------------------------------------------------- AdamW
constexpr int THREADS = 512;
constexpr int CHUNK = 4 * THREADS;      // elements of a workgroup, four a thread

// One tensor of a list, and its random bits' keys.
struct AdamwTensor : AdamwSet {
  void* p;
  const void* g;
  void* m;
  void* v;
  uint8_t* scales;
  int64_t count;
  uint32_t start, key0, key1;
  __device__ __forceinline__ AdamwTensor(const AdamwList& L, int i) : AdamwSet(L.set[(L.about[i] >> ADAMW_SET_BIT) & 7]) {
    p = L.p[i];
    g = L.g[i];
    m = L.m[i];
    v = L.v[i];
    scales = L.scales[i];
    count = (int64_t)(L.about[i] & (((uint64_t)1 << ADAMW_SET_BIT) - 1));
    start = L.start[i];
    key0 = mix32((uint32_t)L.seed ^ mix32((uint32_t)(L.seed >> 32) ^ mix32((uint32_t)(L.about[i] >> ADAMW_PLACE_BIT))));
    key1 = mix32(key0 ^ MIX_C);
  }
};

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
  float p[4], g[4], m[4], v[4];
  load<true>((const PT*)T.p + e, left, p);
  load<true>((const GT*)T.g + e, left, g);
  load<true>((const float*)T.m + e, left, m);
  load<true>((const float*)T.v + e, left, v);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    moments(g[j] * clip, m[j], v[j], L);
    p[j] = updated(p[j], m[j], v[j], T, L.eps);
  }
  store<true>((PT*)T.p + e, left, p);
  store<true>((float*)T.m + e, left, m);
  store<true>((float*)T.v + e, left, v);
}

// ---- 8-bit moments: blocks of 32 elements (eight lanes of four), a biased exponent for each moment.
// 32 random bits for the elements 2c and 2c + 1 of a tensor. base: key0 and the index's upper half mixed.
__device__ __forceinline__ uint32_t random32(uint32_t c, uint32_t base, uint32_t k1) {
  uint32_t x = c + base;
  x = ((x ^ (x >> 16)) * MIX_A) ^ k1;
  x = (x ^ (x >> 15)) * MIX_B;
  return x ^ (x >> 16);
}

// Largest value over the eight lanes of a block.
__device__ __forceinline__ uint32_t block_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, false));   // lane ^ 1
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, false));   // lane ^ 2
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xF, 0xF, false));   // mirrored in eight
}

// The 16 bits of a lane's element j.
__device__ __forceinline__ uint32_t random_of(const uint32_t (&r)[2], int j) {
  return j & 1 ? r[j >> 1] >> 16 : r[j >> 1] & 0xFFFFu;
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
__device__ __forceinline__ void encode_any(const float (&m)[4], const float (&v)[4], const uint32_t (&r)[2],
                                           uint32_t& co, uint32_t& cv, int& em, int& ev) {
  uint32_t tm = 0, tv = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t a = __float_as_uint(m[j]) & 0x7FFFFFFFu, b = __float_as_uint(v[j]) & 0x7FFFFFFFu;
    tm = max(tm, a < INF_BITS ? a : 0u);
    tv = max(tv, b < INF_BITS ? b : 0u);
  }
  em = min(block_exponent(block_max(tm), 18), 254);
  ev = min(block_exponent(block_max(tv), 35), 254);
  co = cv = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float y = fminf(fmaxf(m[j] * two_to(135 - em), -448.f), 448.f);
    const uint32_t a = isfinite(m[j]) ? (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y, y, 0, false) & 255u : 0x7Fu;
    const uint32_t y20 = __float_as_uint(__builtin_amdgcn_ldexpf(v[j], 31 - ev)) + (random_of(r, j) << 4);
    const uint32_t b = isfinite(v[j]) ? min(max(y20 >> 20, v[j] > 0.f ? 1u : 0u), 254u) : 255u;
    co |= a << (8 * j);
    cv |= b << (8 * j);
  }
}

template <typename PT, typename GT>
__device__ __forceinline__ void chunk8(const AdamwTensor& T, const AdamwList& L, float clip, int64_t e, int64_t left) {
  float p[4] = {}, g[4] = {}, m[4], v[4];
  uint8_t* const mq = (uint8_t*)T.m + e;
  uint8_t* const vq = (uint8_t*)T.v + e;
  u16u* const sq = reinterpret_cast<u16u*>(T.scales + (e >> 5) * 2);
  uint32_t mc = 0, vc = 0, sc = 0;
  if (left > 0) {
    load<true>((const PT*)T.p + e, left, p);
    load<true>((const GT*)T.g + e, left, g);
    if (left >= 4) {
      mc = GET(true, reinterpret_cast<const u32u*>(mq));
      vc = GET(true, reinterpret_cast<const u32u*>(vq));
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j < left) {
          mc |= (uint32_t)mq[j] << (8 * j);
          vc |= (uint32_t)vq[j] << (8 * j);
        }
    }
    sc = *sq;
  }
  int em = sc & 255, ev = sc >> 8;
  {
    const float s = two_to(max(em, 18) - 135);
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)mc, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)mc, true);
    m[0] = a[0] * s; m[1] = a[1] * s; m[2] = b[0] * s; m[3] = b[1] * s;
  }
  uint32_t tc = 0, tv = 0;
  float tm = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    // a code's bits below the sign and three bits of a 32-bit float are its value times 2^(31 - ev)
    const int sh = 20 - 8 * j;
    const uint32_t c = (sh >= 0 ? vc << (sh & 31) : vc >> (-sh & 31)) & 0x0FF00000u;
    tc = max(tc, c);
    v[j] = __builtin_amdgcn_ldexpf(__uint_as_float(c), ev - 31);
    moments(g[j] * clip, m[j], v[j], L);
    p[j] = updated(p[j], m[j], v[j], T, L.eps);
    tm = fmaxf(tm, fabsf(m[j]));
    tv = max(tv, __float_as_uint(v[j]));
  }
  // the code 255 stands for NaN: as every value that is not finite, it is over TOP_BITS
  const uint32_t qm = block_max(__float_as_uint(tm)), qv = block_max(tc == 0x0FF00000u ? 0xFFFFFFFFu : tv);
  const uint64_t c0 = (uint64_t)e >> 1;
  const uint32_t base = (uint32_t)(c0 >> 32) * MIX_C + T.key0;
  const uint32_t r[2] = {random32((uint32_t)c0, base, T.key1), random32((uint32_t)c0 + 1, base, T.key1)};
  uint32_t co, cv;
  if (max(qm, qv) <= TOP_BITS) {
    em = block_exponent(qm, 18);
    ev = block_exponent(qv, 35);
    const float sm = two_to(135 - em);
    co = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(m[0] * sm, m[1] * sm, 0, false);
    co = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(m[2] * sm, m[3] * sm, (int)co, true);
    cv = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t y = __float_as_uint(__builtin_amdgcn_ldexpf(v[j], 31 - ev)) + (random_of(r, j) << 4);
      cv |= max(y >> 20, min(__float_as_uint(v[j]), 1u)) << (8 * j);      // not 0 where v is above 0
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (((vc >> (8 * j)) & 255u) == 255u) v[j] = p[j] = __builtin_nanf("");
    encode_any(m, v, r, co, cv, em, ev);
  }
  if (left <= 0) return;
  store<true>((PT*)T.p + e, left, p);
  if (left >= 4) {
    PUT(true, reinterpret_cast<u32u*>(mq), (u32u)co);
    PUT(true, reinterpret_cast<u32u*>(vq), (u32u)cv);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < left) {
        mq[j] = (uint8_t)(co >> (8 * j));
        vq[j] = (uint8_t)(cv >> (8 * j));
      }
  }
  if ((threadIdx.x & 7) == 0) *sq = (uint16_t)(em | ev << 8);
}

// One chunk a workgroup: two or four in a row measured 7 and 12 % slower, eight elements a thread 2 %
// faster on aligned bf16 and 5 % slower elsewhere, 256 threads 2 % slower. Reads and writes are
// non-temporal: the next reader of a line is the next step or the next forward pass (32 bits, 66 M
// elements 275 -> 254 us; 8 bits, 262 M elements 485 -> 419 us). Measured, bf16 parameters and gradients:
// 32 bits 237 us for 66 M elements, 6.1 TB/s; 8 bits 433 us for 262 M elements, 6.1 TB/s (its arithmetic
// alone, about 50 issue slots an element, would take 340). fp32 parameters that start on odd elements:
// 8 bits, 66 M elements, 169 us, 5.5 TB/s.
template <typename PT, typename GT, int BITS>
__global__ __launch_bounds__(THREADS) void k_adamw(AdamwList L) {
  const uint32_t t = blockIdx.x;
  const AdamwTensor T(L, find_tensor(L.n, t, [&](int j) { return L.start[j]; }));
  const float clip = L.clip ? *L.clip : 1.f;
  if (!(clip == clip)) return;
  const int64_t e0 = (int64_t)(t - T.start) * CHUNK, e = e0 + 4 * threadIdx.x;
  if (T.count - e0 >= CHUNK) {      // no lane asks what is left
    if (BITS == 8) chunk8<PT, GT>(T, L, clip, e, 4);
    else chunk32<PT, GT>(T, L, clip, e, 4);
  } else {
    if (BITS == 8) chunk8<PT, GT>(T, L, clip, e, T.count - e);
    else chunk32<PT, GT>(T, L, clip, e, T.count - e);
  }
}

}  // namespace

uint32_t grad_tiles(int64_t count) { return (uint32_t)((count + GRAD_TILE - 1) / GRAD_TILE); }
uint32_t adamw_tiles(int64_t count) { return (uint32_t)((count + CHUNK - 1) / CHUNK); }

// Lists over the 256 MB of the memory-side cache leave nothing there for the next reader of the
// gradients: they are read past it (1.62 GB 263 -> 237 us); smaller ones stay (norm and clipping of 132 MB
// 71 us, past the cache 77).
hipError_t launch_grad_norm(const GradList& l, bool once, double* partial, uint32_t& filled, hipStream_t st) {
  const uint32_t wgs = l.tiles < NORM_WGS ? l.tiles : NORM_WGS;
  const dim3 g(wgs), b(256);
  if (once) hipLaunchKernelGGL((k_grad_norm<true>), g, b, 0, st, l, partial, filled);
  else hipLaunchKernelGGL((k_grad_norm<false>), g, b, 0, st, l, partial, filled);
  if (wgs > filled) filled = wgs;
  return hipGetLastError();
}

hipError_t launch_grad_norm_end(const double* partial, uint32_t filled, float max_norm, float* out, hipStream_t st) {
  hipLaunchKernelGGL(k_grad_norm_end, dim3(1), dim3(256), 0, st, partial, filled, max_norm, out);
  return hipGetLastError();
}

hipError_t launch_grad_scale(const GradList& l, bool once, const float* coef, hipStream_t st) {
  // 2.3 GB of fp32: 834 us with 16384 workgroups, 855 with 2048, 800 with one for each tile, which take 8 us
  // more to find that the coefficient is 1
  const dim3 g(l.tiles < 16384 ? l.tiles : 16384), b(256);
  if (once) hipLaunchKernelGGL((k_grad_scale<true>), g, b, 0, st, l, coef);
  else hipLaunchKernelGGL((k_grad_scale<false>), g, b, 0, st, l, coef);
  return hipGetLastError();
}

hipError_t launch_adamw(const AdamwList& l, bool p_bf16, bool g_bf16, int bits, uint32_t total, hipStream_t st) {
  const dim3 g(total), b(THREADS);
#define ADAMW(P, G)                                                           \
  do {                                                                        \
    if (bits == 8) hipLaunchKernelGGL((k_adamw<P, G, 8>), g, b, 0, st, l);    \
    else hipLaunchKernelGGL((k_adamw<P, G, 32>), g, b, 0, st, l);             \
  } while (0)
  if (p_bf16 && g_bf16) ADAMW(bf16, bf16);
  else if (p_bf16) ADAMW(bf16, float);
  else if (g_bf16) ADAMW(float, bf16);
  else ADAMW(float, float);
#undef ADAMW
  return hipGetLastError();
}
