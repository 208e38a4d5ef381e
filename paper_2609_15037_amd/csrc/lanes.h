// Tokens whose experts (or groups of values) are shared among 8 to 64 lanes of a wave: reductions over these lanes,
// and rows of fp32 or bf16 of any alignment.
#pragma once
#include "common.h"

namespace {

typedef uint16_t u16x4u __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));

// ---- reductions over the LANES (8 to 64) lanes of a token; every lane gets the result. Sixteen lanes are
// one row of the cross-lane data path: neighbours, neighbouring pairs, mirrored halves and rows.
template <int CTRL> __device__ __forceinline__ uint32_t dpp(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xF, 0xF, true);     // every lane has its source
}
template <int CTRL> __device__ __forceinline__ float dpp(float x) {
  return __uint_as_float(dpp<CTRL>(__float_as_uint(x)));
}
template <int CTRL> __device__ __forceinline__ double dpp(double x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  return __builtin_bit_cast(double, (uint64_t)dpp<CTRL>((uint32_t)(b >> 32)) << 32 | dpp<CTRL>((uint32_t)b));
}
// The two values, a lane's and that of the lane DIST (16 or 32) away, in the same order for both lanes.
template <int DIST> __device__ __forceinline__ void rows_apart(uint32_t x, uint32_t& a, uint32_t& b) {
  const auto r = DIST == 16 ? __builtin_amdgcn_permlane16_swap(x, x, false, false)
                            : __builtin_amdgcn_permlane32_swap(x, x, false, false);
  a = r[0];
  b = r[1];
}
template <int DIST> __device__ __forceinline__ void rows_apart(float x, float& a, float& b) {
  uint32_t p, q;
  rows_apart<DIST>(__float_as_uint(x), p, q);
  a = __uint_as_float(p);
  b = __uint_as_float(q);
}
template <int DIST> __device__ __forceinline__ void rows_apart(double x, double& a, double& b) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  uint32_t p0, q0, p1, q1;
  rows_apart<DIST>((uint32_t)u, p0, q0);
  rows_apart<DIST>((uint32_t)(u >> 32), p1, q1);
  a = __builtin_bit_cast(double, (uint64_t)p1 << 32 | p0);
  b = __builtin_bit_cast(double, (uint64_t)q1 << 32 | q0);
}
template <int LANES, typename T, typename F> __device__ __forceinline__ T reduce(T x, F f) {
  x = f(x, dpp<0xB1>(x));     // lane ^ 1
  x = f(x, dpp<0x4E>(x));     // lane ^ 2
  x = f(x, dpp<0x141>(x));    // mirrored within eight lanes
  if (LANES >= 16) x = f(x, dpp<0x140>(x));     // mirrored within sixteen
  T a, b;
  if (LANES >= 32) {
    rows_apart<16>(x, a, b);
    x = f(a, b);
  }
  if (LANES == 64) {
    rows_apart<32>(x, a, b);
    x = f(a, b);
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

// Four experts of a row, from element i: fp32 or bf16, of any alignment; n of them exist, the others are
// -inf and are not written.
__device__ __forceinline__ void load4(const void* row, bool is_bf16, int64_t i, int n, float* x) {
  const float* f = (const float*)row + i;
  const bf16* h = (const bf16*)row + i;
  if (n >= 4 && is_bf16) {
    const u16x4u a = *reinterpret_cast<const u16x4u*>(h);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = __uint_as_float((uint32_t)a[j] << 16);
  } else if (n >= 4) {
    const f32x4u a = *reinterpret_cast<const f32x4u*>(f);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = a[j];
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = j >= n ? -__builtin_inff() : is_bf16 ? bf2f(h[j]) : f[j];
  }
}
__device__ __forceinline__ void store4(void* row, bool is_bf16, int64_t i, int n, const float* x) {
  float* f = (float*)row + i;
  bf16* h = (bf16*)row + i;
  if (n >= 4 && is_bf16) {
    u16x4u a;
#pragma unroll
    for (int j = 0; j < 4; ++j) a[j] = __builtin_bit_cast(uint16_t, f2bf(x[j]));
    *reinterpret_cast<u16x4u*>(h) = a;
  } else if (n >= 4) {
    *reinterpret_cast<f32x4u*>(f) = f32x4u{x[0], x[1], x[2], x[3]};
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < n) {
        if (is_bf16) h[j] = f2bf(x[j]); else f[j] = x[j];
      }
  }
}
__device__ __forceinline__ float load1(const void* row, bool is_bf16, int64_t i) {
  return is_bf16 ? bf2f(((const bf16*)row)[i]) : ((const float*)row)[i];
}

// Expert of a lane's value j: groups of four consecutive experts are dealt to the lanes in turn, so that
// a load of the row is contiguous; a lane's experts ascend with j.
template <int LANES> __device__ __forceinline__ int expert_of(int j, int lane) {
  return (j >> 2) * (4 * LANES) + lane * 4 + (j & 3);
}

}  // namespace
