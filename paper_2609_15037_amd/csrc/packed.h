// Packed sequences of tokens cut into cells (train.h): which sequence a cell belongs to, and its tokens.
#pragma once
#include "lanes.h"
#include "train.h"

namespace {

// First token of sequence s (s = sequences: the end of the last), inside [0, tokens] whatever the offsets are.
__device__ __forceinline__ int64_t first_token(const Packed& q, int64_t s) {
  if (!q.offsets) return s * q.length;
  const int64_t o = q.offsets[s];
  return o < 0 ? 0 : o > q.tokens ? q.tokens : o;
}
// A cell: tokens [begin, end) of a sequence, or none (seq -1: before the first sequence). Tokens [fill0, fill1) and
// [fill2, fill3) are in no sequence and in the cell's tile: a gradient has zeros there.
struct Cell { int64_t seq, tile, begin, end, fill0, fill1, fill2, fill3; };

__device__ __forceinline__ int64_t lane_value(int64_t x, int lane) {
  return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32 |
                   (uint32_t)__builtin_amdgcn_readlane((int)x, lane));
}

// Cell i, with tiles of 2^shift tokens, found by a whole wave: the largest s with s + first_token(s) / tile <= i. Each
// round 64 lanes probe at equal steps, so 4096 sequences take two; the bounds of the sequence found are among the probed.
__device__ __forceinline__ Cell cell_at(const Packed& q, int64_t i, int shift) {
  const int lane = threadIdx.x & 63;
  int64_t lo = -1, hi = q.sequences;            // the key is at most i at lo, and more at hi
  int64_t b = 0, e = first_token(q, hi);        // first tokens of lo and hi
  while (hi - lo > 1) {
    const int64_t step = (hi - lo + 62) / 64, s = lo + 1 + lane * step;
    const int64_t v = s < hi ? first_token(q, s) : 0;
    const bool under = s < hi && s + (v >> shift) <= i;
    const int n = __popcll(__ballot(under));
    const int64_t next = lo + 1 + n * step;
    if (next < hi) {
      hi = next;
      e = lane_value(v, n);
    }
    if (n) {
      lo = next - step;
      b = lane_value(v, n - 1);
    }
  }
  const int64_t tile = i - (lo < 0 ? 0 : lo), t0 = tile << shift, size = (int64_t)1 << shift;
  const int64_t t1 = t0 + size < q.tokens ? t0 + size : q.tokens;
  Cell c = {lo, t0, 0, 0, 0, 0, 0, 0};
  if (lo < 0) {                                 // before the first sequence, which begins at e
    c.fill0 = t0;
    c.fill1 = e < t1 ? e : t1;
    return c;
  }
  if (e < b) e = b;
  c.begin = b > t0 ? b : t0;
  c.end = e < t1 ? e : t1;
  if (lo == 0 && tile == b >> shift) {
    c.fill0 = t0;
    c.fill1 = b;
  }
  if (lo == q.sequences - 1) {
    c.fill2 = e > t0 ? e : t0;
    c.fill3 = t1;
  }
  return c;
}

// Cells of sequence s: [first, last), none of an empty one.
__device__ __forceinline__ void cells_of(const Packed& q, int64_t s, int shift, int64_t& first, int64_t& last) {
  const int64_t b = first_token(q, s), e = first_token(q, s + 1);
  first = s + (b >> shift);
  last = e > b ? s + ((e - 1) >> shift) + 1 : first;
}

// Sums of N values over a workgroup of THREADS, in an order of their own; every thread gets them. part is for one use.
template <int THREADS, int N> __device__ __forceinline__ void group_sums(double (&x)[N], double (*part)[N]) {
  constexpr int WAVES = THREADS / 64;
  static_assert(WAVES <= 16);
#pragma unroll
  for (int k = 0; k < N; ++k) x[k] = sum_of<64>(x[k]);
  if ((threadIdx.x & 63) == 0)
#pragma unroll
    for (int k = 0; k < N; ++k) part[threadIdx.x >> 6][k] = x[k];
  __syncthreads();
  const int i = threadIdx.x & 15;
#pragma unroll
  for (int k = 0; k < N; ++k) x[k] = sum_of<16>(i < WAVES ? part[i][k] : 0.0);
}

}  // namespace

inline int64_t cells_of_all(const Packed& q, int shift) {
  return q.sequences + ((q.tokens + ((int64_t)1 << shift) - 1) >> shift) - 1;
}
