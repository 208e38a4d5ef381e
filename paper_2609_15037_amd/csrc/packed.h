// Packed sequences of tokens cut into cells (train.h): which sequence a cell belongs to, and its tokens.
#pragma once
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
struct Cell { int64_t seq, begin, end, fill0, fill1, fill2, fill3; };

// Cell i, with tiles of `tile` tokens, found by a whole wave: the largest s with s + first_token(s) / tile <= i.
// Each round 64 lanes probe at equal steps, so 4096 sequences take two.
__device__ __forceinline__ Cell cell_at(const Packed& q, int64_t i, int tile) {
  const int lane = threadIdx.x & 63;
  int64_t lo = -1, hi = q.sequences;            // the key is at most i at lo, and more at hi
  while (hi - lo > 1) {
    const int64_t step = (hi - lo + 62) / 64, s = lo + 1 + lane * step;
    const bool under = s < hi && s + first_token(q, s) / tile <= i;
    const int n = __popcll(__ballot(under));
    const int64_t next = lo + 1 + n * step;
    if (n) lo = next - step;
    if (next < hi) hi = next;
  }
  // the same in every lane: scalar registers
  const int64_t s = (int64_t)__builtin_amdgcn_readfirstlane((int)lo);
  const int64_t at = i - (s < 0 ? 0 : s), t0 = at * tile;
  const int64_t t1 = t0 + tile < q.tokens ? t0 + tile : q.tokens;
  Cell c = {s, 0, 0, 0, 0, 0, 0};
  const int64_t b = first_token(q, s < 0 ? 0 : s);
  if (s < 0) {
    c.fill0 = t0;
    c.fill1 = b < t1 ? b : t1;
    return c;
  }
  int64_t e = first_token(q, s + 1);
  if (e < b) e = b;
  c.begin = b > t0 ? b : t0;
  c.end = e < t1 ? e : t1;
  if (s == 0 && at == b / tile) {
    c.fill0 = t0;
    c.fill1 = b;
  }
  if (s == q.sequences - 1) {
    c.fill2 = e > t0 ? e : t0;
    c.fill3 = t1;
  }
  return c;
}

// Cells of sequence s: [first, last), none of an empty one.
__device__ __forceinline__ void cells_of(const Packed& q, int64_t s, int tile, int64_t& first, int64_t& last) {
  const int64_t b = first_token(q, s), e = first_token(q, s + 1);
  first = s + b / tile;
  last = e > b ? s + (e - 1) / tile + 1 : first;
}

// Sum over a workgroup of THREADS, in an order of its own; every thread gets it.
template <int THREADS> __device__ __forceinline__ double group_sum(double x, double* part) {
  x = wave_sum_d(x);
  __syncthreads();              // the last sum has been read
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
  __syncthreads();
  double sum = 0;
#pragma unroll
  for (int i = 0; i < THREADS / 64; ++i) sum += part[i];
  return sum;
}

}  // namespace

inline int64_t cells_of_all(const Packed& q, int tile) { return q.sequences + (q.tokens + tile - 1) / tile - 1; }
