// Losses over packed sequences of tokens' log-probabilities: pairs of responses, and a clipped policy. Both sum
// over a sequence's tokens, so their forward pass is two steps: a wave sums a cell (the tokens of one sequence in one
// tile) in 64 bits, and a workgroup of several the neighbouring cells of one sequence, then one workgroup adds up each
// sequence's sums, in order, and forms the loss: no atomics, so the same bits each time. Few cells take both steps in one
// launch: 4 pairs of 1000 tokens 7.7 us, of which half is the chain of a search, a load, two sums over the workgroup and the
// loss itself. Their gradients are one launch, a wave for each cell.
// Tiles of 512 tokens: of 256, twice the sums to be gathered in the last step; of 1024, too few waves, both slower at 2 M
// tokens; up to 65536 tokens 256, for the waves. Times below are of 2 M tokens in 2048 (pairs) and 1024 (policy) sequences, in a
// captured graph of many such calls; in a trace of whole steps a kernel takes up to 1.5 us more.
#include "packed.h"

namespace {

constexpr int END_THREADS = 1024;           // of both steps
constexpr int ONE = 8;          // a tile of which a lane takes four tokens, as a power of 2
constexpr int FEW = END_THREADS / 64;   // cells that one launch takes
constexpr int GROUP = 8;                // else cells of a workgroup

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32u __attribute__((aligned(1)));
typedef double f64x2u __attribute__((ext_vector_type(2), aligned(8)));
// A cell's tokens counted from its tile's first: its own [begin, end), those it clears, and how many there are at all.
struct Span {
  int64_t seq, tile;
  int begin, end, fill0, fill1, fill2, fill3, left;
};
template <int SHIFT> __device__ __forceinline__ Span span_of(const Packed& q, int64_t i) {
  const Cell c = cell_at(q, i, SHIFT);
  auto from_tile = [&](int64_t t) {
    const int64_t d = t - c.tile;
    return d < 0 ? 0 : d > 1 << SHIFT ? 1 << SHIFT : (int)d;
  };
  return Span{c.seq, c.tile, from_tile(c.begin), from_tile(c.end), from_tile(c.fill0), from_tile(c.fill1), from_tile(c.fill2),
              from_tile(c.fill3), from_tile(q.tokens)};
}
__device__ __forceinline__ int within(int r, int from, int to) { return r >= from && r < to; }
// Four tokens from the r-th of a tile, in one access. Only in the last tile (WHOLE: not that one) may some not exist: what
// asks for that, lane by lane and load by load, is kept out of all other cells.
template <bool WHOLE> __device__ __forceinline__ void load4(const float* q, const Span& c, int r, float (&x)[4]) {
  q += c.tile;
  if (WHOLE || r + 4 <= c.left) {
    const f32x4u a = *reinterpret_cast<const f32x4u*>(q + r);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = a[j];
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = r + j < c.left ? q[r + j] : 0.f;
  }
}
__device__ __forceinline__ void zero4(float (&x)[4]) { x[0] = x[1] = x[2] = x[3] = 0.f; }
// Which of four tokens are in the cell: bit j for token r + j. And of these the ones that count: the mask's bytes are asked
// for with the tokens' values, not before them.
__device__ __forceinline__ int inside4(const Span& c, int r) {
  int in = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) in |= within(r + j, c.begin, c.end) << j;
  return in;
}
template <bool WHOLE> __device__ __forceinline__ uint32_t mask4(const Packed& q, const Span& c, int r) {
  if (!q.mask) return 0x01010101u;
  const uint8_t* m = q.mask + c.tile;
  if (WHOLE || r + 4 <= c.left) return *reinterpret_cast<const u32u*>(m + r);
  uint32_t x = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (r + j < c.left) x |= (uint32_t)m[r + j] << (8 * j);
  return x;
}
__device__ __forceinline__ int live4(int in, uint32_t mask) {
#pragma unroll
  for (int j = 0; j < 4; ++j) in &= ~((mask >> (8 * j) & 0xFF ? 0 : 1) << j);
  return in;
}
// Writes four tokens' gradients, the cell's and the zeros it has to clear.
__device__ __forceinline__ void store4(float* q, const Span& c, int r, const float (&x)[4]) {
  const int own = inside4(c, r);
  int clear = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) clear |= (within(r + j, c.fill0, c.fill1) | within(r + j, c.fill2, c.fill3)) << j;
  q += c.tile;
  if ((own | clear) == 15) {
    f32x4u a;
#pragma unroll
    for (int j = 0; j < 4; ++j) a[j] = own >> j & 1 ? x[j] : 0.f;
    *reinterpret_cast<f32x4u*>(q + r) = a;
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if ((own | clear) >> j & 1) q[r + j] = own >> j & 1 ? x[j] : 0.f;
  }
}

// Lanes of a sequence in the second step: as many as there are for each.
__device__ __forceinline__ int lanes_of_each(int64_t groups) {
  int lanes = 64;
  while (lanes > 1 && groups * lanes > END_THREADS) lanes >>= 1;
  return lanes;
}
// Sum over `lanes` neighbouring lanes.
__device__ __forceinline__ double over_lanes(double x, int lanes) {
  for (int o = lanes >> 1; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}

// Cells' sums of a workgroup, and whose they are.
template <int N, int W> struct CellSums {
  double sum[W][N];
  int64_t seq[W];
};
// What the workgroup's cells, from cell i0 on, leave: at the first cell of each sequence the sum of its cells among them, at the
// others 0, which only offsets that fall lead to.
template <int N, int W> __device__ __forceinline__ void leave(const CellSums<N, W>& s, int64_t i0, int64_t cells, double* sums) {
  __syncthreads();
  const int w = threadIdx.x / N, k = threadIdx.x % N;
  if (w >= W || i0 + w >= cells) return;
  double x = 0;
  if (w == 0 || s.seq[w] != s.seq[w - 1])
    for (int v = w; v < W && i0 + v < cells && s.seq[v] == s.seq[w]; ++v) x += s.sum[v][k];
  sums[(i0 + w) * N + k] = x;
}
// Adds up the sums of K sequences, of cells [first, last), by `lanes` lanes: those at its first cell and at each workgroup's
// first. The loads of several turns are on their way together, 16 bytes each, and only for sums that there are: one workgroup's
// scattered addresses are what this costs.
template <int W, int K, int N> __device__ __forceinline__ void gather(const double* sums, const int64_t (&first)[K],
                                                               const int64_t (&last)[K], int lane, int lanes, double (&own)[K][N]) {
  constexpr int TURNS = 4 / K;
  int64_t group[K], n[K], most = 0;
#pragma unroll
  for (int s = 0; s < K; ++s) {
    group[s] = first[s] / W;
    n[s] = last[s] > first[s] ? (last[s] - 1) / W - group[s] + 1 : 0;
    most = n[s] > most ? n[s] : most;
#pragma unroll
    for (int k = 0; k < N; ++k) own[s][k] = 0;
  }
  for (int64_t j = lane; j < most; j += TURNS * lanes) {
    f64x2u x[K][TURNS][N / 2];
#pragma unroll
    for (int s = 0; s < K; ++s)
#pragma unroll
      for (int u = 0; u < TURNS; ++u) {
        const int64_t at = j + u * lanes;
        const f64x2u* q = reinterpret_cast<const f64x2u*>(sums + N * (at ? (group[s] + at) * W : first[s]));
#pragma unroll
        for (int k = 0; k < N / 2; ++k) x[s][u][k] = f64x2u{0, 0};
        if (at < n[s])
#pragma unroll
          for (int k = 0; k < N / 2; ++k) x[s][u][k] = q[k];
      }
#pragma unroll
    for (int s = 0; s < K; ++s)
#pragma unroll
      for (int u = 0; u < TURNS; ++u)
#pragma unroll
        for (int k = 0; k < N; ++k) own[s][k] += x[s][u][k / 2][k % 2];
  }
}

// ---------------------------------------------------------------- pairs of responses
constexpr int PREFERENCE_SUMS = 2;      // of logp - ref, and the number of tokens

// A token that does not count has zeros for its inputs, and so for its terms; here and below.
template <int SHIFT, bool WHOLE>
__device__ __forceinline__ void preference_sums(const PreferenceParams& p, const Span& c, double& sum, int& count) {
  constexpr int TURNS = 1 << (SHIFT - ONE);
  int in[TURNS];
  uint32_t mask[TURNS];
  float x[TURNS][4], y[TURNS][4];
#pragma unroll
  for (int v = 0; v < TURNS; ++v) {     // all of a lane's loads are on their way before the first is used
    const int r = 4 * (threadIdx.x & 63) + 256 * v;
    in[v] = inside4(c, r);
    if (!in[v]) continue;
    mask[v] = mask4<WHOLE>(p.q, c, r);
    load4<WHOLE>(p.logp, c, r, x[v]);
    if (p.ref) load4<WHOLE>(p.ref, c, r, y[v]); else zero4(y[v]);
  }
#pragma unroll
  for (int v = 0; v < TURNS; ++v) {
    if (!in[v]) continue;
    const int on = live4(in[v], mask[v]);
    count += __popc(on);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool live = on >> j & 1;
      sum += (double)(live ? x[v][j] : 0.f) - (double)(live ? y[v][j] : 0.f);
    }
  }
}
template <int SHIFT, int W>
__device__ __forceinline__ void preference_cell(const PreferenceParams& p, int64_t i, CellSums<PREFERENCE_SUMS, W>& s) {
  const Span c = span_of<SHIFT>(p.q, i);
  double sum = 0;
  int count = 0;
  if (c.left >= 1 << SHIFT) preference_sums<SHIFT, true>(p, c, sum, count);
  else preference_sums<SHIFT, false>(p, c, sum, count);
  sum = sum_of<64>(sum);
  const double n = sum_of<64>((double)count);
  if ((threadIdx.x & 63) == 0) {
    const int w = threadIdx.x >> 6;
    s.sum[w][0] = sum;
    s.sum[w][1] = n;
    s.seq[w] = c.seq;
  }
}

template <int SHIFT, int W> __device__ __forceinline__ void preference_end(const PreferenceParams& p, const double* sums) {
  __shared__ double part[END_THREADS / 64][4];
  const int64_t pairs = p.q.sequences / 2;
  const int lanes = lanes_of_each(pairs), lane = threadIdx.x & (lanes - 1);
  double all[4] = {};           // loss, pairs ahead, margin, pairs with a token
  for (int64_t pair = threadIdx.x / lanes; pair < pairs; pair += END_THREADS / lanes) {
    int64_t first[2], last[2];
    double own[2][PREFERENCE_SUMS], d[2], n[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) cells_of(p.q, 2 * pair + k, SHIFT, first[k], last[k]);
    gather<W>(sums, first, last, lane, lanes, own);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      d[k] = over_lanes(own[k][0], lanes);
      n[k] = over_lanes(own[k][1], lanes);
    }
    if (lane == 0) {
      const double per0 = p.average && n[0] > 0 ? 1 / n[0] : 1, per1 = p.average && n[1] > 0 ? 1 / n[1] : 1;
      d[0] *= per0;
      d[1] *= per1;
      const double h = d[0] - d[1], z = p.beta * h - p.margin;
      double l, dl;             // the loss and its derivative by h
      if (p.kind == 0) {
        // log(1 + e^-z) = max(-z, 0) + log(1 + u), u = e^-|z|, and the same of z; 1 / (1 + e^z) from u too
        const double u = exp(-fabs(z)), log = log1p(u), y = 1 / (1 + u);
        l = (p.smoothing != 1 ? (1 - p.smoothing) * (fmax(-z, 0.0) + log) : 0) +
            (p.smoothing != 0 ? p.smoothing * (fmax(z, 0.0) + log) : 0);
        dl = p.beta * (p.smoothing - (z > 0 ? u * y : y));
      } else if (p.kind == 1) {
        l = z < 1 ? 1 - z : z != z ? z : 0;
        dl = z < 1 ? -p.beta : 0;
      } else {
        const double off = h - 0.5 / p.beta;
        l = off * off;
        dl = 2 * off;
      }
      p.rewards[2 * pair] = (float)(p.beta * d[0]);
      p.rewards[2 * pair + 1] = (float)(p.beta * d[1]);
      const bool on = n[0] + n[1] > 0;
      p.slope[2 * pair] = on ? (float)(dl * per0) : 0.f;
      p.slope[2 * pair + 1] = on ? (float)(-dl * per1) : 0.f;
      if (on) {
        all[0] += l;
        all[1] += h > 0 ? 1 : 0;
        all[2] += p.beta * h;
        all[3] += 1;
      }
    }
  }
  group_sums<END_THREADS>(all, part);
  if (threadIdx.x == 0) {
    const double share = all[3] > 0 ? 1 / all[3] : 0;
#pragma unroll
    for (int k = 0; k < 3; ++k) p.out[k] = (float)(all[k] * share);
    if (p.loss) *p.loss = (float)(all[0] * share);
    p.slope[p.q.sequences] = (float)share;
  }
}

// 8 us for 10 MB: one set of waves, each with a search of two rounds, its loads and the sums over its lanes one after another.
template <int SHIFT> __global__ __launch_bounds__(64 * GROUP) void k_preference_cells(PreferenceParams p, int64_t cells) {
  __shared__ CellSums<PREFERENCE_SUMS, GROUP> s;
  const int64_t i0 = (int64_t)blockIdx.x * GROUP, i = i0 + (threadIdx.x >> 6);
  if (i < cells) preference_cell<SHIFT>(p, i, s);
  leave(s, i0, cells, p.sums);
}
// 6.8 us: one workgroup's latencies (offsets, sums, an exponential and a logarithm in 64 bits, the sums over the pairs).
template <int SHIFT> __global__ __launch_bounds__(END_THREADS) void k_preference_end(PreferenceParams p) {
  preference_end<SHIFT, GROUP>(p, p.sums);
}
// All cells in one workgroup.
__global__ __launch_bounds__(END_THREADS) void k_preference_small(PreferenceParams p, int64_t cells) {
  __shared__ CellSums<PREFERENCE_SUMS, FEW> s;
  __shared__ double sums[FEW * PREFERENCE_SUMS];
  const int64_t i = threadIdx.x >> 6;
  if (i < cells) preference_cell<ONE>(p, i, s);
  leave(s, 0, cells, sums);
  __syncthreads();
  preference_end<ONE, FEW>(p, sums);
}

// A token's gradient is its sequence's slope: written once, nothing but the mask is read for it. 8.0 us where its 10 MB alone
// would take 2: with two sequences of equal rows it takes 5.8 (a launch, then search, mask and store one after another, once for
// each wave), with 2048 of them 7.0 (a round of the search more), with offsets of the same rows 7.7 (their loads), of uneven
// ones 8.0.
__global__ __launch_bounds__(256) void k_preference_backward(Packed q, const float* __restrict__ slope,
                                                             const float* __restrict__ grad_loss, float* __restrict__ grad,
                                                             int64_t cells) {
  const int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (i >= cells) return;
  const float all = slope[q.sequences] * *grad_loss;
  const Span c = span_of<ONE>(q, i);
  const int r = 4 * (threadIdx.x & 63);
  const float g = c.seq >= 0 ? slope[c.seq] * all : 0.f;
  const int in = inside4(c, r), on = live4(in, !in ? 0 : c.left >= 1 << ONE ? mask4<true>(q, c, r) : mask4<false>(q, c, r));
  float x[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = on >> j & 1 ? g : 0.f;
  store4(grad, c, r, x);
}

// ---------------------------------------------------------------- clipped policy
// e^q - q - 1, of q and e = e^q. The terms cancel near 0: there a series, q^2 (1/2 + q/6 + ..), good to 1e-9 of
// its value at |q| = 1/2.
__device__ __forceinline__ float exp_excess(float q, float e) {
  float s = 1.f / 3628800.f;
  s = fmaf(s, q, 1.f / 362880.f);
  s = fmaf(s, q, 1.f / 40320.f);
  s = fmaf(s, q, 1.f / 5040.f);
  s = fmaf(s, q, 1.f / 720.f);
  s = fmaf(s, q, 1.f / 120.f);
  s = fmaf(s, q, 1.f / 24.f);
  s = fmaf(s, q, 1.f / 6.f);
  s = fmaf(s, q, 0.5f);
  return fabsf(q) < 0.5f ? s * q * q : e - 1.f - q;
}
// e^q by the hardware's 2^x: the product's rounding, and what log2 e has beyond fp32, are put back to first order.
__device__ __forceinline__ float exp_of(float q) {
  constexpr float A = 1.44269504088896340736f, B = (float)(1.44269504088896340736 - (double)A), LN2 = 0.693147180559945309f;
  const float t = q * A, e = __builtin_amdgcn_exp2f(t), r = fmaf(q, B, fmaf(q, A, -t));
  return fabsf(t) < 128.f ? fmaf(e, r * LN2, e) : e;
}

// A token's terms. d and the comparison with the bounds are 64 bits: a ratio next to a bound falls on the side
// that the difference of the two fp32 log-probabilities says. KL: the kind of the distance, or NO_REF.
constexpr int NO_REF = -1;
struct Token { float gain, slope, kl, dkl, excess; bool clipped; };
template <int KL> __device__ __forceinline__ Token policy_token(const PolicyParams& p, float logp, float old, float ref, float a) {
  Token t;
  const double d = p.old ? (double)logp - (double)old : 0.0;
  const float df = (float)d, ratio = exp_of(df);
  const bool up = d > p.high && a > 0, down = d < p.low && a < 0;
  t.clipped = up || down;
  const bool none = a == 0 && df == df;         // an advantage of 0 has no part where the ratio overflows either; a NaN has
  t.gain = none ? 0.f : (up ? p.at_high : down ? p.at_low : ratio) * a;
  t.slope = t.clipped || none ? 0.f : -ratio * a;
  t.excess = exp_excess(df, ratio);
  const float q = KL == NO_REF ? 0.f : (float)((double)ref - (double)logp), e = KL == 0 ? exp_of(q) : 0.f;
  const float far = KL == 0 ? exp_excess(q, e) : 0.f;
  t.kl = KL == 0 ? far : KL == 1 ? -q : 0.5f * q * q;
  t.dkl = KL == 0 ? -(fabsf(q) < 0.5f ? q + far : e - 1.f) : KL == 1 ? 1.f : -q;
  return t;
}
struct Four { float logp[4], old[4], ref[4], a[4]; };
template <int KL, bool WHOLE>
__device__ __forceinline__ void fetch(const PolicyParams& p, const Span& c, int r, float each, Four& x) {
  load4<WHOLE>(p.logp, c, r, x.logp);
  if (p.old) load4<WHOLE>(p.old, c, r, x.old); else zero4(x.old);
  if (KL != NO_REF) load4<WHOLE>(p.ref, c, r, x.ref); else zero4(x.ref);
  if (!p.sequence_advantages) load4<WHOLE>(p.advantages, c, r, x.a);
  else
#pragma unroll
    for (int j = 0; j < 4; ++j) x.a[j] = each;
}
template <int KL, int SHIFT, bool WHOLE>
__device__ __forceinline__ void policy_sums(const PolicyParams& p, const Span& c, double (&sum)[POLICY_SUMS]) {
  constexpr int TURNS = 1 << (SHIFT - ONE);
  const float each = p.sequence_advantages && c.begin < c.end ? p.advantages[c.seq] : 0.f;    // there may be none of no tokens
  int count = 0, clipped = 0;
  Four x[TURNS];
  float entropy[TURNS][4];
  uint32_t mask[TURNS];
  int in[TURNS];
#pragma unroll
  for (int v = 0; v < TURNS; ++v) {     // all of a lane's loads are on their way before the first is used
    const int r = 4 * (threadIdx.x & 63) + 256 * v;
    in[v] = inside4(c, r);
    if (!in[v]) continue;
    mask[v] = mask4<WHOLE>(p.q, c, r);
    fetch<KL, WHOLE>(p, c, r, each, x[v]);
    if (p.entropy) load4<WHOLE>(p.entropy, c, r, entropy[v]); else zero4(entropy[v]);
  }
#pragma unroll
  for (int v = 0; v < TURNS; ++v) {
    if (!in[v]) continue;
    const int on = live4(in[v], mask[v]);
    count += __popc(on);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool live = on >> j & 1;
      auto of = [&](const float (&y)[4]) { return live ? y[j] : 0.f; };
      const Token y = policy_token<KL>(p, of(x[v].logp), of(x[v].old), of(x[v].ref), of(x[v].a));
      sum[1] -= (double)y.gain;
      if (KL != NO_REF) sum[2] += (double)y.kl;
      sum[3] += (double)of(entropy[v]);
      clipped += y.clipped;
      sum[5] += (double)y.excess;
    }
  }
  sum[0] = count;
  sum[4] = clipped;
}
template <int KL, int SHIFT, int W>
__device__ __forceinline__ void policy_cell(const PolicyParams& p, int64_t i, CellSums<POLICY_SUMS, W>& s) {
  const Span c = span_of<SHIFT>(p.q, i);
  double sum[POLICY_SUMS] = {};
  if (c.left >= 1 << SHIFT) policy_sums<KL, SHIFT, true>(p, c, sum); else policy_sums<KL, SHIFT, false>(p, c, sum);
#pragma unroll
  for (int k = 0; k < POLICY_SUMS; ++k) sum[k] = sum_of<64>(sum[k]);
  if ((threadIdx.x & 63) == 0) {
    const int w = threadIdx.x >> 6;
#pragma unroll
    for (int k = 0; k < POLICY_SUMS; ++k) s.sum[w][k] = sum[k];
    s.seq[w] = c.seq;
  }
}

template <int SHIFT, int W> __device__ __forceinline__ void policy_end(const PolicyParams& p, const double* sums) {
  constexpr int N = POLICY_SUMS + 1;
  __shared__ double part[END_THREADS / 64][N];
  const int64_t S = p.q.sequences;
  const int lanes = lanes_of_each(S), lane = threadIdx.x & (lanes - 1);
  double all[N] = {};           // the cells' sums, by sequence over its tokens, and the sequences with tokens
  for (int64_t s = threadIdx.x / lanes; s < S; s += END_THREADS / lanes) {
    int64_t first[1], last[1];
    cells_of(p.q, s, SHIFT, first[0], last[0]);
    double sum[1][POLICY_SUMS];
    gather<W>(sums, first, last, lane, lanes, sum);
    const double (&own)[POLICY_SUMS] = sum[0];
    // a sum over the lanes waits for the others' sums below, except where it divides them
    const double n = over_lanes(own[0], lanes), per = !p.by_sequence ? 1 : n > 0 ? 1 / n : 0;
    all[0] += own[0];
#pragma unroll
    for (int k = 1; k < POLICY_SUMS; ++k) all[k] += own[k] * per;
    if (lane == 0) {
      all[POLICY_SUMS] += n > 0 ? 1 : 0;
      p.weight[s] = n > 0 ? (float)per : 0.f;
    }
  }
  group_sums<END_THREADS>(all, part);
  if (threadIdx.x == 0) {
    const double over = p.divisor > 0 ? p.divisor : p.by_sequence ? all[POLICY_SUMS] : all[0], share = over > 0 ? 1 / over : 0;
    const double policy = all[1] * share, kl = all[2] * share, entropy = all[3] * share;
    // a coefficient of 0 leaves its term out, also where that is not finite
    const float loss = (float)(policy + (p.ref && p.kl_coef != 0 ? p.kl_coef * kl : 0) -
                               (p.entropy && p.entropy_coef != 0 ? p.entropy_coef * entropy : 0));
    p.out[0] = loss;
    if (p.loss) *p.loss = loss;
    p.out[1] = (float)policy;
    p.out[2] = (float)kl;
    p.out[3] = (float)entropy;
    p.out[4] = (float)(all[4] * share);
    p.out[5] = (float)(all[5] * share);
    p.weight[S] = (float)share;
  }
}

// 15.5 us for 42 MB, 2.7 TB/s: all waves are resident, and their phases follow one another: the search, the loads, some 100
// vector instructions a token, the sums; of its 10 us a wave waits 6.4 for memory and the workgroup. A kernel for each kind of
// distance: as branches of each token, though alike for all, 16.2 (backward 13.4 for 12.3).
template <int SHIFT, int KL> __global__ __launch_bounds__(64 * GROUP) void k_policy_cells(PolicyParams p, int64_t cells) {
  __shared__ CellSums<POLICY_SUMS, GROUP> s;
  const int64_t i0 = (int64_t)blockIdx.x * GROUP, i = i0 + (threadIdx.x >> 6);
  if (i < cells) policy_cell<KL, SHIFT>(p, i, s);
  leave(s, i0, cells, p.sums);
}
// 5.7 us, one workgroup's latencies; 7 with loads of 8 bytes, also of sums that are not there.
template <int SHIFT> __global__ __launch_bounds__(END_THREADS) void k_policy_end(PolicyParams p) { policy_end<SHIFT, GROUP>(p, p.sums); }
// All cells in one workgroup.
template <int KL> __global__ __launch_bounds__(END_THREADS) void k_policy_small(PolicyParams p, int64_t cells) {
  __shared__ CellSums<POLICY_SUMS, FEW> s;
  __shared__ double sums[FEW * POLICY_SUMS];
  const int64_t i = threadIdx.x >> 6;
  if (i < cells) policy_cell<KL, ONE>(p, i, s);
  leave(s, 0, cells, sums);
  __syncthreads();
  policy_end<ONE, FEW>(p, sums);
}

// The terms again (their inputs are half the bytes of what they would be stored as), the derivative in fp32, rounded once a
// product. 12 us for 50 MB, 4.1 TB/s; tiles of 512 tokens took as long.
template <int KL> __global__ __launch_bounds__(256) void k_policy_backward(PolicyParams p, int64_t cells) {
  const int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (i >= cells) return;
  const float all = p.weight[p.q.sequences] * *p.grad_loss;
  const Span c = span_of<ONE>(p.q, i);
  const int r = 4 * (threadIdx.x & 63);
  const float each = p.sequence_advantages && c.begin < c.end ? p.advantages[c.seq] : 0.f;
  const float w = c.seq >= 0 ? p.weight[c.seq] * all : 0.f;
  const float kl_coef = (float)p.kl_coef, bonus = -(float)p.entropy_coef * w;
  const int in = inside4(c, r);
  float g[4] = {}, h[4] = {};
  if (in) {
    Four x;
    uint32_t mask;
    if (c.left >= 1 << ONE) {
      mask = mask4<true>(p.q, c, r);
      fetch<KL, true>(p, c, r, each, x);
    } else {
      mask = mask4<false>(p.q, c, r);
      fetch<KL, false>(p, c, r, each, x);
    }
    const int on = live4(in, mask);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const Token y = policy_token<KL>(p, x.logp[j], x.old[j], x.ref[j], x.a[j]);
      const bool live = on >> j & 1;
      g[j] = live ? (y.slope + (KL != NO_REF ? kl_coef * y.dkl : 0.f)) * w : 0.f;
      h[j] = live ? bonus : 0.f;
    }
  }
  store4(p.grad_logp, c, r, g);
  if (p.grad_entropy) store4(p.grad_entropy, c, r, h);
}

}  // namespace

#define ON_CELLS(kernel, st, ...) \
  hipLaunchKernelGGL(kernel, dim3((uint32_t)((cells + 3) / 4)), dim3(256), 0, st, __VA_ARGS__, cells)
// Both steps of a forward pass over cells of 2^SHIFT tokens: two launches, or one where there are few cells.
#define FORWARD(SMALL, CELLS, END, SHIFT)                                                                   \
  do {                                                                                                      \
    const int64_t cells = cells_of_all(p.q, SHIFT);                                                         \
    if (SHIFT == ONE && cells <= FEW) {                                                                     \
      SMALL(dim3(1), dim3(END_THREADS), 0, st, p, cells);                                                   \
      return hipGetLastError();                                                                             \
    }                                                                                                       \
    CELLS(SHIFT, dim3((uint32_t)((cells + GROUP - 1) / GROUP)), dim3(64 * GROUP), 0, st, p, cells);         \
    const hipError_t e = hipGetLastError();                                                                 \
    if (e != hipSuccess) return e;                                                                          \
    hipLaunchKernelGGL(END<SHIFT>, dim3(1), dim3(END_THREADS), 0, st, p);                                   \
    return hipGetLastError();                                                                               \
  } while (0)
#define PREFERENCE_SMALL(...) hipLaunchKernelGGL(k_preference_small, __VA_ARGS__)
#define PREFERENCE_CELLS(SHIFT, ...) hipLaunchKernelGGL(k_preference_cells<SHIFT>, __VA_ARGS__)
// A kernel for each kind of distance: decided for each token, even alike for all, the branches were a third of the work.
#define POLICY_SMALL(...)                                                                \
  do {                                                                                   \
    if (!p.ref) hipLaunchKernelGGL(k_policy_small<NO_REF>, __VA_ARGS__);                 \
    else if (p.kl == 0) hipLaunchKernelGGL(k_policy_small<0>, __VA_ARGS__);              \
    else if (p.kl == 1) hipLaunchKernelGGL(k_policy_small<1>, __VA_ARGS__);              \
    else hipLaunchKernelGGL(k_policy_small<2>, __VA_ARGS__);                             \
  } while (0)
#define POLICY_CELLS(SHIFT, ...)                                                         \
  do {                                                                                   \
    if (!p.ref) hipLaunchKernelGGL((k_policy_cells<SHIFT, NO_REF>), __VA_ARGS__);        \
    else if (p.kl == 0) hipLaunchKernelGGL((k_policy_cells<SHIFT, 0>), __VA_ARGS__);     \
    else if (p.kl == 1) hipLaunchKernelGGL((k_policy_cells<SHIFT, 1>), __VA_ARGS__);     \
    else hipLaunchKernelGGL((k_policy_cells<SHIFT, 2>), __VA_ARGS__);                    \
  } while (0)

hipError_t launch_preference(const PreferenceParams& p, hipStream_t st) {
  if (p.q.tokens > LOSS_FEW_TOKENS)
    FORWARD(PREFERENCE_SMALL, PREFERENCE_CELLS, k_preference_end, LOSS_CELL_SHIFT);
  else
    FORWARD(PREFERENCE_SMALL, PREFERENCE_CELLS, k_preference_end, ONE);
}
hipError_t launch_preference_backward(const Packed& q, const float* slope, const float* grad_loss, float* grad, hipStream_t st) {
  const int64_t cells = cells_of_all(q, ONE);
  ON_CELLS(k_preference_backward, st, q, slope, grad_loss, grad);
  return hipGetLastError();
}
hipError_t launch_policy(const PolicyParams& p, hipStream_t st) {
  if (p.q.tokens > LOSS_FEW_TOKENS)
    FORWARD(POLICY_SMALL, POLICY_CELLS, k_policy_end, LOSS_CELL_SHIFT);
  else
    FORWARD(POLICY_SMALL, POLICY_CELLS, k_policy_end, ONE);
}
hipError_t launch_policy_backward(const PolicyParams& p, hipStream_t st) {
  const int64_t cells = cells_of_all(p.q, ONE);
  if (!p.ref || (float)p.kl_coef == 0) ON_CELLS(k_policy_backward<NO_REF>, st, p);
  else if (p.kl == 0) ON_CELLS(k_policy_backward<0>, st, p);
  else if (p.kl == 1) ON_CELLS(k_policy_backward<1>, st, p);
  else ON_CELLS(k_policy_backward<2>, st, p);
  return hipGetLastError();
}
