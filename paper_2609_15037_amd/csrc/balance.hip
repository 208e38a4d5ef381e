// Load-balancing loss of expert routing, its counts and its gradient. Forward: a workgroup sums the scores and counts
// the experts of a cell's tokens, a second launch adds up each sequence's cells and forms its loss, and where there
// are several sequences a third one their mean; a few tokens of one sequence take one launch. Backward: the scores
// again, and a row of the gradient for each token.
#include <float.h>

#include "packed.h"

namespace {

constexpr int FORWARD_THREADS = 1024, BACKWARD_THREADS = 256, END_THREADS = 1024;

// What a cell leaves in the workspace, experts padded to an even number: its scores' sums, its counts, z and its tokens.
struct CellSums {
  char* at;
  int E;
  __device__ __forceinline__ int64_t size() const { return 8 * (int64_t)((E + 1) & ~1) + 16; }
  __device__ __forceinline__ double* about(int64_t i) const { return (double*)(at + i * size()); }       // z, tokens
  __device__ __forceinline__ float* scores(int64_t i) const { return (float*)(about(i) + 2); }
  __device__ __forceinline__ uint32_t* counts(int64_t i) const { return (uint32_t*)(scores(i) + ((E + 1) & ~1)); }
};
// What a sequence leaves: its balance, whether it has tokens, z, its tokens; and its experts' scores, where the cells are
// added up by columns first.
__device__ __forceinline__ double* about_sequences(const BalanceParams& p, int64_t cells) {
  return (double*)((char*)p.workspace + cells * CellSums{nullptr, p.E}.size());
}
__device__ __forceinline__ double* scores_of_sequences(const BalanceParams& p, int64_t cells) {
  return about_sequences(p, cells) + 4 * p.q.sequences;
}

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896340736f); }

// A token's scores s[j] y, as parts of their sum (of a sigmoid too, which so exist where they underflow); for the gradient
// w = 1 - sigmoid; with z the softmax and the logits' log-sum-exp. False where it has no scores.
template <int LANES, int V, bool SIGMOID, bool Z, bool BACKWARD>
__device__ __forceinline__ bool token_scores(const float (&l)[V], float (&s)[V], float& y, float (&w)[V], float (&soft)[V],
                                             float& lse) {
  float top = 0, sum = 0;
  auto find_top = [&] {
    top = l[0];
#pragma unroll
    for (int j = 1; j < V; ++j) top = fmaxf(top, l[j]);
    top = max_of<LANES>(top);
  };
  if (Z || !SIGMOID) find_top();
  lse = 0;
  if (!SIGMOID) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      s[j] = exp_of(l[j] - top);
      sum += s[j];
    }
    sum = sum_of<LANES>(sum);
    y = __builtin_amdgcn_rcpf(sum);
    if (Z) lse = top + logf(sum);
    return sum > 0;                     // not NaN: a row of -infinity, one with a NaN or +infinity
  }
#pragma unroll
  for (int j = 0; j < V; ++j) {         // 1 / (1 + q), and q / (1 + q); q may overflow where the score is 0
    const float q = exp_of(-l[j]);
    s[j] = __builtin_amdgcn_rcpf(1.f + q);
    if (BACKWARD) w[j] = fminf(q, 0x1p126f) * s[j];
    sum += s[j];
  }
  sum = sum_of<LANES>(sum);
  if (!(sum > 0x1p-30f)) {              // small ones, or none: their quotients from the logits less the largest
    if (!Z) find_top();
    const float shift = fminf(top, 0.f);
    sum = 0;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float q = exp_of(-fabsf(l[j])), r = __builtin_amdgcn_rcpf(1.f + q);
      s[j] = exp_of(fminf(l[j], 0.f) - shift) * r;
      if (BACKWARD) w[j] = l[j] < 0 ? r : q * r;
      sum += s[j];
    }
    sum = sum_of<LANES>(sum);
  }
  y = __builtin_amdgcn_rcpf(sum);
  if (Z) {
    float total = 0;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      soft[j] = exp_of(l[j] - top);
      total += soft[j];
    }
    total = sum_of<LANES>(total);
    lse = top + logf(total);
    const float v = __builtin_amdgcn_rcpf(total);
#pragma unroll
    for (int j = 0; j < V; ++j) soft[j] *= v;
  }
  return sum > 0;                       // not NaN, not a row of -infinity
}

template <int LANES, int V> __device__ __forceinline__ void fetch(const BalanceParams& p, int64_t t, int lane, float (&l)[V]) {
#pragma unroll
  for (int j = 0; j < V; j += 4) {
    const int e = expert_of<LANES>(j, lane);
    load4(p.logits, p.bf16, t * p.ld + e, p.E - e, l + j);
  }
}

// Sum over the tokens that share a wave: over the lanes of the same place in each group of LANES.
template <int LANES> __device__ __forceinline__ float over_tokens(float x) {
  float a, b;
  if (LANES <= 8) x += __shfl_xor(x, 8, 64);
  if (LANES <= 16) {
    rows_apart<16>(x, a, b);
    x = a + b;
  }
  if (LANES <= 32) {
    rows_apart<32>(x, a, b);
    x = a + b;
  }
  return x;
}

// The sums of tokens [begin, end): scores in red[0 .. E), counts in hist, z and the number of tokens in about[0 .. 2).
template <int LANES, int V, bool SIGMOID, bool Z> struct Sums {
  static constexpr int WAVES = FORWARD_THREADS / 64, WIDE = LANES * V;
  float red[WAVES][WIDE];
  uint32_t hist[WIDE];
  double part[WAVES][2];
  __device__ __forceinline__ void add(const BalanceParams& p, int64_t begin, int64_t end, double (&about)[2]) {
    constexpr int TOK = FORWARD_THREADS / LANES;
    const int lane = threadIdx.x % LANES, slot = threadIdx.x / LANES, wave = threadIdx.x >> 6;
    for (int e = threadIdx.x; e < WIDE; e += FORWARD_THREADS) hist[e] = 0;
    float sum[V] = {}, l[V];
    about[0] = about[1] = 0;
    if (begin + slot < end) fetch<LANES, V>(p, begin + slot, lane, l);
    __syncthreads();
    for (int64_t t = begin + slot; t < end; t += TOK) {
      const bool live = !p.q.mask || p.q.mask[t];
      int e = lane < p.k ? p.index[t * p.k + lane] : -1;
      float s[V], y, w[V], soft[V], lse;
      const bool on = token_scores<LANES, V, SIGMOID, Z, false>(l, s, y, w, soft, lse) && live;
      if (t + TOK < end) fetch<LANES, V>(p, t + TOK, lane, l);
      if (!on) continue;
#pragma unroll
      for (int j = 0; j < V; ++j) sum[j] = fmaf(s[j], y, sum[j]);
      if (lane == 0) {
        about[0] += (double)lse * (double)lse;
        about[1] += 1;
      }
      for (int j = lane; j < p.k; j += LANES) {
        if (j != lane) e = p.index[t * p.k + j];
        if (e >= 0 && e < p.E) atomicAdd(&hist[e], 1u);
      }
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float x = over_tokens<LANES>(sum[j]);
      if ((threadIdx.x & 63) < LANES) red[wave][expert_of<LANES>(j, lane)] = x;
    }
    group_sums<FORWARD_THREADS>(about, part);           // its barrier is red's and hist's too
  }
  __device__ __forceinline__ float score(int e) const {
    float x = 0;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) x += red[i][e];
    return x;
  }
};

// A lane keeps its experts' sums of a cell in registers, fp32 (a cell's tokens over FORWARD_THREADS / LANES lanes: at 256
// experts four each), the cells' are joined in 64 bits; counts are LDS atomics of whole numbers. 32768 tokens of 256 sigmoid
// scores fp32, 16 sequences: 13 us, 33.5 MB at 2.6 TB/s: half of it is the search of the cell, the first load and the sums
// over the workgroup at its end; more tokens on their way ahead (two turns instead of one, or whole vectors taken apart
// later) did not shorten it. 16384 of 64 softmax scores 5.6 us.
template <int LANES, int V, bool SIGMOID, bool Z>
__global__ __launch_bounds__(FORWARD_THREADS) void k_balance(BalanceParams p, int shift) {
  __shared__ Sums<LANES, V, SIGMOID, Z> sums;
  const int64_t i = blockIdx.x;
  const Cell c = cell_at(p.q, i, shift);
  double about[2];
  sums.add(p, c.begin, c.end, about);
  const CellSums w = {(char*)p.workspace, p.E};
  if ((int)threadIdx.x < p.E) {
    w.scores(i)[threadIdx.x] = sums.score(threadIdx.x);
    w.counts(i)[threadIdx.x] = sums.hist[threadIdx.x];
  }
  if (threadIdx.x < 2) w.about(i)[threadIdx.x] = about[threadIdx.x];
}

// out and the factors of the gradient, from the sums over the sequences.
__device__ __forceinline__ void balance_out(const BalanceParams& p, double balance, double live, double z, double n) {
  const double each = live > 0 ? 1 / live : 0, per = n > 0 ? 1 / n : 0;
  const float loss = (float)(p.balance_coef * balance * each + p.z_coef * z * per);
  p.out[0] = loss;
  if (p.loss) *p.loss = loss;
  p.out[1] = (float)(balance * each);
  p.out[2] = (float)(z * per);
  float* tail = p.slope + p.q.sequences * p.E;
  tail[0] = (float)(p.balance_coef * each);
  tail[1] = (float)(2 * p.z_coef * per);
}

// A sequence's balance from its experts' sums, x and c of expert e in the threads of one row (mine); total: of c.
__device__ __forceinline__ double sequence_balance(const BalanceParams& p, int64_t s, int e, bool mine, double x, double c,
                                                   double total, double n, double (*part)[1]) {
  // f less its mean, 1: scores sum to 1, so a constant has no gradient, and nothing cancels where the load is even
  const double f = total > 0 ? p.E * c / total : 0, per = n > 0 ? 1 / n : 0;
  if (mine) p.slope[s * p.E + e] = total > 0 ? (float)((f - 1) * per) : 0.f;
  double balance[1] = {mine ? f * x * per : 0.0};
  group_sums<END_THREADS>(balance, part);
  return balance[0];
}

// All tokens of one sequence in one workgroup: 512 of 8 experts 6.2 us, 2 of them the launch's.
template <int LANES, int V, bool SIGMOID, bool Z>
__global__ __launch_bounds__(FORWARD_THREADS) void k_balance_small(BalanceParams p, int shift) {
  __shared__ Sums<LANES, V, SIGMOID, Z> sums;
  __shared__ double part[END_THREADS / 64][1], part2[END_THREADS / 64][1];
  const int64_t begin = first_token(p.q, 0), end = first_token(p.q, 1);
  double about[2];
  sums.add(p, begin, end, about);
  const int e = threadIdx.x;
  const bool mine = e < p.E;
  const int64_t own = mine ? sums.hist[e] : 0, c = mine && p.load ? p.load[e] : own;
  if (mine) p.counts[e] = own;
  double total[1] = {(double)c};
  group_sums<END_THREADS>(total, part);
  const double balance = sequence_balance(p, 0, e, mine, mine ? sums.score(e) : 0.0, (double)c, total[0], about[1], part2);
  if (threadIdx.x == 0) balance_out(p, balance, about[1] > 0 ? 1 : 0, about[0], about[1]);
}

// Many cells of many experts: a workgroup adds up 64 experts of a sequence's cells, a wave every sixteenth.
__global__ __launch_bounds__(END_THREADS) void k_balance_columns(BalanceParams p, int shift, int64_t cells) {
  constexpr int ROWS = END_THREADS / 64;
  __shared__ double score[ROWS][64], part[ROWS][2];
  __shared__ long long count[ROWS][64];
  const int64_t s = blockIdx.x;
  const CellSums w = {(char*)p.workspace, p.E};
  int64_t first, last;
  cells_of(p.q, s, shift, first, last);
  const int lane = threadIdx.x & 63, row = threadIdx.x >> 6, e = blockIdx.y * 64 + lane;
  double x = 0;
  long long c = 0;
  if (e < p.E) {
#pragma unroll 4
    for (int64_t i = first + row; i < last; i += ROWS) {
      x += (double)w.scores(i)[e];
      c += w.counts(i)[e];
    }
  }
  score[row][lane] = x;
  count[row][lane] = c;
  double all[2] = {};                   // z, tokens
  if (blockIdx.y == 0)
    for (int64_t i = first + threadIdx.x; i < last; i += END_THREADS) {
      all[0] += w.about(i)[0];
      all[1] += w.about(i)[1];
    }
  group_sums<END_THREADS>(all, part);
  if (blockIdx.y == 0 && threadIdx.x < 2) about_sequences(p, cells)[4 * s + 2 + threadIdx.x] = all[threadIdx.x];
  if (row || e >= p.E) return;
#pragma unroll 5
  for (int k = 1; k < ROWS; ++k) {
    x += score[k][lane];
    c += count[k][lane];
  }
  scores_of_sequences(p, cells)[s * p.E + e] = x;
  p.counts[s * p.E + e] = c;
}

// One workgroup for each sequence: threads take an expert and every so many-th cell, or what its columns left. 5.6 us for 128
// cells of 64 experts, latencies: offsets, cells, two sums over the workgroup.
template <bool COLUMNS>
__global__ __launch_bounds__(END_THREADS) void k_balance_end(BalanceParams p, int shift, int64_t cells) {
  __shared__ double score[COLUMNS ? 1 : END_THREADS];
  __shared__ long long count[COLUMNS ? 1 : END_THREADS];
  __shared__ double part[END_THREADS / 64][3], part2[END_THREADS / 64][1];
  const int64_t s = blockIdx.x;
  double* const about = about_sequences(p, cells) + 4 * s;
  int width = 64;
  while (width < p.E) width *= 2;
  const int e = threadIdx.x & (width - 1), row = threadIdx.x / width, rows = END_THREADS / width;
  const bool mine = row == 0 && e < p.E;
  const long long load = mine && p.load ? p.load[e] : 0;
  double all[3] = {}, x = 0;            // counts, z, tokens
  long long c = 0;
  if (COLUMNS) {
    if (threadIdx.x == 0) {
      all[1] = about[2];
      all[2] = about[3];
    }
    if (mine) {
      x = scores_of_sequences(p, cells)[s * p.E + e];
      c = p.counts[s * p.E + e];
    }
  } else {
    const CellSums w = {(char*)p.workspace, p.E};
    int64_t first, last;
    cells_of(p.q, s, shift, first, last);
    for (int64_t i = first + threadIdx.x; i < last; i += END_THREADS) {
      all[1] += w.about(i)[0];
      all[2] += w.about(i)[1];
    }
    if (e < p.E) {
#pragma unroll 4
      for (int64_t i = first + row; i < last; i += rows) {
        x += (double)w.scores(i)[e];
        c += w.counts(i)[e];
      }
    }
    score[threadIdx.x] = x;
    count[threadIdx.x] = c;
  }
  all[0] = p.load ? (double)load : (double)c;
  group_sums<END_THREADS>(all, part);
  if (mine) {
    if (!COLUMNS) {
#pragma unroll 4
      for (int k = 1; k < rows; ++k) {
        x += score[k * width + e];
        c += count[k * width + e];
      }
      p.counts[s * p.E + e] = c;
    }
    if (p.load) c = load;
  }
  const double balance = sequence_balance(p, s, e, mine, x, (double)c, all[0], all[2], part2);
  if (threadIdx.x) return;
  if (p.q.sequences == 1) {
    balance_out(p, balance, all[2] > 0 ? 1 : 0, all[1], all[2]);
  } else {
    about[0] = balance;
    about[1] = all[2] > 0 ? 1 : 0;
    about[2] = all[1];
    about[3] = all[2];
  }
}
__global__ __launch_bounds__(END_THREADS) void k_balance_out(BalanceParams p, int64_t cells) {
  __shared__ double part[END_THREADS / 64][4];
  const double* a = about_sequences(p, cells);
  double sum[4] = {};
  for (int64_t s = threadIdx.x; s < p.q.sequences; s += END_THREADS)
#pragma unroll
    for (int k = 0; k < 4; ++k) sum[k] += a[4 * s + k];
  group_sums<END_THREADS>(sum, part);
  if (threadIdx.x == 0) balance_out(p, sum[0], sum[1], sum[2], sum[3]);
}

// The scores again, then s_j y (f_j - sum_i f_i s_i y), of sigmoids with 1 - sigma_j, plus 2 z lse softmax_j: one read and one
// write of a row, rounded once to its type. 32768 x 256 fp32 15 us, 67 MB at 4.5 TB/s; 16384 x 64 4.6 us.
template <int LANES, int V, bool SIGMOID, bool Z>
__global__ __launch_bounds__(BACKWARD_THREADS) void k_balance_backward(BalanceParams p, int shift) {
  constexpr int TOK = BACKWARD_THREADS / LANES;
  const int lane = threadIdx.x % LANES, slot = threadIdx.x / LANES;
  const float* tail = p.slope + p.q.sequences * p.E;
  const float g = *p.grad_loss, a = g * tail[0], b = g * tail[1];
  const Cell c = cell_at(p.q, blockIdx.x, shift);
  float f[V], l[V];
  if (c.begin + slot < c.end) fetch<LANES, V>(p, c.begin + slot, lane, l);
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int e = expert_of<LANES>(j, lane);
    f[j] = c.seq >= 0 && e < p.E ? p.slope[c.seq * p.E + e] * a : 0.f;
  }
  for (int64_t t = c.begin + slot; t < c.end; t += TOK) {
    const bool live = !p.q.mask || p.q.mask[t];
    float s[V], y, w[V], soft[V], lse;
    const bool on = token_scores<LANES, V, SIGMOID, Z, true>(l, s, y, w, soft, lse) && live;
    if (t + TOK < c.end) fetch<LANES, V>(p, t + TOK, lane, l);
    float mean = 0;
#pragma unroll
    for (int j = 0; j < V; ++j) mean = fmaf(f[j], s[j], mean);
    mean = sum_of<LANES>(mean) * y;
    const float zl = b * lse;
#pragma unroll
    for (int j = 0; j < V; j += 4) {
      float x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float d = (f[j + i] - mean) * (SIGMOID ? w[j + i] * y : y) * s[j + i];
        if (Z) d = fmaf(zl, SIGMOID ? soft[j + i] : s[j + i] * y, d);
        x[i] = on ? d : 0.f;
      }
      const int e = expert_of<LANES>(j, lane);
      store4(p.grad, p.bf16, t * p.E + e, p.E - e, x);
    }
  }
  auto clear = [&](int64_t from, int64_t to) {
    const float zero[4] = {};
    for (int64_t t = from + slot; t < to; t += TOK)
#pragma unroll
      for (int j = 0; j < V; j += 4) {
        const int e = expert_of<LANES>(j, lane);
        store4(p.grad, p.bf16, t * p.E + e, p.E - e, zero);
      }
  };
  clear(c.fill0, c.fill1);
  clear(c.fill2, c.fill3);
}

// Tokens of a tile, as a power of 2: no more workgroups than `most`, if 2^20 tokens a tile do.
int tile_of(const BalanceParams& p, int64_t most) {
  int shift = BALANCE_LEAST_SHIFT;
  while (most << shift < p.q.tokens && shift < 20) ++shift;
  return shift;
}

#define BALANCE_FORM(kernel, LANES, V)                                                                              \
  do {                                                                                                              \
    if (p.sigmoid && p.want_z) hipLaunchKernelGGL((kernel<LANES, V, true, true>), g, b, 0, st, p, shift);           \
    else if (p.sigmoid) hipLaunchKernelGGL((kernel<LANES, V, true, false>), g, b, 0, st, p, shift);                 \
    else if (p.want_z) hipLaunchKernelGGL((kernel<LANES, V, false, true>), g, b, 0, st, p, shift);                  \
    else hipLaunchKernelGGL((kernel<LANES, V, false, false>), g, b, 0, st, p, shift);                               \
  } while (0)
#define BALANCE_ON(kernel)                                \
  do {                                                    \
    if (p.E <= 32) BALANCE_FORM(kernel, 8, 4);            \
    else if (p.E <= 64) BALANCE_FORM(kernel, 16, 4);      \
    else if (p.E <= 128) BALANCE_FORM(kernel, 16, 8);     \
    else if (p.E <= 256) BALANCE_FORM(kernel, 32, 8);     \
    else if (p.E <= 512) BALANCE_FORM(kernel, 64, 8);     \
    else BALANCE_FORM(kernel, 64, 16);                    \
  } while (0)

int lanes_of(int E) { return E <= 32 ? 8 : E <= 128 ? 16 : E <= 256 ? 32 : 64; }

}  // namespace

hipError_t launch_balance(const BalanceParams& p, hipStream_t st) {
  int shift = 0;
  const dim3 b(FORWARD_THREADS);
  if (p.q.sequences == 1 && p.q.tokens <= 8 * (FORWARD_THREADS / lanes_of(p.E))) {
    const dim3 g(1);
    BALANCE_ON(k_balance_small);
    return hipGetLastError();
  }
  // fewer cells are added up sooner: 65536 tokens of 64 experts 13.7 us with 128 tiles, 15.9 with 256, 17.1 with 64; 32768 of
  // 256 experts 20.5, 19.2 and 26.7
  shift = tile_of(p, p.E <= 128 ? 128 : 256);
  const int64_t cells = cells_of_all(p.q, shift);
  if (cells > 0) {
    const dim3 g((uint32_t)cells);
    BALANCE_ON(k_balance);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 each((uint32_t)p.q.sequences), end(END_THREADS);
  // by columns first where one thread of k_balance_end would add up more than eight cells on average: all 32768 tokens of 256
  // experts together 19.2 us instead of 29, 8192 of 1024 experts 19.6 instead of 80 (16384 of 64 experts, 128 cells: 10.3, and
  // with a launch more 13.9)
  int width = 64;
  while (width < p.E) width *= 2;
  if ((p.q.tokens / p.q.sequences >> shift) * width > 8 * END_THREADS) {
    hipLaunchKernelGGL(k_balance_columns, dim3((uint32_t)p.q.sequences, (uint32_t)(p.E + 63) / 64), end, 0, st, p, shift, cells);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_balance_end<true>, each, end, 0, st, p, shift, cells);
  } else {
    hipLaunchKernelGGL(k_balance_end<false>, each, end, 0, st, p, shift, cells);
  }
  e = hipGetLastError();
  if (e != hipSuccess || p.q.sequences == 1) return e;
  hipLaunchKernelGGL(k_balance_out, dim3(1), dim3(END_THREADS), 0, st, p, cells);
  return hipGetLastError();
}

hipError_t launch_balance_backward(const BalanceParams& p, hipStream_t st) {
  const int shift = tile_of(p, 2048);
  const int64_t cells = cells_of_all(p.q, shift);
  if (cells > 0) {
    const dim3 g((uint32_t)cells), b(BACKWARD_THREADS);
    BALANCE_ON(k_balance_backward);
  }
  return hipGetLastError();
}
