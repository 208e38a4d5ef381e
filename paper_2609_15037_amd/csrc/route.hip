// Routing of tokens to experts: scores, selection (groups, top-k), weights, their gradient, and the step
// of the balancing bias.
#include <float.h>

#include "lanes.h"
#include "train.h"

namespace {

// Floats as unsigned integers of the same order; 0 is left for what cannot be chosen (-inf, NaN, none).
__device__ __forceinline__ uint32_t order_key(float c) {
  const uint32_t b = __float_as_uint(c);           // no -0: a score, or a sum of one with a bias
  return c > -__builtin_inff() ? b ^ ((uint32_t)((int)b >> 31) | 0x80000000u) : 0u;
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float((int)k < 0 ? k & 0x7FFFFFFFu : ~k);
}
// The key of a + b. Two finite values (biases of the type's lowest one) may sum to less than fp32 holds: half of it,
// at most -2^127, has a key from 2^23 to 2^24 - 1, half of which is above 0 and below all keys of finite sums.
__device__ __forceinline__ uint32_t sum_key(float a, float b) {
  const float s = a + b;
  return s > -__builtin_inff() ? order_key(s) : order_key(0.5f * a + 0.5f * b) >> 1;
}

// A row's largest logit and its sum of exponentials (softmax). The sum is taken in 64 bits: an expert's
// score must not depend on the order of the others.
struct Row { float top, total; };
__device__ __forceinline__ float score(float l, const Row& r, int sigmoid) {
  return sigmoid ? 1.f / (1.f + expf(-l)) : expf(l - r.top) / r.total;
}
// The same scores, to the bit, of all of a lane's logits, and the row. The quotients are rounded correctly
// without the division's scaling. 1 / d with d from 1 to 2^100: one Newton step on the hardware's reciprocal
// (compared for every such d). e / d with e from 2^-78: the correctly rounded reciprocal's product and one step
// on its remainder (Markstein 1990). Lanes with other values divide.
template <int LANES, int V> __device__ __forceinline__ Row scores(const float (&l)[V], int sigmoid, float (&s)[V]) {
  if (sigmoid) {
    float most = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      s[j] = expf(-l[j]);
      most = fmaxf(most, s[j]);
    }
    if (most < 0x1p99f) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float d = 1.f + s[j], y = __builtin_amdgcn_rcpf(d);
        s[j] = fmaf(fmaf(-d, y, 1.f), y, y);
      }
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) s[j] = 1.f / (1.f + s[j]);
    }
    return Row{0.f, 1.f};
  }
  float top = l[0];
#pragma unroll
  for (int j = 1; j < V; ++j) top = fmaxf(top, l[j]);
  top = max_of<LANES>(top);
  double sum = 0;
  uint32_t least = 0xFFFFFFFFu;         // of the exponentials that are not zero, their bits less 1
#pragma unroll
  for (int j = 0; j < V; ++j) {
    s[j] = expf(l[j] - top);
    sum += (double)s[j];
    least = min(least, __float_as_uint(s[j]) - 1u);
  }
  const float total = (float)sum_of<LANES>(sum);
  if (least >= 0x18800000u - 1u) {      // 2^-78
    const float y = 1.f / total;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float q = s[j] * y;
      s[j] = fmaf(fmaf(-q, total, s[j]), y, q);
    }
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) s[j] = s[j] / total;
  }
  return Row{top, total};
}

// u_j of the chosen experts, one a lane (lanes without one: there = false): the score itself, or its share
// of the chosen ones' sum, from the logits less their largest, so that shares exist where scores underflow
// (the sigmoid as exp(min(l, 0)) / (1 + exp(-|l|))). No share where every chosen logit is -inf.
template <int LANES> __device__ __forceinline__ float chosen_share(float l, bool there, const Row& r, const RouteParams& p) {
  if (!p.renorm) return there ? score(l, r, p.sigmoid) : 0.f;
  const float x = p.sigmoid ? fminf(l, 0.f) : l;
  const float top = max_of<LANES>(there ? x : -FLT_MAX);
  float u = there ? expf(x - fmaxf(top, -FLT_MAX)) : 0.f;
  if (p.sigmoid) u /= 1.f + expf(-fabsf(l));
  const float total = sum_of<LANES>(u);
  return total > 0.f ? u / total : 0.f;
}

// ---- selection. A candidate is a positive double that orders as (key, lowest index first): key / 2 above
// 2^31 key - index - 1 below; the upper half is 0 for what cannot be chosen. (Keys of numbers and infinity
// stay under the doubles' infinity.) One instruction then compares and moves key and index together. For the
// lanes' heads, two rounds on 32 bits, whose moves and comparisons are one instruction, are shorter again.
__device__ __forceinline__ double candidate(uint32_t key, int e) {
  return __builtin_bit_cast(double, (uint64_t)(key >> 1) << 32 | (key << 31 | (0x7FFFFFFFu - (uint32_t)e)));
}
__device__ __forceinline__ void in_order(double& a, double& b) {
  const double hi = fmax(a, b), lo = fmin(a, b);
  a = hi;
  b = lo;
}
// d[B .. B + N) in falling order: Batcher's odd-even merge sort.
template <int B, int N, int V> __device__ __forceinline__ void sort_falling(double (&d)[V]) {
#pragma unroll
  for (int p = 1; p < N; p *= 2)
#pragma unroll
    for (int k = p; k >= 1; k /= 2)
#pragma unroll
      for (int j = k % p; j + k < N; j += 2 * k)
#pragma unroll
        for (int i = 0; i < k; ++i)
          if (i + j + k < N && (i + j) / (2 * p) == (i + j + k) / (2 * p)) in_order(d[B + i + j], d[B + i + j + k]);
}
// The largest DEP of d, falling, in d[0 .. DEP).
template <int DEP, int V> __device__ __forceinline__ void best_falling(double (&d)[V]) {
  if (DEP == V) {
    sort_falling<0, V>(d);
  } else {              // two sorted halves: the larger of each and its mirror, a bitonic run, then merged
    static_assert(DEP == V || 2 * DEP == V);
    sort_falling<0, V / 2>(d);
    sort_falling<V / 2, V / 2>(d);
#pragma unroll
    for (int j = 0; j < V / 2; ++j) d[j] = fmax(d[j], d[V - 1 - j]);
#pragma unroll
    for (int k = V / 4; k >= 1; k /= 2)
#pragma unroll
      for (int j = 0; j < V / 2; ++j)
        if (!(j & k)) in_order(d[j], d[j + k]);
  }
}

// Orders a wave's accesses to LDS: a token's lanes share a wave, what they exchange concerns no other.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// What a token's lanes exchange about its groups.
template <int LANES, int V> struct Groups {
  static constexpr int MOST = LANES * V < ROUTE_MAX_GROUPS ? LANES * V : ROUTE_MAX_GROUPS;
  uint64_t value[MOST];         // the two best keys, then (key of the group, lowest index first)
  uint32_t kept[MOST];
};

// The two best keys over `span` neighbouring lanes, a power of two.
template <int LANES> __device__ __forceinline__ void two_best(uint32_t& best, uint32_t& next, int span) {
  auto with = [&](uint32_t ob, uint32_t on) {
    next = max(min(best, ob), max(next, on));
    best = max(best, ob);
  };
  if (span > 1) with(dpp<0xB1>(best), dpp<0xB1>(next));
  if (span > 2) with(dpp<0x4E>(best), dpp<0x4E>(next));
  if (span > 4) with(dpp<0x141>(best), dpp<0x141>(next));
  if (LANES >= 16 && span > 8) with(dpp<0x140>(best), dpp<0x140>(next));
  if (LANES >= 32 && span > 16) with((uint32_t)__shfl_xor(best, 16, 64), (uint32_t)__shfl_xor(next, 16, 64));
}

// Keys of experts outside the kept groups become 0. The two best keys of a group: where a group is 4, 8, .. 64
// consecutive experts (EVEN) they are found across the lanes that hold it, else by lanes that share it in LDS. A group
// counts with its best, or the sum of the two best (what cannot be chosen adds nothing); a lane ranks it.
template <int LANES, int V, bool EVEN>
__device__ __forceinline__ void keep_groups(uint32_t (&key)[V], const RouteParams& p, uint32_t* rk, Groups<LANES, V>& x,
                                            int lane) {
  const int shift = EVEN ? __builtin_ctz(p.group_size) - 2 : 0, span = 1 << shift;      // EVEN: lanes of a group
  if (EVEN) {
#pragma unroll
    for (int c = 0; c < V / 4; ++c) {
      const uint32_t* k = key + 4 * c;
      const uint32_t b0 = max(k[0], k[1]), b1 = max(k[2], k[3]);
      uint32_t best = max(b0, b1), next = max(min(b0, b1), max(min(k[0], k[1]), min(k[2], k[3])));
      two_best<LANES>(best, next, span);
      const int g = (c * LANES + lane) >> shift;
      if (g < p.groups && !(lane & (span - 1))) x.value[g] = (uint64_t)best << 32 | next;
    }
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) rk[expert_of<LANES>(j, lane)] = key[j];
    wave_sync();
    // lanes of a group: as many as there are for each, a power of two
    const int share = p.groups >= LANES ? 0 : 31 - __builtin_clz(LANES) - (32 - __builtin_clz(p.groups - 1)), span = 1 << share;
    for (int g = lane >> share; g < p.groups; g += LANES >> share) {
      uint32_t best = 0, next = 0;
      for (uint32_t q = lane & (span - 1); q < p.group_size; q += span) {
        const uint32_t k = rk[g * p.group_size + q];
        next = max(next, min(best, k));
        best = max(best, k);
      }
      two_best<LANES>(best, next, span);
      if (!(lane & (span - 1))) x.value[g] = (uint64_t)best << 32 | next;
    }
  }
  wave_sync();
  for (int g = lane; g < p.groups; g += LANES) {
    const uint32_t best = (uint32_t)(x.value[g] >> 32), next = (uint32_t)x.value[g];
    const uint32_t v = p.group_best == 2 && next ? sum_key(key_value(best), key_value(next)) : best;
    x.value[g] = (uint64_t)v << 32 | (uint32_t)(ROUTE_MAX_GROUPS - 1 - g);
  }
  wave_sync();
  for (int g = lane; g < p.groups; g += LANES) {
    const uint64_t own = x.value[g];
    int rank = 0;
    for (int q = 0; q < p.groups; ++q) rank += x.value[q] > own;
    x.kept[g] = rank < p.top_groups;
  }
  wave_sync();
#pragma unroll
  for (int j = 0; j < V; j += EVEN ? 4 : 1) {
    const int e = expert_of<LANES>(j, lane);
    const int g = EVEN ? e >> (shift + 2) : (int)(((uint32_t)e * p.group_inv) >> 20);
    const bool out = g >= p.groups || !x.kept[g];
#pragma unroll
    for (int i = 0; i < (EVEN ? 4 : 1); ++i) key[j + i] = out ? 0u : +key[j + i];
  }
  wave_sync();          // what is in LDS is read before the next token's is written
}

// LANES lanes take one token, V experts each. Bound by its arithmetic: the exponentials (about 20
// instructions each), then the choice. Every lane sorts its own candidates; the token's next expert is the
// largest of the lanes' heads, whose lane moves up. The next token's logits are on their way meanwhile. A
// workgroup counts the experts' tokens in LDS and adds them to the counts at its end: an address takes an
// addition in about 20 ns, so at most 256 workgroups walk over the tokens (with 1024 the counts cost 20 us of
// 26 for 16384 tokens of 64 experts, with 128 the rest takes as much longer). They are whole numbers: the
// order of the additions does not change them.
// fp32 logits, with bias and counts, in a captured graph (a kernel trace gives up to 10 % more): 113 tokens, 64
// experts, top 6: 4.8 us; 16384 tokens of the same 8.6 us (6.4 without counts); 32768 tokens, 256 experts in 8 groups,
// top 8: 23.4 us (18.1; a scan of all candidates for each choice, with divisions and one lane for a group, took 41);
// without groups 20.1 (15.3); 16384 tokens, 512 experts, top 12: 27.9 us.
enum { NO_GROUPS, EVEN_GROUPS, ANY_GROUPS };
constexpr int ROUTE_THREADS = 1024;
template <int LANES, int V, int DEP, int GROUPS>
__global__ __launch_bounds__(ROUTE_THREADS) void k_route(RouteParams p) {
  constexpr int TOK = ROUTE_THREADS / LANES;      // tokens of a workgroup at a time
  __shared__ uint32_t hist[LANES * V];
  __shared__ float bias[LANES * V];     // what scores are raised by; -inf for experts that do not exist
  __shared__ uint32_t rowkey[GROUPS == ANY_GROUPS ? TOK * LANES * V : 1];
  __shared__ Groups<LANES, V> grouped[GROUPS != NO_GROUPS ? TOK : 1];
  const int lane = threadIdx.x % LANES, slot = threadIdx.x / LANES;
  const bool half = p.bf16;
  for (int e = threadIdx.x; e < LANES * V; e += ROUTE_THREADS) {
    hist[e] = 0;
    bias[e] = e >= p.E ? -__builtin_inff() : p.bias ? p.bias[e] : 0.f;
  }
  __syncthreads();
  float l[V];
  auto fetch = [&](int64_t t) {         // a token's logits, past the end another's
    const int64_t row = (t < p.tokens ? t : 0) * p.ld;
#pragma unroll
    for (int j = 0; j < V; j += 4) {
      const int e = expert_of<LANES>(j, lane);
      load4(p.logits, half, row + e, p.E - e, l + j);
    }
  };
  const int64_t step = (int64_t)gridDim.x * TOK;
  fetch((int64_t)blockIdx.x * TOK + slot);
  for (int64_t t = (int64_t)blockIdx.x * TOK + slot; t - slot < p.tokens; t += step) {
    const int64_t row = (t < p.tokens ? t : 0) * p.ld;
    const bool live = t < p.tokens && !(p.mask && !p.mask[t]);
    float s[V];
    const Row r = scores<LANES, V>(l, p.sigmoid, s);
    if (t - slot + step < p.tokens) fetch(t + step);        // arrives during the choice
    uint32_t key[V];
#pragma unroll
    for (int j = 0; j < V; ++j) key[j] = order_key(s[j] + bias[expert_of<LANES>(j, lane)]);
    if (GROUPS != NO_GROUPS)
      keep_groups<LANES, V, GROUPS == EVEN_GROUPS>(key, p, rowkey + (GROUPS == ANY_GROUPS ? slot * (LANES * V) : 0),
                                                   grouped[slot], lane);
    double d[V];
#pragma unroll
    for (int j = 0; j < V; ++j) d[j] = candidate(key[j], expert_of<LANES>(j, lane));
    best_falling<DEP>(d);
    uint32_t hi[DEP], lo[DEP];
#pragma unroll
    for (int j = 0; j < DEP; ++j) {
      hi[j] = (uint32_t)(__builtin_bit_cast(uint64_t, d[j]) >> 32);
      lo[j] = (uint32_t)__builtin_bit_cast(uint64_t, d[j]);
    }
    uint32_t own = 0;     // of lane i < k: 2^31 - 1 less the token's i-th expert, in 31 bits; 0 where there is none
    // keep: how much of the list later choices may still ask for
    auto choose = [&](int i, int keep) {
      const uint32_t th = max_of<LANES>(hi[0]), head = hi[0] == th ? lo[0] : 0u, tl = max_of<LANES>(head);
      const bool up = head == tl;
      // the + makes values of the operands: of two elements of an array the choice would be an index
#pragma unroll
      for (int j = 0; j + 1 < DEP; ++j)
        if (j < keep) {
          hi[j] = up ? +hi[j + 1] : +hi[j];
          lo[j] = up ? +lo[j + 1] : +lo[j];
        }
      if (DEP <= keep) {
        hi[DEP - 1] = up ? 0u : +hi[DEP - 1];
        lo[DEP - 1] = up ? 0u : +lo[DEP - 1];
      }
      if (lane == i) own = th ? tl & 0x7FFFFFFFu : 0u;
    };
    if (DEP < V) {        // at most DEP choices
#pragma unroll
      for (int i = 0; i < DEP; ++i)
        if (i < p.k) choose(i, DEP - 1 - i);
    } else {
      for (int i = 0; i < p.k; ++i) choose(i, DEP);
    }
    const int chosen = live && own ? (int)(0x7FFFFFFFu - own) : -1;
    const bool there = chosen >= 0;
    const float u = chosen_share<LANES>(there ? load1(p.logits, half, row + chosen) : 0.f, there, r, p);
    if (lane < p.k && t < p.tokens) {
      p.index[t * p.k + lane] = chosen;
      p.weight[t * p.k + lane] = u * p.scale;
      if (p.counts && there) atomicAdd(&hist[chosen], 1u);
    }
  }
  if (!p.counts) return;
  __syncthreads();
  for (int e = threadIdx.x; e < p.E; e += ROUTE_THREADS)
    if (hist[e]) atomicAdd(&p.counts[e], (unsigned long long)hist[e]);
}

// Gradient of the weights -> gradient of the logits. With u_j the chosen experts' shares and s their scores:
// renormalised, t_j = u_j (dw_j - sum dw u) and d l_j = t_j, times 1 - s_j for the sigmoid (the softmax's own
// sum vanishes); else t_j = dw_j s_j, times 1 - s_j for the sigmoid, and d l_e = t_e - s_e sum t for the softmax,
// the only form that needs the whole row.
// A row is put together in LDS and written once. 32768 tokens, 256 experts, fp32 (in a captured graph): renormalised 9.1
// us, 3.9 TB/s of which the write alone would take 6: a token's index, its logit, the shares and the row follow one
// another, and a workgroup begins the next token when they are done; the whole softmax row 13.4 us, 5.2 TB/s;
// 16384 tokens of 64 experts 3.3 and 4.0 us, most of it the launch.
template <int LANES, int V>
__global__ __launch_bounds__(256) void k_route_backward(RouteParams p) {
  constexpr int TOK = 256 / LANES;
  __shared__ float out[TOK * LANES * V];
  const int lane = threadIdx.x % LANES, slot = threadIdx.x / LANES;
  const bool whole = !p.sigmoid && !p.renorm, half = p.bf16;
  for (int64_t t0 = (int64_t)blockIdx.x * TOK; t0 < p.tokens; t0 += (int64_t)gridDim.x * TOK) {
    const int64_t t = t0 + slot;
    const bool in = t < p.tokens;
    const int64_t row = (in ? t : 0) * p.ld;
    const int chosen = in && lane < p.k ? p.index[t * p.k + lane] : -1;
    const bool there = chosen >= 0 && chosen < p.E;
    const float dw = there ? p.weight[t * p.k + lane] : 0.f;
    const float lc = there ? load1(p.logits, half, row + chosen) : 0.f;
    float l[V], s[V];
    Row r = {0.f, 1.f};
    if (whole) {
#pragma unroll
      for (int j = 0; j < V; j += 4) {
        const int e = expert_of<LANES>(j, lane);
        load4(p.logits, half, row + e, p.E - e, l + j);
      }
      r = scores<LANES, V>(l, 0, s);
    }
    const float u = chosen_share<LANES>(lc, there, r, p);
    const float mean = p.renorm ? sum_of<LANES>(dw * u) : 0.f;
    float d = there ? p.scale * u * (dw - mean) : 0.f;
    if (p.sigmoid) d *= 1.f / (1.f + expf(lc));
    const float total = whole ? sum_of<LANES>(d) : 0.f;
    const bool any = max_of<LANES>((uint32_t)there) != 0;
    float* o = out + slot * (LANES * V);        // the lanes of a token share a wave
    wave_sync();
#pragma unroll
    for (int j = 0; j < V; ++j) o[expert_of<LANES>(j, lane)] = whole && any ? -s[j] * total : 0.f;
    wave_sync();
    if (there) o[chosen] += d;
    wave_sync();
    if (in) {
#pragma unroll
      for (int j = 0; j < V; j += 4) {
        const int e = expert_of<LANES>(j, lane);
        store4(p.grad, half, t * p.E + e, p.E - e, o + e);
      }
    }
  }
}

// bias += rate sign(mean of the counts - count), then the counts start again from zero.
__global__ __launch_bounds__(256) void k_route_balance(int E, long long* __restrict__ counts, float* __restrict__ bias,
                                                       float rate) {
  __shared__ long long part[4];
  long long sum = 0;
  for (int e = threadIdx.x; e < E; e += 256) sum += counts[e];
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
  __syncthreads();
  sum = part[0] + part[1] + part[2] + part[3];
  for (int e = threadIdx.x; e < E; e += 256) {
    const long long d = sum - counts[e] * E;
    bias[e] += d > 0 ? rate : d < 0 ? -rate : 0.f;
    counts[e] = 0;
  }
}

// Lanes of a token: as few as hold its choices, and its experts at sixteen a lane (eight lanes: at four, or at
// eight where there are tokens for half of the CUs). Fewer lanes share a wave's instructions among more
// tokens: 65536 tokens of 8 experts, top 2, take 6 us on eight lanes and 12 on sixteen; 16384 of 512 experts, top
// 12, with counts 28 us on 32 lanes and 34 on a wave. Top 6 of 64 experts on eight and on sixteen lanes, with counts:
// 4096 tokens 6.6 and 6.0 us, 8192 7.2 and 7.4, 14000 8.2 and 9.4, 16384 8.6 and 10.3, 65536 15.5 and 18.5; without:
// 8192 6.3 and 4.7, 16384 6.4 and 4.8, 32768 6.7 and 7.6, 65536 10.7 and 13.1. One rule for both, between the two
// crossings.
// Few tokens take more lanes, as long as one round of workgroups holds them (of 64 where each adds to the
// counts: 8192 tokens of 256 experts 10.8 us with 128 workgroups, 12.5 with 256): a lane's experts are straight
// code that such a call runs once (113 tokens of 138 experts 7.9 us on sixteen lanes, 5.3 on a wave).
// The backward pass takes the same lanes: over these shapes it is at most 0.4 us behind the best for it (4096 tokens
// of 256 experts 3.7 us on a wave, 3.4 on sixteen or 32 lanes).
int lanes_of(const RouteParams& p) {
  const int most8 = p.tokens >= 128 * (ROUTE_THREADS / 8) ? 64 : 32;
  int lanes = p.k <= 8 && p.E <= most8 ? 8 : p.k <= 16 && p.E <= 256 ? 16 : p.k <= 32 && p.E <= 512 ? 32 : 64;
  while (lanes >= 16 && lanes < 64 && p.E > 4 * lanes &&
         p.tokens <= (p.counts ? 64 : 256) * (ROUTE_THREADS / (2 * lanes)))
    lanes *= 2;
  return lanes;
}
int64_t workgroups(const RouteParams& p, int threads, int64_t most) {
  const int64_t tok = threads / lanes_of(p), n = (p.tokens + tok - 1) / tok;
  return n < most ? n : most;
}

}  // namespace

hipError_t launch_route(const RouteParams& p, hipStream_t st) {
  const dim3 g((uint32_t)workgroups(p, ROUTE_THREADS, 256)), b(ROUTE_THREADS);
  const int s = (int)p.group_size;
  // the same 32768 tokens, with counts: 23.3 us, through the form for groups of any size 26.7
  const int groups = p.groups == 1 ? NO_GROUPS : s >= 4 && s <= 64 && (s & (s - 1)) == 0 ? EVEN_GROUPS : ANY_GROUPS;
#define ROUTE(LANES, V, DEP)                                                                                     \
  do {                                                                                                           \
    if (groups == NO_GROUPS) hipLaunchKernelGGL((k_route<LANES, V, DEP, NO_GROUPS>), g, b, 0, st, p);            \
    else if (groups == EVEN_GROUPS) hipLaunchKernelGGL((k_route<LANES, V, DEP, EVEN_GROUPS>), g, b, 0, st, p);   \
    else hipLaunchKernelGGL((k_route<LANES, V, DEP, ANY_GROUPS>), g, b, 0, st, p);                               \
  } while (0)
  const int lanes = lanes_of(p);
  // a lane's best eight are enough: 32768 tokens of 256 experts in 8 groups, with counts, 23.3 us, with lists of
  // sixteen 26.2
  const bool few = p.k <= 8;
#define ROUTE_ON(LANES)                                   \
  do {                                                    \
    if (p.E <= 4 * LANES) ROUTE(LANES, 4, 4);             \
    else if (p.E <= 8 * LANES) ROUTE(LANES, 8, 8);        \
    else if (few) ROUTE(LANES, 16, 8);                    \
    else ROUTE(LANES, 16, 16);                            \
  } while (0)
  if (lanes == 8 && p.E <= 32) ROUTE(8, 4, 4);
  else if (lanes == 8) ROUTE(8, 8, 8);
  else if (lanes == 16) ROUTE_ON(16);
  else if (lanes == 32) ROUTE_ON(32);
  else ROUTE_ON(64);
#undef ROUTE_ON
#undef ROUTE
  return hipGetLastError();
}

hipError_t launch_route_backward(const RouteParams& p, hipStream_t st) {
  const dim3 g((uint32_t)workgroups(p, 256, 1024)), b(256);
  const int lanes = lanes_of(p);
#define BACKWARD(LANES, V) hipLaunchKernelGGL((k_route_backward<LANES, V>), g, b, 0, st, p)
#define BACKWARD_ON(LANES)                                \
  do {                                                    \
    if (p.E <= 4 * LANES) BACKWARD(LANES, 4);             \
    else if (p.E <= 8 * LANES) BACKWARD(LANES, 8);        \
    else BACKWARD(LANES, 16);                             \
  } while (0)
  if (lanes == 8 && p.E <= 32) BACKWARD(8, 4);
  else if (lanes == 8) BACKWARD(8, 8);
  else if (lanes == 16) BACKWARD_ON(16);
  else if (lanes == 32) BACKWARD_ON(32);
  else BACKWARD_ON(64);
#undef BACKWARD_ON
#undef BACKWARD
  return hipGetLastError();
}

hipError_t launch_route_balance(int E, long long* counts, float* bias, float rate, hipStream_t st) {
  hipLaunchKernelGGL(k_route_balance, dim3(1), dim3(256), 0, st, E, counts, bias, rate);
  return hipGetLastError();
}
