// Operators a training step needs beside the projected matrices: gradient norm and clipping, AdamW
// over lists of tensors, routing of tokens to experts. Lists of tensors travel in the kernels'
// arguments (at most 4 KB), so a call needs no device descriptors, no copy and no workspace for them.
#pragma once
#include "common.h"

// A failed call's status with its message for moara_last_error (moara_api.hip holds the message).
__attribute__((visibility("hidden"))) int moara_fail(int code, const char* fmt, ...);

// ---------------------------------------------------------------- gradient norm, clipping
constexpr int GRAD_MAX = 160;
struct GradList {
  void* g[GRAD_MAX];
  int64_t count[GRAD_MAX];
  uint32_t start[GRAD_MAX];     // first tile
  uint32_t bf16[(GRAD_MAX + 31) / 32];   // bit i: tensor i is bf16
  int n;
  uint32_t tiles;
};
constexpr int NORM_WGS = 2048;  // partial sums; the workspace of moara_grad_norm holds them
uint32_t grad_tiles(int64_t count);
// filled: how many partial sums the launches before this one have stored, raised to what there is after
// it (a launch adds to those, and stores the others). once: the list is read past the caches.
hipError_t launch_grad_norm(const GradList& l, bool once, double* partial, uint32_t& filled, hipStream_t st);
hipError_t launch_grad_norm_end(const double* partial, uint32_t filled, float max_norm, float* out, hipStream_t st);
hipError_t launch_grad_scale(const GradList& l, bool once, const float* coef, hipStream_t st);

// ---------------------------------------------------------------- AdamW
constexpr int ADAMW_MAX = 75, ADAMW_SETS = 8;
struct AdamwSet {               // numbers that tensors of a launch share
  float decay;                  // 1 - lr weight_decay
  float lr;                     // lr / (1 - beta1^t)
  float rbc2;                   // 1 / (1 - beta2^t)
};
struct AdamwList {
  void* p[ADAMW_MAX];
  const void* g[ADAMW_MAX];
  void* m[ADAMW_MAX];
  void* v[ADAMW_MAX];
  uint8_t* scales[ADAMW_MAX];   // 8 bits: two exponents for each block of 32
  uint64_t about[ADAMW_MAX];    // elements (34 bits), set (3), place in the caller's list (27)
  uint32_t start[ADAMW_MAX];    // first workgroup
  AdamwSet set[ADAMW_SETS];
  const float* clip;
  uint64_t seed;
  float b1, c1, b2, c2, eps;    // c = 1 - b
  int n;
};
constexpr int ADAMW_SET_BIT = 34, ADAMW_PLACE_BIT = 37;
// Mixes 32 bits; digits of the golden ratio, sqrt 2 and e (odd).
constexpr uint32_t MIX_A = 0x9E3779B1u, MIX_B = 0x6A09E667u, MIX_C = 0xB7E15163u;
__host__ __device__ __forceinline__ uint32_t mix32(uint32_t x) {
  x = (x ^ (x >> 16)) * MIX_A;
  x = (x ^ (x >> 15)) * MIX_B;
  return x ^ (x >> 16);
}
static_assert(sizeof(GradList) <= 4096 && sizeof(AdamwList) <= 4096, "lists travel in the kernels' arguments");
uint32_t adamw_tiles(int64_t count);
hipError_t launch_adamw(const AdamwList& l, bool p_bf16, bool g_bf16, int bits, uint32_t total, hipStream_t st);

// ---------------------------------------------------------------- routing to experts
struct RouteParams {
  const void* logits;
  int64_t tokens, ld;           // ld: elements from one token's logits to the next one's
  const float* bias;            // null: none
  const uint8_t* mask;          // null: every token is routed
  int32_t* index;
  float* weight;                // forward: out; backward: the gradient of the weights
  unsigned long long* counts;   // null: not wanted
  void* grad;                   // backward: tokens x experts, type of the logits
  int E, k, groups, top_groups, group_best;
  uint32_t group_size, group_inv;   // group of expert e: (e * group_inv) >> 20
  int sigmoid, renorm, bf16;
  float scale;
};
constexpr int ROUTE_MAX_EXPERTS = 1024, ROUTE_MAX_K = 64, ROUTE_MAX_GROUPS = 64;
hipError_t launch_route(const RouteParams& p, hipStream_t st);
hipError_t launch_route_backward(const RouteParams& p, hipStream_t st);
hipError_t launch_route_balance(int E, long long* counts, float* bias, float rate, hipStream_t st);
