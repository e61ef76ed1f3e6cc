// Routing from logits: softmax or sigmoid scores s, a bias b that balances the experts' load, groups of experts, top-k,
// renormalised weights.  Per token, over the experts it may use (with a slot table the resident ones, Masked Gating):
//   c_e = s_e + b_e;  value of a group = sum of its group_top largest c;  the topk_groups best groups are kept, and further ones as
//   long as they hold fewer than k experts to choose from;  the k largest c of the kept groups are chosen, ties to the lowest
//   index;  weight = scale * s_e, or scale * s_e / sum of the chosen s.
//
// A warp routes a token; lane l holds the experts l * N ... l * N + N - 1, so the order of lanes is that of indices and a tie goes to
// the lowest lane.  The order of the choices is that of 64-bit scores: of thousands of tokens some have two experts closer than
// fp32 tells apart.  Without a bias, and with groups valued by their best expert, it is that of the logits themselves.
#pragma once
#include <math_constants.h>

#include "../../include/swapmoe.h"
#include "common.cuh"
#include "launch.cuh"

namespace swapmoe {

constexpr int kRouteMaxE = 512, kRouteMaxTopK = 16, kRouteMaxGroups = 32;
constexpr int kRouteWarps = 4;

struct RouteGate {
  int score, n_groups, topk_groups, group_top, renorm;
  float scale;
  int group_size;
  uint32_t group_magic;      // e / group_size = 2 e * group_magic >> 32 for the indices that occur
};

struct RouteGroupsArgs {
  const float* logits;
  const float* bias;                // [E] or nullptr
  const int32_t* expert_to_slot;    // [E] or nullptr
  int32_t* experts;                 // [T, k]
  float* weights;                   // [T, k]
  int32_t* slots;                   // [T, k] or nullptr
  long long stride;
  int T, E, k;
  RouteGate gate;
};

// Order-preserving key of a choice, never 0; NaN counts as -infinity.
__device__ __forceinline__ unsigned long long choice_key(double c) {
  c = c == c ? c + 0.0 : -CUDART_INF;                       // (-0 becomes +0)
  const unsigned long long b = (unsigned long long)__double_as_longlong(c);
  return b >> 63 ? ~b : b | 0x8000000000000000ull;
}
__device__ __forceinline__ unsigned long long warp_max_key(unsigned long long key) {
  const uint32_t hi = __reduce_max_sync(0xffffffffu, (uint32_t)(key >> 32));
  const uint32_t lo = __reduce_max_sync(0xffffffffu, (uint32_t)(key >> 32) == hi ? (uint32_t)key : 0u);
  return (unsigned long long)hi << 32 | lo;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
// exp(l - m) for l <= m; 1 where both are the same infinity.
__device__ __forceinline__ float exp_below(float l, float m) { return l == m ? 1.f : expf(l - m); }

// The experts chosen for one token by a warp: lane j < k returns the j-th one's index, or -1 where the allowed ones ran out.
// l: logits of the lane's experts (NaN replaced by -infinity), allow: which of them may be chosen, s_choice: E doubles of the warp's own.
template <int N>
__device__ __forceinline__ int route_choose(const RouteGate& g, const float (&l)[N], const float* bias, uint32_t allow, int E, int k,
                                            double* s_choice) {
  const int lane = threadIdx.x & 31, e0 = lane * N;
  unsigned long long key[N];
  const bool groups = g.n_groups > 1;
  const bool by_score = bias != nullptr || (groups && g.group_top > 1);
  double c[N];
  if (by_score) {
    double total = 0.0, m = 0.0;
    if (g.score == SWAPMOE_SCORE_SOFTMAX) {
      float mf = -CUDART_INF_F;
#pragma unroll
      for (int i = 0; i < N; ++i) mf = fmaxf(mf, (allow >> i) & 1u ? l[i] : -CUDART_INF_F);
      m = (double)warp_max(mf);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const double x = (double)l[i];
      if (g.score == SWAPMOE_SCORE_SOFTMAX) {
        c[i] = (allow >> i) & 1u ? (x == m ? 1.0 : exp(x - m)) : 0.0;
        total += c[i];
      } else {
        c[i] = 1.0 / (1.0 + exp(-x));
      }
    }
    if (g.score == SWAPMOE_SCORE_SOFTMAX) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
#pragma unroll
      for (int i = 0; i < N; ++i) c[i] /= total;
    }
    if (bias != nullptr)
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (e0 + i < E) c[i] += (double)bias[e0 + i];
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) c[i] = (double)l[i];
  }
#pragma unroll
  for (int i = 0; i < N; ++i) key[i] = (allow >> i) & 1u ? choice_key(c[i]) : 0ull;
  if (groups) {
    // lane g values group g
    __syncwarp();
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (e0 + i < E) s_choice[e0 + i] = (allow >> i) & 1u ? c[i] : CUDART_NAN;      // NaN: not to be chosen
    __syncwarp();
    unsigned long long value = 0ull;
    int have = 0;
    if (lane < g.n_groups) {
      unsigned long long k1 = 0ull, k2 = 0ull;
      double v1 = 0.0, v2 = 0.0;
      for (int i = 0; i < g.group_size; ++i) {
        const double v = s_choice[lane * g.group_size + i];
        if (v != v) continue;
        ++have;
        const unsigned long long kv = choice_key(v);
        if (kv > k1) { k2 = k1; v2 = v1; k1 = kv; v1 = v; }
        else if (kv > k2) { k2 = kv; v2 = v; }
      }
      if (have > 0) value = choice_key(g.group_top > 1 && have > 1 ? v1 + v2 : v1);
    }
    uint32_t kept = 0u;
    for (int taken = 0, pool = 0; taken < g.topk_groups || pool < k; ++taken) {
      const unsigned long long best = warp_max_key(value);
      if (best == 0ull) break;
      const int winner = __ffs(__ballot_sync(0xffffffffu, value == best)) - 1;
      kept |= 1u << winner;
      pool += __shfl_sync(0xffffffffu, have, winner);
      if (lane == winner) value = 0ull;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (!((kept >> (__umulhi(2u * (uint32_t)(e0 + i), g.group_magic) & 31u)) & 1u)) key[i] = 0ull;
  }
  int mine = -1;
  for (int j = 0; j < k; ++j) {
    unsigned long long best = key[0];
#pragma unroll
    for (int i = 1; i < N; ++i) best = key[i] > best ? key[i] : best;
    const unsigned long long top = warp_max_key(best);
    if (top == 0ull) break;
    const int winner = __ffs(__ballot_sync(0xffffffffu, best == top)) - 1;
    int at = 0;
#pragma unroll
    for (int i = N - 1; i >= 0; --i) at = key[i] == top ? i : at;
    const int e = __shfl_sync(0xffffffffu, e0 + at, winner);
    if (lane == winner)
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (i == at) key[i] = 0ull;
    if (lane == j) mine = e;
  }
  return mine;
}

// Weight of the chosen expert of every lane j < k (`chosen` < 0: none, weight 0) from its logit lc.
template <int N>
__device__ __forceinline__ float route_weight(const RouteGate& g, const float (&l)[N], uint32_t allow, int chosen, float lc) {
  const float low = -CUDART_INF_F;
  float w;
  if (g.renorm) {
    // s / sum of s from values relative to the largest chosen one: scores far below 1 keep their ratios
    const float m = warp_max(chosen >= 0 ? lc : low);
    if (g.score == SWAPMOE_SCORE_SOFTMAX) w = exp_below(lc, m);
    else w = m >= 0.f ? 1.f / (1.f + expf(-lc)) : exp_below(lc, m) / (1.f + expf(lc));
    w = chosen >= 0 ? w : 0.f;
    const float sum = warp_sum(w);
    w = w / sum;
  } else if (g.score == SWAPMOE_SCORE_SOFTMAX) {
    float m = low;
#pragma unroll
    for (int i = 0; i < N; ++i) m = fmaxf(m, (allow >> i) & 1u ? l[i] : low);
    m = warp_max(m);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) sum += (allow >> i) & 1u ? exp_below(l[i], m) : 0.f;
    w = exp_below(lc, m) / warp_sum(sum);
  } else {
    w = 1.f / (1.f + expf(-lc));
  }
  return chosen >= 0 ? w * g.scale : 0.f;
}

template <int N>
__global__ void __launch_bounds__(kRouteWarps * 32) route_groups_kernel(const RouteGroupsArgs a) {
  __shared__ double s_choice[kRouteWarps][32 * N];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long token = (long long)blockIdx.x * kRouteWarps + warp;
  pdl_wait();
  pdl_trigger();
  if (token >= a.T) return;
  const float* row = a.logits + token * a.stride;
  float l[N];
  uint32_t allow = 0u;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int e = lane * N + i;
    l[i] = -CUDART_INF_F;
    if (e < a.E) {
      l[i] = fmaxf(row[e], -CUDART_INF_F);
      if (a.expert_to_slot == nullptr || a.expert_to_slot[e] >= 0) allow |= 1u << i;
    }
  }
  const int e = route_choose<N>(a.gate, l, a.bias, allow, a.E, a.k, s_choice[warp]);
  const float lc = e >= 0 ? fmaxf(row[e], -CUDART_INF_F) : -CUDART_INF_F;
  const float w = route_weight<N>(a.gate, l, allow, e, lc);
  if (lane < a.k) {
    a.experts[token * a.k + lane] = e;
    a.weights[token * a.k + lane] = w;
    if (a.slots != nullptr) a.slots[token * a.k + lane] = e >= 0 ? a.expert_to_slot[e] : -1;
  }
}

inline cudaError_t route_groups_launch(const RouteGroupsArgs& a, cudaStream_t st, bool pdl) {
  const dim3 grid((unsigned)((a.T + kRouteWarps - 1) / kRouteWarps)), block(kRouteWarps * 32);
  auto go = [&](auto kernel) { return launch_kernel(kernel, grid, block, 0, st, pdl, a); };
  return a.E <= 32 ? go(route_groups_kernel<1>) : a.E <= 64 ? go(route_groups_kernel<2>) : a.E <= 128 ? go(route_groups_kernel<4>)
       : a.E <= 256 ? go(route_groups_kernel<8>) : go(route_groups_kernel<16>);
}

}  // namespace swapmoe
