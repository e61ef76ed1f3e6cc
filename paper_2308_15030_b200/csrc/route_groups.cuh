// Routing from logits: softmax or sigmoid scores s, a bias b that balances the experts' load, groups of experts, top-k,
// renormalised weights.  Per token, over the experts it may use (with a slot table the resident ones, Masked Gating):
//   c_e = s_e + b_e;  value of a group = sum of its group_top largest c;  the topk_groups best groups are kept, and further ones as
//   long as they hold fewer than k experts to choose from;  the k largest c of the kept groups are chosen, ties to the lowest
//   index;  weight = scale * s_e, or scale * s_e / sum of the chosen s.
//
// A warp routes a token; lane l holds the experts l * N ... l * N + N - 1, so the order of lanes is that of indices and a tie goes to
// the lowest lane.  The order of the choices is that of 64-bit scores: of thousands of tokens some have two experts closer than
// fp32 tells apart.  Without a bias, and with groups valued by their best expert, it is that of the logits themselves.
//
// Bound by instructions, not by bytes (a row is 4 E bytes; 16384 x 256 with eight groups, a bias and top-8: 25.2 us, 2.8 of bytes,
// about 1000 instructions per token): so scores are fp32, and where a choice hangs on a gap that is not clear of their error the
// experts or groups in doubt are compared in 64 bits, a lane each; only what that cannot settle is routed again with all scores in
// 64 bits (one token's worth of that takes some 10 us on its own; with 64 bits for all tokens 60 us).  Each lane sorts its experts
// once, with their places in the keys' last bits; then a choice is one warp reduction, one vote and a step down the winner's list.
#pragma once
#include <math_constants.h>

#include <cmath>

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

// Checks a gate for layers of E experts and top_k of them per token.
inline bool route_gate_from(const swapmoe_gate_t& g, int E, int top_k, RouteGate* out) {
  if (g.score != SWAPMOE_SCORE_SOFTMAX && g.score != SWAPMOE_SCORE_SIGMOID) return false;
  if (g.n_groups < 1 || g.n_groups > kRouteMaxGroups || g.n_groups > E || E % g.n_groups) return false;
  if (g.topk_groups < 1 || g.topk_groups > g.n_groups || g.topk_groups * (E / g.n_groups) < top_k) return false;
  if ((g.group_top != 1 && g.group_top != 2) || (g.renorm != 0 && g.renorm != 1) || !std::isfinite(g.scale)) return false;
  out->score = g.score; out->n_groups = g.n_groups; out->topk_groups = g.topk_groups; out->group_top = g.group_top;
  out->renorm = g.renorm; out->scale = g.scale;
  out->group_size = E / g.n_groups;
  out->group_magic = (uint32_t)((0x80000000ull + out->group_size - 1) / out->group_size);
  return true;
}

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
__device__ __forceinline__ float warp_max(float v) {              // (not for NaN)
  return gate_key_value(__reduce_max_sync(0xffffffffu, gate_key(v)));
}
// exp(l - m) for l <= m; 1 where both are the same infinity.
__device__ __forceinline__ float exp_below(float l, float m) { return l == m ? 1.f : expf(l - m); }

// Lanes per group where groups are whole runs of 2^i lanes, else 0.
__host__ __device__ constexpr int route_group_lanes(int group_size, int n) {
  const int lanes = group_size % n == 0 ? group_size / n : 0;
  return lanes > 0 && (lanes & (lanes - 1)) == 0 && lanes <= 32 ? lanes : 0;
}

// The experts chosen for one token by a warp: lane j < k returns the j-th one's index, or -1 where the allowed ones ran out.
// row: logits, allow: which of the lane's experts may be chosen, s_choice: E doubles of the warp's own.  In 64 bits, out of line.
template <int N>
static __device__ __noinline__ int route_choose_exact(const RouteGate& g, const float* row, const float* bias, uint32_t allow, int E,
                                                      int k, double* s_choice) {
  const int lane = threadIdx.x & 31, e0 = lane * N;
  float l[N];
#pragma unroll
  for (int i = 0; i < N; ++i) l[i] = e0 + i < E ? fmaxf(row[e0 + i], -CUDART_INF_F) : -CUDART_INF_F;
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
    // lane g values group g: groups on whole runs of lanes from the lanes' two best choices, others from shared memory
    unsigned long long value = 0ull;
    int have = 0;
    const int lanes = route_group_lanes(g.group_size, N);
    double v1 = -CUDART_INF, v2 = -CUDART_INF;
    if (lanes > 0) {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if ((allow >> i) & 1u) {
          const double v = c[i] == c[i] ? c[i] : -CUDART_INF;
          v2 = fmax(v2, fmin(v1, v));
          v1 = fmax(v1, v);
          ++have;
        }
      for (int o = 1; o < lanes; o <<= 1) {
        const double w1 = __shfl_xor_sync(0xffffffffu, v1, o), w2 = __shfl_xor_sync(0xffffffffu, v2, o);
        have += __shfl_xor_sync(0xffffffffu, have, o);
        v2 = fmax(fmin(v1, w1), fmax(v2, w2));
        v1 = fmax(v1, w1);
      }
      const int from = min(lane * lanes, 31);
      v1 = __shfl_sync(0xffffffffu, v1, from);
      v2 = __shfl_sync(0xffffffffu, v2, from);
      have = __shfl_sync(0xffffffffu, have, from);
      if (lane >= g.n_groups) have = 0;
    } else {
      __syncwarp();
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (e0 + i < E) s_choice[e0 + i] = !((allow >> i) & 1u) ? CUDART_NAN : c[i] == c[i] ? c[i] : -CUDART_INF;   // NaN: not to be chosen
      __syncwarp();
      if (lane < g.n_groups)
        for (int i = 0; i < g.group_size; ++i) {
          const double v = s_choice[lane * g.group_size + i];
          if (v != v) continue;
          ++have;
          v2 = fmax(v2, fmin(v1, v));
          v1 = fmax(v1, v);
        }
    }
    if (have > 0) value = choice_key(g.group_top > 1 && have > 1 ? v1 + v2 : v1);
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

// ----------------------------------------------------------------------------- fp32, with a check of the gaps
// 2^x and 1 / x by the hardware's approximations (errors 2^-22 and 2^-23), denormal results as 0.
__device__ __forceinline__ float fast_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float fast_reciprocal(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__host__ __device__ constexpr int route_pow2(int n) { return n <= 1 ? 1 : n <= 2 ? 2 : n <= 4 ? 4 : n <= 8 ? 8 : 16; }

// Descending order of M = 2^m keys (Batcher's odd-even merge sort: 19 exchanges for eight, 63 for sixteen).
template <int M>
__device__ __forceinline__ void sort_keys(uint32_t (&k)[M]) {
#pragma unroll
  for (int p = 1; p < M; p *= 2)
#pragma unroll
    for (int h = p; h >= 1; h /= 2)
#pragma unroll
      for (int j = h % p; j + h < M; j += 2 * h)
#pragma unroll
        for (int i = 0; i < h; ++i)
          if (i + j + h < M && (i + j) / (2 * p) == (i + j + h) / (2 * p)) {
            const uint32_t x = k[i + j], y = k[i + j + h];
            k[i + j] = max(x, y);
            k[i + j + h] = min(x, y);
          }
}

// What a warp keeps for all its tokens: which of the lane's experts may be chosen (bits, and masks of their keys), and how many of
// the lane's group.
template <int N>
struct RouteLane {
  uint32_t allow;
  uint32_t mask[N];
  bool all;                  // no table: every expert may be chosen
  int have;                  // aligned groups: allowed experts of the lane's group
};

__device__ __forceinline__ uint32_t magnitude_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

template <int N>
__device__ __forceinline__ RouteLane<N> route_lane(const RouteGate& g, const int32_t* expert_to_slot, int E) {
  const int lane = threadIdx.x & 31;
  RouteLane<N> r;
  r.allow = 0u;
  r.all = expert_to_slot == nullptr;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int e = lane * N + i;
    const bool may = e < E && (expert_to_slot == nullptr || expert_to_slot[e] >= 0);
    r.allow |= (may ? 1u : 0u) << i;
    r.mask[i] = may ? 0xffffffffu : 0u;
  }
  r.have = __popc(r.allow);
  const int lanes = route_group_lanes(g.group_size, N);
  for (int o = 1; o < lanes; o <<= 1) r.have += __shfl_xor_sync(0xffffffffu, r.have, o);
  return r;
}

// As route_choose_exact, from the lane's logits l (NaN replaced by -infinity) and biases b.  s_list: 32 M + 64 words of the warp's own.  *clear: no gap that the
// choice hangs on is within the error of what was compared; if not, the result is not to be used.
template <int N>
__device__ __forceinline__ int route_choose_fast(const RouteGate& g, const float (&l)[N], const float (&b)[N], bool with_bias,
                                                 const RouteLane<N>& rl, int E, int k, const float* row, const float* bias, float* s_choice,
                                                 uint32_t* s_list, bool* clear) {
  constexpr int M = route_pow2(N);
  constexpr uint32_t kPlace = M - 1;                        // bits of a key that hold the expert's place (first places larger)
  const int lane = threadIdx.x & 31, e0 = lane * N;
  const bool groups = g.n_groups > 1 && g.topk_groups < g.n_groups;
  const bool by_score = with_bias || (g.n_groups > 1 && g.group_top > 1);
  float c[N], error = 0.f;                                  // error: bound on a choice's, but for its own rounding
  if (by_score) {
    if (g.score == SWAPMOE_SCORE_SOFTMAX) {
      float m = -CUDART_INF_F, sum = 0.f;
#pragma unroll
      for (int i = 0; i < N; ++i) m = fmaxf(m, (rl.allow >> i) & 1u ? l[i] : -CUDART_INF_F);
      m = warp_max(m);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        c[i] = (rl.allow >> i) & 1u ? (l[i] == m ? 1.f : fast_exp2((l[i] - m) * 1.44269504f)) : 0.f;
        sum += c[i];
      }
      const float inv = 1.f / warp_sum(sum);
#pragma unroll
      for (int i = 0; i < N; ++i) c[i] *= inv;
      // exponentials: (2 + |x|) 2^-22 of themselves, that is 5e-7 of the largest score (1 / sum) where it counts; sums of up to 21
      // steps, reciprocal and product: 24 x 2^-24 of the score
      error = 2e-6f * inv;
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) c[i] = fast_reciprocal(1.f + fast_exp2(l[i] * -1.44269504f));
      // exponential: |x| 2^-23 from its argument and 2^-22 of itself, times s (1 - s): below 2e-7; two roundings and the reciprocal's 2^-23
      error = 5e-7f;
    }
    if (with_bias)
#pragma unroll
      for (int i = 0; i < N; ++i) c[i] += b[i];
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) c[i] = l[i] + 0.f;                      // (-0 becomes +0)
  }
  uint32_t key[M];
#pragma unroll
  for (int i = 0; i < M; ++i) {
    key[i] = 0u;
    if (i < N) {
      const uint32_t u = __float_as_uint(fmaxf(c[i < N ? i : 0], -CUDART_INF_F));         // NaN (of a bias) as -infinity
      key[i] = (((u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u)) & ~kPlace) | (kPlace - i)) & rl.mask[i < N ? i : 0];
    }
  }
  // (without its place bits the key of -infinity is that of a NaN)
  auto value_of = [&](uint32_t q) { return fmaxf(gate_key_value(q & ~kPlace), -CUDART_INF_F); };
  constexpr float kCut = 2.f * M * 0x1p-23f;                // what the places cost a pair of keys, and the roundings, relative
  float group_size = 0.f;
  uint32_t group_at = 0u, choice_at = 0u;                   // lane i: key of the i-th group, of the i-th choice (0: none)
  const int lanes = groups ? route_group_lanes(g.group_size, N) : 0;
  if (groups && lanes == 0) {
    // groups that do not lie on whole runs of lanes: lane q values group q from shared memory
    __syncwarp();
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (e0 + i < E) s_choice[e0 + i] = (rl.allow >> i) & 1u ? fmaxf(c[i], -CUDART_INF_F) : CUDART_NAN_F;
    __syncwarp();
  }
  if (lanes > 0) sort_keys<M>(key);
  if (groups) {
    float v1 = -CUDART_INF_F, v2 = -CUDART_INF_F;
    int have = rl.have;
    if (lanes > 0) {
      v1 = key[0] ? value_of(key[0]) : -CUDART_INF_F;
      if (M > 1) v2 = key[M > 1 ? 1 : 0] ? value_of(key[M > 1 ? 1 : 0]) : -CUDART_INF_F;
      for (int o = 1; o < lanes; o <<= 1) {
        const float w1 = __shfl_xor_sync(0xffffffffu, v1, o), w2 = __shfl_xor_sync(0xffffffffu, v2, o);
        v2 = fmaxf(fminf(v1, w1), fmaxf(v2, w2));
        v1 = fmaxf(v1, w1);
      }
      if (e0 >= E) have = 0;
    } else {
      have = 0;
      if (lane < g.n_groups)
        for (int i = 0; i < g.group_size; ++i) {
          const float v = s_choice[lane * g.group_size + i];
          if (v != v) continue;
          ++have;
          v2 = fmaxf(v2, fminf(v1, v));
          v1 = fmaxf(v1, v);
        }
    }
    const bool two = g.group_top > 1 && have > 1;
    const float value = fmaxf(two ? v1 + v2 : v1, -CUDART_INF_F);             // inf - inf as -infinity
    // The error of a sum goes by its terms.  Infinite ones have none: they are clear of finite values, and equal ones of each other
    // never (inf - inf exceeds no slack).
    auto magnitude = [](float v) { return fabsf(v) < CUDART_INF_F ? __float_as_uint(fabsf(v)) : 0u; };
    group_size = __uint_as_float(__reduce_max_sync(0xffffffffu, have == 0 ? 0u : max(magnitude(v1), two ? magnitude(v2) : 0u)));
    uint32_t gk = 0u;
    if (have > 0) {
      const uint32_t u = __float_as_uint(value + 0.f);
      gk = u & 0x80000000u ? ~u : u | 0x80000000u;
    }
    uint32_t kept = 0u;                                     // bit per group, or per lane of aligned groups
    if (rl.all) {
      // topk_groups groups hold k experts: a group is kept if fewer than that many are worth more (equal ones: in front of it).
      // Lane q ranks group q.
      const uint32_t mine = lanes > 0 ? __shfl_sync(0xffffffffu, gk, min(lane * lanes, 31)) : gk;
      int rank = 0;
#pragma unroll 4
      for (int q = 0; q < g.n_groups; ++q) {
        const uint32_t other = __shfl_sync(0xffffffffu, mine, q);
        rank += other > mine || (other == mine && q < lane);
      }
      const bool in = lane < g.n_groups && rank < g.topk_groups;
      const uint32_t in_mask = __ballot_sync(0xffffffffu, in);
      kept = lanes > 0 ? __ballot_sync(0xffffffffu, (in_mask >> (lane / max(lanes, 1))) & 1u) : in_mask;
      // only the border between the two kinds matters: the least of the kept ones and the best of the others
      const uint32_t least = ~__reduce_max_sync(0xffffffffu, in ? ~mine : 0u);
      const uint32_t best = __reduce_max_sync(0xffffffffu, !in && lane < g.n_groups ? mine : 0u);
      group_at = lane == 0 ? least : lane == 1 ? best : 0u;
    } else {
      const uint32_t run = lanes > 0 ? (lanes == 32 ? 0xffffffffu : (1u << lanes) - 1u) : 1u;
#pragma unroll 1
      for (int taken = 0, pool = 0;; ++taken) {
        const uint32_t best = __reduce_max_sync(0xffffffffu, gk);
        if (lane == taken) group_at = best;
        if (best == 0u || (taken >= g.topk_groups && pool >= k)) break;
        const int winner = __ffs(__ballot_sync(0xffffffffu, gk == best)) - 1;
        const uint32_t these = run << winner;
        kept |= these;
        if ((these >> lane) & 1u) gk = 0u;
        pool += __shfl_sync(0xffffffffu, have, winner);
      }
    }
    {
      // groups closer than the error allows: the lanes' two best experts in 64 bits, if no third one can matter, and the groups again
      const uint32_t group_below = __shfl_down_sync(0xffffffffu, group_at, 1);
      const float slack = 4.f * error + 2.f * kCut * group_size;
      const bool near = lane < 31 && group_below != 0u && !(gate_key_value(group_at) - gate_key_value(group_below) > slack);
      if (__any_sync(0xffffffffu, near) && lanes > 0 && !(by_score && g.score == SWAPMOE_SCORE_SOFTMAX)) {
        const bool third = M > 2 && key[M > 2 ? 2 : 0] != 0u && !(v2 - value_of(key[M > 2 ? 2 : 0]) > slack);
        if (!__any_sync(0xffffffffu, third)) {
          double w1 = -CUDART_INF, w2 = -CUDART_INF;
#pragma unroll 1
          for (int i = 0; i < 2; ++i) {
            const uint32_t q = i == 0 ? key[0] : M > 1 ? key[M > 1 ? 1 : 0] : 0u;
            if (q == 0u) continue;
            const int e = e0 + (int)(kPlace - (q & kPlace));
            double x = (double)fmaxf(row[e], -CUDART_INF_F);
            if (by_score) x = 1.0 / (1.0 + exp(-x)) + (bias != nullptr ? (double)bias[e] : 0.0);
            w2 = fmax(w2, fmin(w1, x));
            w1 = fmax(w1, x);
          }
          for (int o = 1; o < lanes; o <<= 1) {
            const double u1 = __shfl_xor_sync(0xffffffffu, w1, o), u2 = __shfl_xor_sync(0xffffffffu, w2, o);
            w2 = fmax(fmin(w1, u1), fmax(w2, u2));
            w1 = fmax(w1, u1);
          }
          unsigned long long exact = have > 0 ? choice_key(g.group_top > 1 && have > 1 ? w1 + w2 : w1) : 0ull;
          kept = 0u;
          for (int taken = 0, pool = 0; taken < g.topk_groups || pool < k; ++taken) {
            const unsigned long long best = warp_max_key(exact);
            if (best == 0ull) break;
            const int winner = __ffs(__ballot_sync(0xffffffffu, exact == best)) - 1;
            const bool in = (lane & ~(lanes - 1)) == winner;
            kept |= __ballot_sync(0xffffffffu, in);
            pool += __shfl_sync(0xffffffffu, have, winner);
            if (in) exact = 0ull;
          }
          group_at = 0u;                                    // settled
        }
      }
    }
    if (lanes > 0) {
      if (!((kept >> lane) & 1u))
#pragma unroll
        for (int i = 0; i < M; ++i) key[i] = 0u;
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (!((kept >> (__umulhi(2u * (uint32_t)(e0 + i), g.group_magic) & 31u)) & 1u)) key[i] = 0u;
    }
  }
  if (lanes == 0) sort_keys<M>(key);
  // the lists' heads in registers, what is behind them in shared memory: the winner reads its next one
  uint32_t* const list = s_list + lane * M;
  __syncwarp();
  if constexpr (M >= 4) {
#pragma unroll
    for (int i = 0; i < M; i += 4) *reinterpret_cast<uint4*>(list + i) = make_uint4(key[i], key[i + 1], key[i + 2], key[i + 3]);
  } else {
#pragma unroll
    for (int i = 0; i < M; ++i) list[i] = key[i];
  }
  int mine = -1, at = 0;
  uint32_t head = key[0];
#pragma unroll 1
  for (int j = 0; j < k; ++j) {
    const uint32_t top = __reduce_max_sync(0xffffffffu, head);
    if (top == 0u) break;
    const int winner = __ffs(__ballot_sync(0xffffffffu, head == top)) - 1;
    if (lane == j) { choice_at = top; mine = winner; }
    if (lane == winner) head = ++at < M ? list[at] : 0u;
  }
  const uint32_t behind = __reduce_max_sync(0xffffffffu, head);       // the best one that was not chosen
  if (lane == k) choice_at = behind;
  if (mine >= 0) mine = mine * N + (int)(kPlace - (choice_at & kPlace));
  // the gaps between neighbours of the two lists, and the largest magnitude among the choices (an infinity there: 64 bits decide)
  const uint32_t below = __shfl_down_sync(0xffffffffu, choice_at, 1), group_below = __shfl_down_sync(0xffffffffu, group_at, 1);
  const float v = value_of(choice_at), w = gate_key_value(group_at);
  const uint32_t size = __reduce_max_sync(0xffffffffu, choice_at != 0u ? magnitude_bits(v) : 0u);
  const float slack = 2.f * error + kCut * __uint_as_float(size);
  const float group_slack = 4.f * error + 2.f * kCut * group_size;
  const bool finite = size < 0x7f800000u;
  const bool near_group = lane < 31 && group_below != 0u && !(w - gate_key_value(group_below) > group_slack);
  const bool near = lane < k && below != 0u && !(v - value_of(below) > slack);
  *clear = !__any_sync(0xffffffffu, near || near_group) && finite;
  if (*clear || __any_sync(0xffffffffu, near_group) || !finite || (by_score && g.score == SWAPMOE_SCORE_SOFTMAX)) return mine;
  // Only the order within the list is in doubt, if the best one that was not chosen is clear of the next one: then 64-bit values of
  // the list's k + 1 experts settle it, a lane each.
  const int winner = __ffs(__ballot_sync(0xffffffffu, head == behind)) - 1;
  if (lane == winner) head = ++at < M ? list[at] : 0u;
  const uint32_t next = __reduce_max_sync(0xffffffffu, head);
  if (behind != 0u && next != 0u && !(value_of(behind) - value_of(next) > slack)) return mine;
  if (lane == k) mine = behind != 0u ? winner * N + (int)(kPlace - (behind & kPlace)) : -1;
  unsigned long long exact = 0ull;
  if (lane <= k && mine >= 0) {
    const double x = (double)fmaxf(row[mine], -CUDART_INF_F);
    exact = choice_key(!by_score ? x : 1.0 / (1.0 + exp(-x)) + (bias != nullptr ? (double)bias[mine] : 0.0));
  }
  int rank = 0;
  for (int i = 0; i <= k; ++i) {
    const unsigned long long other = __shfl_sync(0xffffffffu, exact, i);
    const int e = __shfl_sync(0xffffffffu, mine, i);
    rank += other > exact || (other == exact && e < mine && other != 0ull);
  }
  __syncwarp();
  if (lane <= k) s_list[exact != 0ull ? rank : 32 + lane] = (uint32_t)mine;      // (places of those that do not exist: nobody's)
  const int chosen = __popc(__ballot_sync(0xffffffffu, lane <= k && exact != 0ull));
  __syncwarp();
  mine = lane < min(k, chosen) ? (int)s_list[lane] : -1;
  __syncwarp();
  *clear = true;
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
    // (quotients by __fdividef: denominators are at least 0.5; where 1 + exp(-l) leaves its range, beyond 2^126, the score is 0)
    if (g.score == SWAPMOE_SCORE_SOFTMAX) w = exp_below(lc, m);
    else w = m >= 0.f ? __fdividef(1.f, 1.f + expf(-lc)) : __fdividef(exp_below(lc, m), 1.f + expf(lc));
    w = chosen >= 0 ? w : 0.f;
    w = __fdividef(w, warp_sum(w));
  } else if (g.score == SWAPMOE_SCORE_SOFTMAX) {
    float m = low;
#pragma unroll
    for (int i = 0; i < N; ++i) m = fmaxf(m, (allow >> i) & 1u ? l[i] : low);
    m = warp_max(m);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) sum += (allow >> i) & 1u ? exp_below(l[i], m) : 0.f;
    w = __fdividef(exp_below(lc, m), warp_sum(sum));
  } else {
    w = __fdividef(1.f, 1.f + expf(-lc));
  }
  return chosen >= 0 ? w * g.scale : 0.f;
}

// One row's logits of the lane's experts, NaN as -infinity.  vec: rows start at multiples of 16 bytes and E is a multiple of N.
template <int N>
__device__ __forceinline__ void route_load(const float* row, int E, bool vec, float (&l)[N]) {
  const int e0 = (threadIdx.x & 31) * N;
  if constexpr (N % 4 == 0) {
    if (vec) {
#pragma unroll
      for (int i = 0; i < N; i += 4) {
        float4 v = make_float4(-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F);
        if (e0 < E) v = *reinterpret_cast<const float4*>(row + e0 + i);
        l[i] = v.x; l[i + 1] = v.y; l[i + 2] = v.z; l[i + 3] = v.w;
      }
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) l[i] = e0 + i < E ? row[e0 + i] : -CUDART_INF_F;
}

template <int N>
__global__ void __launch_bounds__(kRouteWarps * 32, N <= 8 ? 8 : 4) route_groups_kernel(const __grid_constant__ RouteGroupsArgs a, int vec) {
  __shared__ double s_choice[kRouteWarps][32 * N];
  __shared__ __align__(16) uint32_t s_list[kRouteWarps][32 * route_pow2(N) + 64];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  pdl_wait();
  pdl_trigger();
  long long token = (long long)blockIdx.x * kRouteWarps + warp;
  if (token >= a.T) return;
  const long long step = (long long)gridDim.x * kRouteWarps;
  const float* row = a.logits + token * a.stride;
  float l[N], next[N], b[N];
  route_load<N>(row, a.E, vec, next);
  const RouteLane<N> rl = route_lane<N>(a.gate, a.expert_to_slot, a.E);
#pragma unroll
  for (int i = 0; i < N; ++i) b[i] = a.bias != nullptr && lane * N + i < a.E ? a.bias[lane * N + i] : 0.f;
  auto write = [&](long long t, int e, float w) {
    if (lane < a.k) {
      a.experts[t * a.k + lane] = e;
      a.weights[t * a.k + lane] = w;
      if (a.slots != nullptr) a.slots[t * a.k + lane] = e >= 0 ? a.expert_to_slot[e] : -1;
    }
  };
  auto logit = [&](const float* r, int e) { return e >= 0 ? fmaxf(r[e], -CUDART_INF_F) : -CUDART_INF_F; };
  // Tokens that need 64 bits throughout are noted and routed behind the others, 64 tokens at a time: with a call in the loop over the tokens, whatever
  // it calls, more registers spill (16384 x 256: 30 us, 25 so; at eight experts per lane 116 bytes are spilled even so).
#pragma unroll 1
  while (token < a.T) {
    const long long first = token;
    unsigned long long unclear = 0ull;
#pragma unroll 1
    for (int i = 0; i < 64 && token < a.T; ++i, token += step, row += step * a.stride) {
#pragma unroll
      for (int j = 0; j < N; ++j) l[j] = fmaxf(next[j], -CUDART_INF_F);
      if (token + step < a.T) route_load<N>(row + step * a.stride, a.E, vec, next);
      bool clear;
      const int e = route_choose_fast<N>(a.gate, l, b, a.bias != nullptr, rl, a.E, a.k, row, a.bias, reinterpret_cast<float*>(s_choice[warp]),
                                         s_list[warp], &clear);
      if (!clear) { unclear |= 1ull << i; continue; }
      write(token, e, route_weight<N>(a.gate, l, rl.allow, e, logit(row, e)));
    }
#pragma unroll 1
    for (; unclear != 0ull; unclear &= unclear - 1) {
      const long long t = first + (__ffsll((long long)unclear) - 1) * step;
      const float* r = a.logits + t * a.stride;
      const int e = route_choose_exact<N>(a.gate, r, a.bias, rl.allow, a.E, a.k, s_choice[warp]);
      route_load<N>(r, a.E, false, l);
#pragma unroll
      for (int j = 0; j < N; ++j) l[j] = fmaxf(l[j], -CUDART_INF_F);
      write(t, e, route_weight<N>(a.gate, l, rl.allow, e, logit(r, e)));
    }
  }
}

// Experts per lane: the fewest that hold E, or a few more where groups then lie on whole runs of lanes.
constexpr int kRouteSizes[] = {1, 2, 3, 4, 5, 6, 8, 12, 16};
inline int route_lane_experts(int E, int n_groups) {
  int pick = 0;
  for (int n : kRouteSizes) {
    if (32 * n < E) continue;
    if (pick == 0) pick = n;
    if (n_groups > 1 && n <= 2 * pick && route_group_lanes(E / n_groups, n) > 0) return n;
  }
  return pick;
}

inline cudaError_t route_groups_launch(const RouteGroupsArgs& a, int sm_count, cudaStream_t st, bool pdl) {
  const int n = route_lane_experts(a.E, a.gate.n_groups);
  // every warp a token while they last; beyond what the chip holds at once they walk through several (the next row is on its way meanwhile)
  const long long ctas = ((long long)a.T + kRouteWarps - 1) / kRouteWarps, most = (n <= 8 ? 8ll : 4ll) * (sm_count > 0 ? sm_count : 1);
  const dim3 grid((unsigned)(ctas < most ? ctas : most)), block(kRouteWarps * 32);
  const int vec = a.stride % 4 == 0 && reinterpret_cast<uintptr_t>(a.logits) % 16 == 0 && a.E % n == 0;
  auto go = [&](auto kernel) { return launch_kernel(kernel, grid, block, 0, st, pdl, a, vec); };
  switch (n) {
    case 1: return go(route_groups_kernel<1>);
    case 2: return go(route_groups_kernel<2>);
    case 3: return go(route_groups_kernel<3>);
    case 4: return go(route_groups_kernel<4>);
    case 5: return go(route_groups_kernel<5>);
    case 6: return go(route_groups_kernel<6>);
    case 8: return go(route_groups_kernel<8>);
    case 12: return go(route_groups_kernel<12>);
    default: return go(route_groups_kernel<16>);
  }
}

}  // namespace swapmoe
