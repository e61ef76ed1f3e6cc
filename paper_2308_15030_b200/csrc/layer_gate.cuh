// The gate of a layer with a gate of its own (swapmoe_set_gate): both selections of every token - over all experts (feeds Eq. 1)
// and over the resident ones (Masked Gating) - from the logits that the router kernel left, by the routing of
// route_groups.cuh, and the per-CTA partial sums that the permutation starts from.  The router's own gate has run too; what it
// wrote is overwritten.
#pragma once
#include "permute.cuh"
#include "route_groups.cuh"
#include "router_args.cuh"

namespace swapmoe {

static_assert(kMaxE <= 256, "experts per lane of layer_gate_launch");

constexpr int kLayerGateWarps = 8, kLayerGateThreads = kLayerGateWarps * 32, kLayerGateTok = 32;

// a: the router's arguments with the scan of this kernel's CTAs; tok: tokens per CTA (8, 16 or 32).  A warp routes tok / 8 tokens.
template <int N>
__global__ void __launch_bounds__(kLayerGateThreads) layer_gate_kernel(const __grid_constant__ RouterArgs a,
                                                                        const __grid_constant__ RouteGate gate, const float* bias, int tok) {
  __shared__ double s_choice[kLayerGateWarps][32 * N];
  __shared__ __align__(16) uint32_t s_list[kLayerGateWarps][32 * route_pow2(N) + 64];
  __shared__ __align__(16) int s_e[kLayerGateTok * kMaxTopK], s_s[kLayerGateTok * kMaxTopK];      // expert, slot per pair
  __shared__ __align__(16) float s_t[kLayerGateTok * kMaxTopK], s_m[kLayerGateTok * kMaxTopK];    // Eq. (1) terms of both routings
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, E = a.E, k = a.k;
  pdl_wait();
  pdl_trigger();
  const int tok0 = blockIdx.x * tok;
  const RouteLane<N> any = route_lane<N>(gate, nullptr, E), resident = route_lane<N>(gate, a.e2s, E);
  float b[N];
#pragma unroll
  for (int i = 0; i < N; ++i) b[i] = bias != nullptr && lane * N + i < E ? bias[lane * N + i] : 0.f;
#pragma unroll 1
  for (int t = warp; t < tok; t += kLayerGateWarps) {
    const int token = tok0 + t;
    if (token >= a.T) {
      if (lane < k) { s_e[t * k + lane] = s_s[t * k + lane] = -1; s_t[t * k + lane] = s_m[t * k + lane] = 0.f; }
      continue;
    }
    const float* row = a.logits + (size_t)token * E;
    const float xn = a.xnorm[token];
    float l[N];
    route_load<N>(row, E, false, l);
#pragma unroll
    for (int i = 0; i < N; ++i) l[i] = fmaxf(l[i], -CUDART_INF_F);
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {
      RouteLane<N> rl = any;
      if (pass == 1) rl = resident;
      bool clear;
      int e = route_choose_fast<N>(gate, l, b, bias != nullptr, rl, E, k, row, bias, reinterpret_cast<float*>(s_choice[warp]), s_list[warp], &clear);
      if (!clear) e = route_choose_exact<N>(gate, row, bias, rl.allow, E, k, s_choice[warp]);
      const float w = route_weight<N>(gate, l, rl.allow, e, e >= 0 ? fmaxf(row[e], -CUDART_INF_F) : -CUDART_INF_F);
      if (lane < k) {
        const int p = t * k + lane;
        const size_t gp = (size_t)token * k + lane;
        const float term = xn * fabsf(w) * (e >= 0 ? a.enorm[e] : 0.f);
        if (pass == 0) {
          a.uidx[gp] = e; a.ugate[gp] = w;
          s_e[p] = e; s_t[p] = term;
        } else {
          const int slot = e >= 0 ? a.e2s[e] : -1;
          a.midx[gp] = e; a.mgate[gp] = w; a.slot[gp] = slot;
          s_s[p] = slot; s_m[p] = term;
        }
      }
    }
  }
  __syncthreads();
  // partial sums, pairs in order (as the routers' gates): a thread owns an expert or a slot
  const int pairs = tok * k;
  for (int c = tid; c < E + a.K; c += kLayerGateThreads) {
    const bool by_slot = c >= E;
    const int id = by_slot ? c - E : c;
    const int4* ids = reinterpret_cast<const int4*>(by_slot ? s_s : s_e);
    const float4* terms = reinterpret_cast<const float4*>(by_slot ? s_m : s_t);
    float sum = 0.f;
    int n = 0;
#pragma unroll 4
    for (int q = 0; q < pairs / 4; ++q) {
      const int4 i4 = ids[q];
      const float4 t4 = terms[q];
      if (i4.x == id) { sum += t4.x; ++n; }
      if (i4.y == id) { sum += t4.y; ++n; }
      if (i4.z == id) { sum += t4.z; ++n; }
      if (i4.w == id) { sum += t4.w; ++n; }
    }
    if (by_slot) {
      a.cta_hist[(size_t)blockIdx.x * a.K + id] = n;
      if (a.cta_mimp) a.cta_mimp[(size_t)blockIdx.x * a.K + id] = sum;
    } else {
      a.cta_imp[(size_t)blockIdx.x * E + id] = sum;
      if (a.cta_cnt) a.cta_cnt[(size_t)blockIdx.x * E + id] = (float)n;
    }
  }
  finish_router_cta(a.scan);
}

// Tokens per CTA: one per warp for decode batches, while the layer's workspace has a row of partial sums for every CTA.
inline int layer_gate_tok(int T) { return T <= 64 ? 8 : T <= 16 * 256 ? 16 : kLayerGateTok; }

inline cudaError_t layer_gate_launch(const RouterArgs& a, const RouteGate& gate, const float* bias, int tok, cudaStream_t st, bool pdl) {
  auto go = [&](auto kernel) { return launch_kernel(kernel, dim3(a.scan.n_cta), dim3(kLayerGateThreads), 0, st, pdl, a, gate, bias, tok); };
  switch (route_lane_experts(a.E, gate.n_groups)) {
    case 1: return go(layer_gate_kernel<1>);
    case 2: return go(layer_gate_kernel<2>);
    case 3: return go(layer_gate_kernel<3>);
    case 4: return go(layer_gate_kernel<4>);
    case 5: return go(layer_gate_kernel<5>);
    case 6: return go(layer_gate_kernel<6>);
    case 8: return go(layer_gate_kernel<8>);
    default: return go(layer_gate_kernel<12>);       // (up to 256 experts: no more than twelve per lane)
  }
}

}  // namespace swapmoe
