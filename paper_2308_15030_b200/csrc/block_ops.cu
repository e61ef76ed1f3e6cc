// C ABI of the operators around the experts of a served MoE block (see include/swapmoe.h): argument checks and launches.
#include "../../include/swapmoe.h"

#include <cuda_runtime.h>

#include <cmath>
#include <initializer_list>
#include <new>

#include "adapters.cuh"
#include "block_ops.cuh"
#include "common.cuh"
#include "rms_norm.cuh"
#include "route_groups.cuh"

using namespace swapmoe;

static_assert(SWAPMOE_NORM_MAX_WIDTH == kNormMaxWidth, "the header's limit");

struct swapmoe_adapters {
  swapmoe_adapters_config_t cfg;
  int sm_count;
  char* ws;                      // workspace: plan of the tiles
  int32_t *perm, *n_tiles;
  AdapterTile* tiles;
  const void *A, *B;
  const float* scale;
};

namespace {

// SMs of the current device, or 0 (the launch that follows then fails by itself).
int current_sm_count() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
    cudaGetLastError();
    return 0;
  }
  return n;
}

int32_t launched(cudaError_t e, int kernels = 0, int64_t* launches = nullptr) {
  if (e == cudaSuccess) e = cudaGetLastError();
  else cudaGetLastError();
  if (e == cudaSuccess && launches) *launches += kernels;
  return e == cudaSuccess ? SWAPMOE_OK : SWAPMOE_ERR_CUDA;
}

// The choice of dependent launches where no layer has made one: that of the process, read once.
bool standalone_pdl() {
  static const bool pdl = dependent_launch();
  return pdl;
}

// Whether rows of `elem`-byte values at p, `stride` values apart, all start on multiples of `bytes`.
bool rows_aligned(const void* p, long long stride, size_t elem, size_t bytes) {
  return reinterpret_cast<uintptr_t>(p) % bytes == 0 && (size_t)stride * elem % bytes == 0;
}

bool misaligned(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes != 0; }

}  // namespace

namespace swapmoe {

int32_t rms_norm_run(const swapmoe_rms_norm_t* p, void* stream, bool pdl, int64_t* launches) {
  if (!p || p->n_rows < 0 || p->d < 1) return SWAPMOE_ERR_INVALID_ARG;
  if (p->dtype != SWAPMOE_F32 && p->dtype != SWAPMOE_BF16) return SWAPMOE_ERR_INVALID_ARG;
  if (p->residual_dtype != p->dtype && p->residual_dtype != SWAPMOE_F32) return SWAPMOE_ERR_INVALID_ARG;
  if (p->group != 0 && p->group != 32 && p->group != 64 && p->group != 128 && p->group != 256) return SWAPMOE_ERR_INVALID_ARG;
  if (!(p->eps >= 0.f) || std::isinf(p->eps)) return SWAPMOE_ERR_INVALID_ARG;
  if (p->d > kNormMaxWidth) return SWAPMOE_ERR_UNSUPPORTED;
  if (p->n_rows == 0) return SWAPMOE_OK;
  if (!p->x || !p->weight || (!p->out && !p->out8 && !p->residual_out) || (p->residual_out && !p->residual) ||
      (p->out8 == nullptr) != (p->scales == nullptr))
    return SWAPMOE_ERR_INVALID_ARG;
  const size_t elem = p->dtype == SWAPMOE_BF16 ? 2 : 4, relem = p->residual_dtype == SWAPMOE_BF16 ? 2 : 4;
  const long long d = p->d, n_scales = p->group ? (d + p->group - 1) / p->group : 1;
  const int32_t n = p->n_rows;
  struct { const void* p; int32_t n; long long stride, width; size_t elem, vec; } rows[] = {
      {p->x, n, p->x_stride, d, elem, 16},
      {p->residual, n, p->residual_stride, d, relem, 16},
      {p->residual_out, n, p->residual_out_stride, d, relem, 16},
      {p->out, n, p->out_stride, d, elem, 16},
      {p->out8, n, p->out8_stride, d, 1, 8},
      {p->scales, n, p->scales_stride, n_scales, 4, 4},
      {p->weight, 1, d, d, elem, 16}};
  bool vec = d % 8 == 0;
  for (const auto& r : rows) {
    if (!r.p) continue;
    if (r.stride < r.width || reinterpret_cast<uintptr_t>(r.p) % r.elem) return SWAPMOE_ERR_INVALID_ARG;
    vec = vec && rows_aligned(r.p, r.n > 1 ? r.stride : 0, r.elem, r.vec);
  }
  RmsNormArgs a;
  a.x = p->x; a.residual = p->residual; a.weight = p->weight;
  a.residual_out = p->residual_out; a.out = p->out;
  a.out8 = static_cast<uint8_t*>(p->out8); a.scales = p->scales;
  a.x_stride = p->x_stride; a.residual_stride = p->residual_stride; a.residual_out_stride = p->residual_out_stride;
  a.out_stride = p->out_stride; a.out8_stride = p->out8_stride; a.scales_stride = p->scales_stride;
  a.T = p->n_rows; a.d = p->d; a.group = p->group; a.eps = p->eps;
  a.warps_per_row = a.rows_per_cta = 1;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int sms = current_sm_count();
  if (p->dtype == SWAPMOE_F32) return launched(rms_norm_launch_typed<float, float>(a, vec, sms, st, pdl), 1, launches);
  if (p->residual_dtype == SWAPMOE_F32) return launched(rms_norm_launch_typed<bf16, float>(a, vec, sms, st, pdl), 1, launches);
  return launched(rms_norm_launch_typed<bf16, bf16>(a, vec, sms, st, pdl), 1, launches);
}

int32_t adapters_run(swapmoe_adapters_t* b, const void* x, int64_t x_stride, const float* x_scales, const int32_t* ids, const void* y,
                     int64_t y_stride, void* out, int64_t out_stride, int32_t T, void* stream, bool pdl, int64_t* launches) {
  if (!b || T < 0) return SWAPMOE_ERR_INVALID_ARG;
  if (T == 0) return SWAPMOE_OK;
  const swapmoe_adapters_config_t& c = b->cfg;
  if (!x || !ids || !out || x_stride < c.d_in || out_stride < c.d_out || (y && y_stride < c.d_out)) return SWAPMOE_ERR_INVALID_ARG;
  if (x_scales && c.dtype != SWAPMOE_BF16) return SWAPMOE_ERR_INVALID_ARG;
  if (!b->A) return SWAPMOE_ERR_NOT_READY;
  if (T > c.max_tokens) return SWAPMOE_ERR_TOO_MANY_TOKENS;
  const size_t elem = c.dtype == SWAPMOE_BF16 ? 2 : 4;
  const long long many = T > 1;
  if (!rows_aligned(x, many * x_stride, x_scales ? 1 : elem, x_scales ? 8 : 16) || !rows_aligned(out, many * out_stride, elem, 16) ||
      (y && !rows_aligned(y, many * y_stride, elem, 16)) || misaligned(ids, 4) || misaligned(x_scales, 4))
    return SWAPMOE_ERR_INVALID_ARG;
  AdapterArgs a;
  a.x = x; a.x_scales = x_scales; a.ids = ids; a.y = y; a.out = out; a.A = b->A; a.B = b->B; a.scale = b->scale;
  a.perm = b->perm; a.tiles = b->tiles; a.n_tiles = b->n_tiles; a.ctas = 1;
  a.x_stride = x_stride; a.y_stride = y_stride; a.out_stride = out_stride;
  a.T = T; a.d = c.d_in; a.n = c.d_out; a.r = c.rank; a.count = c.n_adapters;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  int kernels = 0;
  const cudaError_t e = c.dtype == SWAPMOE_F32 ? adapters_launch<float, float>(a, b->sm_count, st, pdl, &kernels)
                        : x_scales             ? adapters_launch<__nv_fp8_e4m3, bf16>(a, b->sm_count, st, pdl, &kernels)
                                               : adapters_launch<bf16, bf16>(a, b->sm_count, st, pdl, &kernels);
  return launched(e, kernels, launches);
}

}  // namespace swapmoe

extern "C" {

int32_t swapmoe_rms_norm(const swapmoe_rms_norm_t* p, void* stream) { return rms_norm_run(p, stream, standalone_pdl(), nullptr); }

int32_t swapmoe_route(const swapmoe_gate_t* gate, const float* logits, int64_t stride, const float* bias,
                      const int32_t* expert_to_slot, int32_t T, int32_t E, int32_t top_k, int32_t* experts, float* weights,
                      int32_t* slots, void* stream) {
  RouteGroupsArgs a;
  if (!gate || T < 0 || E < 1 || top_k < 1 || top_k > E || stride < E) return SWAPMOE_ERR_INVALID_ARG;
  if (E > kRouteMaxE || top_k > kRouteMaxTopK) return SWAPMOE_ERR_UNSUPPORTED;
  if (!route_gate_from(*gate, E, top_k, &a.gate)) return SWAPMOE_ERR_INVALID_ARG;
  if (T == 0) return SWAPMOE_OK;
  if (!logits || !experts || !weights || (expert_to_slot == nullptr) != (slots == nullptr)) return SWAPMOE_ERR_INVALID_ARG;
  for (const void* p : {(const void*)logits, (const void*)bias, (const void*)expert_to_slot, (const void*)experts, (const void*)weights, (const void*)slots})
    if (misaligned(p, 4)) return SWAPMOE_ERR_INVALID_ARG;
  a.logits = logits; a.bias = bias; a.expert_to_slot = expert_to_slot;
  a.experts = experts; a.weights = weights; a.slots = slots;
  a.stride = stride; a.T = T; a.E = E; a.k = top_k;
  return launched(route_groups_launch(a, current_sm_count(), static_cast<cudaStream_t>(stream), standalone_pdl()));
}

int32_t swapmoe_adapters_create(swapmoe_adapters_t** out, const swapmoe_adapters_config_t* cfg) {
  if (!out || !cfg) return SWAPMOE_ERR_INVALID_ARG;
  const swapmoe_adapters_config_t c = *cfg;
  if (c.n_adapters < 1 || c.d_in < 1 || c.d_out < 1 || c.rank < 1 || c.max_tokens < 1) return SWAPMOE_ERR_INVALID_ARG;
  if (c.dtype != SWAPMOE_F32 && c.dtype != SWAPMOE_BF16) return SWAPMOE_ERR_INVALID_ARG;
  if (c.n_adapters > kAdMaxCount || c.d_in % 8 || c.d_out % 8 || c.d_in > kAdMaxWidth || c.d_out > kAdMaxWidth || c.rank % 8 ||
      c.rank > kAdMaxRank || c.max_tokens >= 1 << 24)
    return SWAPMOE_ERR_UNSUPPORTED;
  const int sms = current_sm_count();
  int dev = 0, major = 0;
  if (sms == 0 || cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess) {
    cudaGetLastError();
    return SWAPMOE_ERR_CUDA;
  }
  if (major != 10) return SWAPMOE_ERR_UNSUPPORTED;       // kernels are built for sm_100a only
  swapmoe_adapters* b = new (std::nothrow) swapmoe_adapters();
  if (!b) return SWAPMOE_ERR_NO_MEMORY;
  b->cfg = c;
  b->sm_count = sms;
  const size_t tiles = (size_t)ad_max_tiles(c.max_tokens, c.n_adapters) * sizeof(AdapterTile);
  const size_t perm = sizeof(int32_t) * (size_t)c.max_tokens;
  if (cudaMalloc(&b->ws, tiles + 256 + perm) != cudaSuccess) {
    cudaGetLastError();
    delete b;
    return SWAPMOE_ERR_NO_MEMORY;
  }
  b->tiles = reinterpret_cast<AdapterTile*>(b->ws);
  b->n_tiles = reinterpret_cast<int32_t*>(b->ws + tiles);
  b->perm = reinterpret_cast<int32_t*>(b->ws + tiles + 256);
  const cudaError_t limits = c.dtype == SWAPMOE_F32 ? adapters_set_limits<float, float>() : adapters_set_limits<bf16, bf16>();
  if (limits != cudaSuccess || (c.dtype == SWAPMOE_BF16 && adapters_set_limits<__nv_fp8_e4m3, bf16>() != cudaSuccess)) {
    cudaGetLastError();
    swapmoe_adapters_destroy(b);
    return SWAPMOE_ERR_CUDA;
  }
  *out = b;
  return SWAPMOE_OK;
}

int32_t swapmoe_adapters_destroy(swapmoe_adapters_t* b) {
  if (!b) return SWAPMOE_OK;
  cudaFree(b->ws);
  delete b;
  return SWAPMOE_OK;
}

int32_t swapmoe_adapters_set_weights(swapmoe_adapters_t* b, const void* A, const void* B, const float* scale) {
  if (!b || !A || !B || misaligned(A, 16) || misaligned(B, 16) || misaligned(scale, 4)) return SWAPMOE_ERR_INVALID_ARG;
  b->A = A; b->B = B; b->scale = scale;
  return SWAPMOE_OK;
}

int32_t swapmoe_adapters_check(const swapmoe_adapters_t* b, int32_t d_in, int32_t d_out, int32_t dtype, int32_t T) {
  if (!b || T < 0 || b->cfg.d_in != d_in || b->cfg.d_out != d_out || b->cfg.dtype != dtype) return SWAPMOE_ERR_INVALID_ARG;
  if (!b->A) return SWAPMOE_ERR_NOT_READY;
  return T > b->cfg.max_tokens ? SWAPMOE_ERR_TOO_MANY_TOKENS : SWAPMOE_OK;
}

int32_t swapmoe_adapters_forward(swapmoe_adapters_t* b, const void* x, int64_t x_stride, const float* x_scales, const int32_t* ids,
                                 const void* y, int64_t y_stride, void* out, int64_t out_stride, int32_t T, void* stream) {
  return adapters_run(b, x, x_stride, x_scales, ids, y, y_stride, out, out_stride, T, stream, standalone_pdl(), nullptr);
}

}  // extern "C"
