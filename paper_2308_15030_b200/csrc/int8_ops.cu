// C ABI of the operators in 8-bit integers and of the norms around a block (see include/swapmoe.h): argument checks and launches.
#include "../../include/swapmoe.h"

#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <initializer_list>
#include <mutex>
#include <new>

#include "block_norm.cuh"
#include "block_ops.cuh"
#include "common.cuh"
#include "expert_bank.cuh"
#include "int8_gemm.cuh"
#include "int8_split.cuh"
#include "int8_stream.cuh"
#include "quantize_rows.cuh"

using namespace swapmoe;

static_assert(SWAPMOE_NORM_MAX_WIDTH == kNormMaxWidth && SWAPMOE_QUANTIZE_MAX_WIDTH == kQuantMaxWidth, "the header's limits");
static_assert((int)SWAPMOE_QUANTIZE_NONE == (int)kQuantNone && (int)SWAPMOE_QUANTIZE_RELU == (int)kQuantRelu && (int)SWAPMOE_QUANTIZE_SWIGLU == (int)kQuantSwiglu, "the header's values");
static_assert(SWAPMOE_MATMUL_MAX_K == kI8MaxK, "the header's limit");

namespace {

struct Device {
  int id, sms, pairs;                     // SMs; CTA pairs of the products that run at once (product_device)
};
constexpr int kManyDevices = 64;

// The current device.  (Threads whose first calls meet find the same values.)
int32_t current_device(Device* d) {
  static std::atomic<int> known[kManyDevices];           // SMs, 0: not asked yet
  int dev = 0, major = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev >= kManyDevices) {
    cudaGetLastError();
    return SWAPMOE_ERR_CUDA;
  }
  sms = known[dev].load(std::memory_order_relaxed);
  if (sms == 0) {
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess) {
      cudaGetLastError();
      return SWAPMOE_ERR_CUDA;
    }
    if (major != 10) return SWAPMOE_ERR_UNSUPPORTED;     // kernels are built for sm_100a only
    known[dev].store(sms, std::memory_order_relaxed);
  }
  *d = Device{dev, sms, 0};
  return SWAPMOE_OK;
}

// The same with the products' kernels ready: their limits set once, which loads them.
int32_t product_device(Device* d) {
  static std::atomic<int> known[kManyDevices];           // pairs, 0: not ready
  const int32_t rc = current_device(d);
  if (rc != SWAPMOE_OK) return rc;
  d->pairs = known[d->id].load(std::memory_order_acquire);
  if (d->pairs > 0) return SWAPMOE_OK;
  const void* const wide[] = {(const void*)bank_stream_out_kernel<bf16, 1>, (const void*)bank_stream_out_kernel<bf16, 2>,
                              (const void*)bank_stream_out_kernel<float, 1>, (const void*)bank_stream_out_kernel<float, 2>};
  bool ok = true;
  for (const void* k : wide) ok = ok && cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kBankOutRowBytes) == cudaSuccess;
  ok = ok && cudaFuncSetAttribute(int8_split_kernel<bf16>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSplitMaxSmem) == cudaSuccess &&
       cudaFuncSetAttribute(int8_split_kernel<float>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSplitMaxSmem) == cudaSuccess;
  if (ok) d->pairs = int8_gemm_init(d->sms);
  if (d->pairs < 1) {
    cudaGetLastError();
    return SWAPMOE_ERR_CUDA;
  }
  known[d->id].store(d->pairs, std::memory_order_release);
  return SWAPMOE_OK;
}

PFN_encodeTiled encoder() {
  static const PFN_encodeTiled enc = tc_get_encoder();
  return enc;
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

bool misaligned(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes != 0; }
// Whether n rows of `elem`-byte values at p, `stride` values apart, all start on multiples of `bytes`.
bool rows_aligned(const void* p, long long n, long long stride, size_t elem, size_t bytes) {
  return !misaligned(p, bytes) && (n < 2 || (size_t)stride * elem % bytes == 0);
}

}  // namespace

namespace swapmoe {

int32_t block_norm_run(const swapmoe_block_norm_t* p, void* stream, bool pdl, int64_t* launches) {
  if (!p || p->n_rows < 0 || p->d < 1) return SWAPMOE_ERR_INVALID_ARG;
  if (p->dtype != SWAPMOE_F32 && p->dtype != SWAPMOE_BF16) return SWAPMOE_ERR_INVALID_ARG;
  if (p->residual_dtype != p->dtype && p->residual_dtype != SWAPMOE_F32) return SWAPMOE_ERR_INVALID_ARG;
  if (p->type8 != SWAPMOE_E4M3 && p->type8 != SWAPMOE_INT8) return SWAPMOE_ERR_INVALID_ARG;
  if (p->group != 0 && p->group != 32 && p->group != 64 && p->group != 128 && p->group != 256) return SWAPMOE_ERR_INVALID_ARG;
  if (!(p->eps >= 0.f) || std::isinf(p->eps) || !(p->post_eps >= 0.f) || std::isinf(p->post_eps) || !std::isfinite(p->scale))
    return SWAPMOE_ERR_INVALID_ARG;
  if (p->d > kNormMaxWidth) return SWAPMOE_ERR_UNSUPPORTED;
  if (p->n_rows == 0) return SWAPMOE_OK;
  if (!p->x || (!p->out && !p->out8 && !p->residual_out) || ((p->out || p->out8) && !p->weight) || (p->out8 == nullptr) != (p->scales == nullptr))
    return SWAPMOE_ERR_INVALID_ARG;
  const size_t elem = p->dtype == SWAPMOE_BF16 ? 2 : 4, relem = p->residual_dtype == SWAPMOE_BF16 ? 2 : 4;
  const long long d = p->d, n_scales = p->group ? (d + p->group - 1) / p->group : 1;
  const int32_t n = p->n_rows;
  struct { const void* p; int32_t n; long long stride, width; size_t elem, vec; } rows[] = {
      {p->x, n, p->x_stride, d, elem, 16},
      {p->residual, n, p->residual_stride, d, relem, 16},
      {p->gate, p->gate_stride ? n : 1, p->gate_stride ? p->gate_stride : d, d, elem, 16},
      {p->residual_out, n, p->residual_out_stride, d, relem, 16},
      {p->out, n, p->out_stride, d, elem, 16},
      {p->out8, n, p->out8_stride, d, 1, 8},
      {p->scales, n, p->scales_stride, n_scales, 4, 4},
      {p->weight, 1, d, d, elem, 16},
      {p->post_weight, 1, d, d, elem, 16}};
  bool vec = d % 8 == 0;
  for (const auto& r : rows) {
    if (!r.p) continue;
    if (r.stride < r.width || misaligned(r.p, r.elem)) return SWAPMOE_ERR_INVALID_ARG;
    vec = vec && rows_aligned(r.p, r.n, r.stride, r.elem, r.vec);
  }
  BlockNormArgs a;
  a.x = p->x; a.residual = p->residual; a.post_weight = p->post_weight; a.gate = p->gate; a.weight = p->weight;
  a.residual_out = p->residual_out; a.out = p->out; a.out8 = static_cast<uint8_t*>(p->out8); a.scales = p->scales;
  a.x_stride = p->x_stride; a.residual_stride = p->residual_stride; a.gate_stride = p->gate_stride;
  a.residual_out_stride = p->residual_out_stride; a.out_stride = p->out_stride; a.out8_stride = p->out8_stride;
  a.scales_stride = p->scales_stride;
  a.T = p->n_rows; a.d = p->d; a.group = p->group; a.int8 = p->type8 == SWAPMOE_INT8;
  a.eps = p->eps; a.post_eps = p->post_eps; a.scale = p->scale;
  a.warps_per_row = a.rows_per_cta = 1;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  Device dev;
  const int32_t rc = current_device(&dev);
  if (rc != SWAPMOE_OK) return rc;
  if (p->dtype == SWAPMOE_F32) return launched(block_norm_launch_typed<float, float>(a, vec, dev.sms, st, pdl), 1, launches);
  if (p->residual_dtype == SWAPMOE_F32) return launched(block_norm_launch_typed<bf16, float>(a, vec, dev.sms, st, pdl), 1, launches);
  return launched(block_norm_launch_typed<bf16, bf16>(a, vec, dev.sms, st, pdl), 1, launches);
}

}  // namespace swapmoe

struct swapmoe_expert_bank {
  swapmoe_expert_bank_config_t cfg;
  Device dev;
  char* ws;
  long long max_rows;                      // rows of the pairs with the slots' padding
  int8_t *rows8, *h8;
  float *row_scales, *h, *h_scales, *y, *largest;
  int32_t *row_pair, *pair_row, *row_largest, *counts, *cta_base, *n_tiles;
  TileDesc* tiles;
  const int8_t *w_in, *w_out;
  const float *in_scales, *out_scales;
  bool bound;
  CUtensorMap map_in, map_out, map_x[4], map_h[4], map_h_out, map_y_out;
};

namespace {

// Token tiles per scheduling group (see decode_tile) of `rows` rows of k bytes, `height` rows a tile: those of a group stay in L2 across its weight
// tiles.  16 MB of them, six tiles at least; all in one group up to 24 MB.  us at 6 / 10 / 20 / all tiles a group: experts of 4096 x 14336, 8192 pairs,
// first product 690 / 691 / 703 / 753, second 323 / 333 / 346 / 358; 16000 pairs, first product 1305 / 1263 / 1226 / 1416.
int row_group(long long rows, long long k, int height) {
  if (rows * k <= 24ll << 20) return 1 << 30;
  return (int)std::max(6ll, (16ll << 20) / (height * k));
}

// A product of a whole matrix (matmul_scaled).
int32_t matmul_pair(const swapmoe_matmul_t& p, const Device& dev, cudaStream_t st, bool pdl) {
  const PFN_encodeTiled enc = encoder();
  if (!enc) return SWAPMOE_ERR_CUDA;
  I8GemmArgs g = {};
  g.C = p.out; g.x_scales = p.x_scales; g.w_scales = p.w_scales; g.bias = p.bias;
  g.ldc = p.out_stride; g.n_cols = p.n; g.n_col_tiles = (p.n + 255) / 256; g.k_blocks = (p.k + kI8BK - 1) / kI8BK; g.w_rows = p.n;
  g.T = p.n_tokens;
  g.height = int8_tile_height(p.n_tokens, g.n_col_tiles, dev.pairs);
  g.row_group = row_group(p.n_tokens, p.k, g.height);
  const size_t elem = p.dtype == SWAPMOE_BF16 ? 2 : 4;
  // The TMA unit stores sixteen bytes or none of them: a row that ends inside of sixteen is stored by elements, as is one that begins there.
  g.direct = !rows_aligned(p.out, 2, p.out_stride, elem, 16) || p.n * elem % 16 != 0;
  if (g.direct && elem == 2 && p.n % 2 == 0 && rows_aligned(p.out, 2, p.out_stride, elem, 4)) g.direct = 2;
  const long long xs = p.n_tokens > 1 ? p.x_stride : (p.k + 15) / 16 * 16, ws = p.n > 1 ? p.w_stride : (p.k + 15) / 16 * 16;
  CUtensorMap mw, mx[4], mc;
  if (!int8_encode_operand(enc, &mw, p.w, p.n, p.k, ws, 128)) return SWAPMOE_ERR_CUDA;
  const int half = g.height / 2;
  int have = -1;
  for (int i = 0; i < 4; ++i)
    if (half & (128 >> i)) {
      if (!int8_encode_operand(enc, &mx[i], p.x, p.n_tokens, p.k, xs, 128 >> i)) return SWAPMOE_ERR_CUDA;
      have = i;
    }
  for (int i = 0; i < 4; ++i)
    if (!(half & (128 >> i))) mx[i] = mx[have];              // not used
  if (g.direct) mc = mw;                                     // not used
  else if (!int8_encode_2d(enc, &mc, p.out, p.dtype == SWAPMOE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, elem,
                           p.n_tokens, p.n, p.out_stride, 32, kI8Chunk, int8_out_swizzle(p.dtype == SWAPMOE_BF16 ? kI8Bf16 : kI8F32)))
    return SWAPMOE_ERR_CUDA;
  const int epi = p.dtype == SWAPMOE_BF16 ? kI8Bf16 : kI8F32;
  const long long work = (long long)((p.n_tokens + g.height - 1) / g.height) * g.n_col_tiles;
  return launched(launch_kernel(int8_gemm_kernel(epi), dim3(2 * (work > dev.pairs ? dev.pairs : (int)work)), dim3(kI8Threads),
                                int8_smem_bytes(epi), st, pdl, mw, mx[0], mx[1], mx[2], mx[3], mc, g));
}

// Tokens of a cluster and its CTAs, by what a CTA has to do in ns: its bytes, (128 + cols) 128 a k-block at 87 GB/s; the sums' exchange, and
// what becomes of them, by token; clusters of eight on more than half of the SMs start late.  More CTAs than SMs only where nothing is shared.
// us with one group of tokens / as picked: 1024 x 1024 at 32, 64, 128 tokens 3.7 / 3.4, 4.3 / 3.4, 5.6 / 3.7; 2048 -> 512 4.1 / 3.8, 4.7 / 3.8, 6.4 / 3.8;
// 4096 -> 1024 at 64, 128 5.2 / 4.8, 7.0 / 5.1; CTAs of a cluster at 16 tokens, 1 / 2 / 4 / 8: 4096 x 4096 9.0 / 6.9 / 5.7 / 6.8, 4096 -> 1024 8.3 / 5.7 /
// 4.1 / 3.8, 1024 x 1024 3.6 / 3.3 / 2.9 / 3.4.
struct SplitShape { int cols, cluster; };
SplitShape split_shape(int T, int n_tiles, int k_blocks, int sms) {
  constexpr int kExchange[4] = {0, 700, 800, 650}, kToken[4] = {16, 16, 16, 36};
  SplitShape best = {0, 1};
  long long least = -1;
  for (int most = kSplitMaxTokens; most >= 16; most /= 2)
    for (int i = 0; i < 4; ++i) {
      const int cluster = 1 << i, groups = (T + most - 1) / most, step = std::max(16, 4 * cluster);
      if (i > 0 && 2 * cluster > k_blocks) continue;
      const long long ctas = (long long)n_tiles * groups * cluster;
      if ((i > 0 || most < kSplitMaxTokens) && ctas > sms) continue;
      const int cols = ((T + groups - 1) / groups + step - 1) / step * step;
      const long long cost = (k_blocks + cluster - 1) / cluster * (128ll + cols) * 3 / 2 + kToken[i] * cols + kExchange[i] + (i == 3 && 2 * ctas > sms ? 100 : 0);
      if (least < 0 || cost < least) { least = cost; best = SplitShape{cols, cluster}; }
    }
  return best;
}

// The same with a cluster for each 128 rows of weights and up to kSplitMaxTokens tokens.
int32_t matmul_split(const swapmoe_matmul_t& p, const Device& dev, cudaStream_t st, bool pdl) {
  const PFN_encodeTiled enc = encoder();
  if (!enc) return SWAPMOE_ERR_CUDA;
  I8SplitArgs g;
  g.out = p.out; g.x_scales = p.x_scales; g.w_scales = p.w_scales; g.bias = p.bias; g.ldc = p.out_stride;
  g.T = p.n_tokens; g.N = p.n; g.k_blocks = (p.k + kI8BK - 1) / kI8BK;
  const int n_tiles = (p.n + kTcBM - 1) / kTcBM;
  const SplitShape shape = split_shape(p.n_tokens, n_tiles, g.k_blocks, dev.sms);
  const int cluster = shape.cluster;
  g.cols = shape.cols;
  g.share = (g.k_blocks + cluster - 1) / cluster;
  const int stage = kSplitABytes + g.cols * kI8BK;
  g.n_stages = std::max(1, std::min(std::min(g.share, kSplitMaxStages), kSplitRoom / stage));
  const long long xs = p.n_tokens > 1 ? p.x_stride : (p.k + 15) / 16 * 16, ws = p.n > 1 ? p.w_stride : (p.k + 15) / 16 * 16;
  CUtensorMap mw, mx;
  if (!int8_encode_operand(enc, &mw, p.w, p.n, p.k, ws, 128) || !int8_encode_operand(enc, &mx, p.x, p.n_tokens, p.k, xs, g.cols)) return SWAPMOE_ERR_CUDA;
  const size_t smem = std::max(1024 + int8_split_area(g.cols, g.n_stages), kClusterMinSmem);
  const dim3 grid(n_tiles * cluster, (p.n_tokens + g.cols - 1) / g.cols), block(kSplitThreads);
  return launched(p.dtype == SWAPMOE_BF16 ? launch_cluster(int8_split_kernel<bf16>, cluster, grid, block, smem, st, pdl, mw, mx, g)
                                          : launch_cluster(int8_split_kernel<float>, cluster, grid, block, smem, st, pdl, mw, mx, g));
}

// The same for up to kStreamTokens tokens.
int32_t matmul_stream(const swapmoe_matmul_t& p, cudaStream_t st, bool pdl) {
  I8StreamArgs a;
  a.x = static_cast<const int8_t*>(p.x); a.w = static_cast<const int8_t*>(p.w);
  a.x_scales = p.x_scales; a.w_scales = p.w_scales; a.bias = p.bias; a.out = p.out;
  a.x_stride = p.x_stride; a.w_stride = p.w_stride; a.out_stride = p.out_stride;
  a.T = p.n_tokens; a.K = p.k; a.N = p.n;
  const dim3 grid((p.n + 15) / 16), block(kStreamThreads);
  return launched(p.dtype == SWAPMOE_BF16 ? launch_kernel(int8_stream_kernel<bf16>, grid, block, 0, st, pdl, a)
                                          : launch_kernel(int8_stream_kernel<float>, grid, block, 0, st, pdl, a));
}

// The status word, taken: what another stream's kernels write meanwhile is either in it or stays for the next call.
__device__ int32_t g_int8_taken[2];
__global__ void take_status_kernel() {
  g_int8_taken[0] = atomicExch(&g_int8_status[0], 0);
  g_int8_taken[1] = atomicExch(&g_int8_status[1], 0);
}
__global__ void matmul_wait_selftest_kernel(unsigned long long limit_ns) { bounded_wait_selftest(g_int8_status, 99, limit_ns); }

// Experts of few pairs.
cudaError_t bank_stream_in(const BankStreamArgs& a, bool swiglu, cudaStream_t st, bool pdl) {
  const int pairs = std::min(a.in_tokens, a.T) * a.k;
  const dim3 grid(a.F / 16, std::min(pairs, a.S), (a.T + a.in_tokens - 1) / a.in_tokens), block(kStreamThreads);
  if (swiglu) return pairs <= 8 ? launch_kernel(bank_stream_in_kernel<true, 1>, grid, block, 0, st, pdl, a) : launch_kernel(bank_stream_in_kernel<true, 2>, grid, block, 0, st, pdl, a);
  return pairs <= 8 ? launch_kernel(bank_stream_in_kernel<false, 1>, grid, block, 0, st, pdl, a) : launch_kernel(bank_stream_in_kernel<false, 2>, grid, block, 0, st, pdl, a);
}
template <typename T>
cudaError_t bank_stream_out(const BankStreamArgs& a, cudaStream_t st, bool pdl) {
  const int pairs = std::min(a.out_tokens, a.T) * a.k;
  const dim3 grid(a.d / 16, 1, (a.T + a.out_tokens - 1) / a.out_tokens), block(kBankOutThreads);
  const size_t smem = (size_t)pairs * bank_row_bytes(a.F);
  return pairs <= 8 ? launch_kernel(bank_stream_out_kernel<T, 1>, grid, block, smem, st, pdl, a) : launch_kernel(bank_stream_out_kernel<T, 2>, grid, block, smem, st, pdl, a);
}

}  // namespace

extern "C" {

int32_t swapmoe_block_norm(const swapmoe_block_norm_t* p, void* stream) { return block_norm_run(p, stream, standalone_pdl(), nullptr); }

int32_t swapmoe_quantize_rows(const swapmoe_quantize_rows_t* p, void* stream) {
  if (!p || p->n_rows < 0 || p->d < 1) return SWAPMOE_ERR_INVALID_ARG;
  if (p->dtype != SWAPMOE_F32 && p->dtype != SWAPMOE_BF16) return SWAPMOE_ERR_INVALID_ARG;
  if (p->act != kQuantNone && p->act != kQuantRelu && p->act != kQuantSwiglu) return SWAPMOE_ERR_INVALID_ARG;
  if (p->d > kQuantMaxWidth) return SWAPMOE_ERR_UNSUPPORTED;
  if (p->n_rows == 0) return SWAPMOE_OK;
  const size_t elem = p->dtype == SWAPMOE_BF16 ? 2 : 4;
  const long long width = p->act == kQuantSwiglu ? 2ll * p->d : p->d;
  if (!p->x || !p->out8 || !p->scales || p->x_stride < width || p->out8_stride < p->d || misaligned(p->x, elem) || misaligned(p->scales, 4))
    return SWAPMOE_ERR_INVALID_ARG;
  QuantizeArgs a = {};
  a.x = p->x; a.out8 = static_cast<uint8_t*>(p->out8); a.scales = p->scales; a.x_stride = p->x_stride; a.out8_stride = p->out8_stride;
  a.T = p->n_rows; a.d = p->d; a.act = p->act;
  const bool vec = p->d % 8 == 0 && rows_aligned(p->x, p->n_rows, p->x_stride, elem, 16) && rows_aligned(p->out8, p->n_rows, p->out8_stride, 1, 8);
  Device dev;
  const int32_t rc = current_device(&dev);
  if (rc != SWAPMOE_OK) return rc;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  return launched(p->dtype == SWAPMOE_F32 ? quantize_rows_launch<float>(a, vec, dev.sms, st, standalone_pdl())
                                          : quantize_rows_launch<bf16>(a, vec, dev.sms, st, standalone_pdl()));
}

int32_t swapmoe_matmul_scaled(const swapmoe_matmul_t* p, void* stream) {
  if (!p || p->n_tokens < 0 || p->k < 1 || p->n < 1) return SWAPMOE_ERR_INVALID_ARG;
  if (p->dtype != SWAPMOE_F32 && p->dtype != SWAPMOE_BF16) return SWAPMOE_ERR_INVALID_ARG;
  if (p->k > kI8MaxK || p->n > INT32_MAX - 256 || p->n_tokens > INT32_MAX - 256) return SWAPMOE_ERR_UNSUPPORTED;      // (tiles behind the end keep to int32)
  if (p->n_tokens == 0) return SWAPMOE_OK;
  const size_t elem = p->dtype == SWAPMOE_BF16 ? 2 : 4;
  if (!p->x || !p->x_scales || !p->w || !p->w_scales || !p->out || p->x_stride < p->k || p->w_stride < p->k || p->out_stride < p->n)
    return SWAPMOE_ERR_INVALID_ARG;
  if (!rows_aligned(p->x, p->n_tokens, p->x_stride, 1, 16) || !rows_aligned(p->w, p->n, p->w_stride, 1, 16) || misaligned(p->out, elem) ||
      misaligned(p->x_scales, 4) || misaligned(p->w_scales, 4) || misaligned(p->bias, 4))
    return SWAPMOE_ERR_INVALID_ARG;
  Device dev;
  const int32_t rc = product_device(&dev);
  if (rc != SWAPMOE_OK) return rc;
  // Few tokens and a small matrix: the weights straight to registers.  Few tokens, or few tiles: the contraction shared.  us for 8 tokens,
  // registers / shared: 1024 x 1024 2.4 / 3.4, 2048 x 2048 3.3 / 4.2, 4096 -> 1024 4.7 / 4.5, 4096 x 4096 6.3 / 5.9, 4096 -> 14336 15.8 / 12.6.
  // Shared / CTA pairs: 4096 -> 14336 at 32, 64 tokens 12.5 / 12.5, 14.4 / 12.8; 1024 -> 4096 at 128, 256, 320 4.5 / 6.0, 5.3 / 6.2, 6.4 / 6.6; 1024 x
  // 1024 at 256, 1024, 1536 4.0 / 5.6, 5.0 / 6.1, 6.4 / 6.5; 2048 x 2048 at 256, 512, 1024 6.2 / 7.6, 7.1 / 7.8, 9.3 / 8.4; 4096 x 4096 at 128, 256, 320
  // 9.8 / 10.6, 11.6 / 11.4, 13.8 / 12.3; 4096 -> 1024 at 256, 1024 6.1 / 10.5, 10.6 / 11.1; 14336 -> 4096 at 200 25.3 / 28.3; 512 x 512 at 1024 3.4 / 4.8.
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (p->n_tokens <= kStreamTokens && p->k <= 2048 && (long long)p->k * p->n <= 6ll << 20) return matmul_stream(*p, st, standalone_pdl());
  const int tiles = (p->n + kTcBM - 1) / kTcBM;
  const long long groups = p->k >= 4096 ? 2 * ((p->n_tokens + 127) / 128) : (p->n_tokens + 63) / 64;        // (14336 -> 2048 at 576 31.4 / 28.4)
  if (p->n_tokens <= 32 || (2 * tiles <= dev.sms && tiles * groups <= dev.sms)) return matmul_split(*p, dev, st, standalone_pdl());
  return matmul_pair(*p, dev, st, standalone_pdl());
}

int32_t swapmoe_matmul_status(int32_t* detail, void* stream) {
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  int32_t s[2] = {0, 0};
  cudaError_t e = cudaStreamSynchronize(st);
  if (e == cudaSuccess) {
    // one call at a time: they share the place that what was taken passes through
    static std::mutex lock;
    std::lock_guard<std::mutex> hold(lock);
    e = launch_kernel(take_status_kernel, dim3(1), dim3(1), 0, st, false);
    if (e == cudaSuccess) e = cudaMemcpyFromSymbolAsync(s, g_int8_taken, sizeof(s), 0, cudaMemcpyDeviceToHost, st);
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  }
  if (e != cudaSuccess) return launched(e);
  if (detail) *detail = s[0] ? s[1] : 0;
  return s[0] ? SWAPMOE_ERR_DEVICE_TIMEOUT : SWAPMOE_OK;
}

int32_t swapmoe_selftest_matmul_wait(int32_t limit_ms, void* stream) {
  if (limit_ms < 1 || limit_ms > 1000) return SWAPMOE_ERR_INVALID_ARG;
  return launched(launch_kernel(matmul_wait_selftest_kernel, dim3(1), dim3(32), 0, static_cast<cudaStream_t>(stream), false,
                                (unsigned long long)limit_ms * 1000000ull));
}

int32_t swapmoe_expert_bank_create(swapmoe_expert_bank_t** out, const swapmoe_expert_bank_config_t* cfg) {
  if (!out || !cfg) return SWAPMOE_ERR_INVALID_ARG;
  const swapmoe_expert_bank_config_t c = *cfg;
  if (c.n_slots < 1 || c.d_model < 1 || c.d_ff < 1 || c.top_k < 1 || c.max_tokens < 1) return SWAPMOE_ERR_INVALID_ARG;
  if (c.dtype != SWAPMOE_F32 && c.dtype != SWAPMOE_BF16) return SWAPMOE_ERR_INVALID_ARG;
  if (c.act != SWAPMOE_ACT_RELU && c.act != SWAPMOE_ACT_SWIGLU) return SWAPMOE_ERR_INVALID_ARG;
  const int nin = c.act == SWAPMOE_ACT_SWIGLU ? 2 : 1;
  if (c.n_slots > kBankMaxSlots || c.top_k > 16 || c.d_model % 64 || c.d_ff % 64 || c.d_model > kQuantMaxWidth || c.d_ff > kQuantMaxWidth ||
      (long long)c.max_tokens * c.top_k >= 1 << 24 || (long long)c.n_slots * nin * c.d_ff >= 1ll << 31 || (long long)c.n_slots * c.d_model >= 1ll << 31)
    return SWAPMOE_ERR_UNSUPPORTED;
  Device dev;
  const int32_t rc = product_device(&dev);
  if (rc != SWAPMOE_OK) return rc;
  const PFN_encodeTiled enc = encoder();
  if (!enc) return SWAPMOE_ERR_CUDA;
  swapmoe_expert_bank* b = new (std::nothrow) swapmoe_expert_bank();
  if (!b) return SWAPMOE_ERR_NO_MEMORY;
  b->cfg = c;
  b->dev = dev;
  const long long P = (long long)c.max_tokens * c.top_k, d = c.d_model, f = c.d_ff;
  b->max_rows = (P + 31ll * (c.n_slots < P ? c.n_slots : P) + 31) / 32 * 32;
  const size_t R = (size_t)b->max_rows;
  // a slot's tiles: at most one for every 32 rows, 64 rows or more in each but the last
  const size_t n_tiles = R / 32 + 32;
  struct { void** p; size_t bytes; } parts[] = {
      {reinterpret_cast<void**>(&b->rows8), R * d}, {reinterpret_cast<void**>(&b->h8), R * f},
      {reinterpret_cast<void**>(&b->h), R * f * 4}, {reinterpret_cast<void**>(&b->y), R * d * 4},
      {reinterpret_cast<void**>(&b->row_scales), R * 4}, {reinterpret_cast<void**>(&b->h_scales), R * 4},
      {reinterpret_cast<void**>(&b->row_pair), R * 4}, {reinterpret_cast<void**>(&b->row_largest), R * 4}, {reinterpret_cast<void**>(&b->pair_row), (size_t)P * 4},
      {reinterpret_cast<void**>(&b->largest), (size_t)std::min<long long>(P, kStreamPairs) * (f / 16) * 4},
      {reinterpret_cast<void**>(&b->counts), kBankMaxSlots * 4}, {reinterpret_cast<void**>(&b->cta_base), (size_t)kBankMaxCtas * c.n_slots * 4},
      {reinterpret_cast<void**>(&b->n_tiles), 16}, {reinterpret_cast<void**>(&b->tiles), n_tiles * sizeof(TileDesc)}};
  size_t bytes = 0;
  for (auto& q : parts) bytes += (q.bytes + 255) / 256 * 256;
  if (cudaMalloc(&b->ws, bytes) != cudaSuccess) {
    cudaGetLastError();
    delete b;
    return SWAPMOE_ERR_NO_MEMORY;
  }
  char* at = b->ws;
  for (auto& q : parts) {
    *q.p = at;
    at += (q.bytes + 255) / 256 * 256;
  }
  // (the default stream's work is not ordered before that of other streams)
  bool ok = cudaMemset(b->counts, 0, kBankMaxSlots * 4) == cudaSuccess && cudaStreamSynchronize(nullptr) == cudaSuccess;
  for (int i = 0; i < 4; ++i)
    ok = ok && int8_encode_operand(enc, &b->map_x[i], b->rows8, R, d, d, 128 >> i) && int8_encode_operand(enc, &b->map_h[i], b->h8, R, f, f, 128 >> i);
  ok = ok && int8_encode_2d(enc, &b->map_h_out, b->h, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, R, f, f, nin == 2 ? 16 : 32, kI8Chunk, int8_out_swizzle(nin == 2 ? kI8Swiglu : kI8Relu)) &&
       int8_encode_2d(enc, &b->map_y_out, b->y, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, R, d, d, 32, kI8Chunk, int8_out_swizzle(kI8F32));
  if (!ok) {
    cudaGetLastError();
    swapmoe_expert_bank_destroy(b);
    return SWAPMOE_ERR_CUDA;
  }
  *out = b;
  return SWAPMOE_OK;
}

int32_t swapmoe_expert_bank_destroy(swapmoe_expert_bank_t* b) {
  if (!b) return SWAPMOE_OK;
  cudaFree(b->ws);
  delete b;
  return SWAPMOE_OK;
}

int32_t swapmoe_expert_bank_set_weights(swapmoe_expert_bank_t* b, const void* w_in, const float* in_scales, const void* w_out,
                                        const float* out_scales) {
  if (!b || !w_in || !in_scales || !w_out || !out_scales || misaligned(w_in, 16) || misaligned(w_out, 16) || misaligned(in_scales, 4) ||
      misaligned(out_scales, 4))
    return SWAPMOE_ERR_INVALID_ARG;
  const swapmoe_expert_bank_config_t& c = b->cfg;
  const PFN_encodeTiled enc = encoder();
  const cuuint64_t d = (cuuint64_t)c.d_model, f = (cuuint64_t)c.d_ff, S = (cuuint64_t)c.n_slots;
  CUtensorMap in, outm;
  if (c.act == SWAPMOE_ACT_SWIGLU) {
    // sixteen rows of the first matrix, the same sixteen of the second, the next sixteen of the first ...
    const cuuint64_t dims[5] = {d, 16, 2, f / 16, S};
    const cuuint64_t strides[4] = {d, f * d, 16 * d, 2 * f * d};
    const cuuint32_t box[5] = {(cuuint32_t)kI8BK, 16, 2, 4, 1};
    const cuuint32_t estr[5] = {1, 1, 1, 1, 1};
    if (enc(&in, CU_TENSOR_MAP_DATA_TYPE_UINT8, 5, const_cast<void*>(w_in), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      return SWAPMOE_ERR_CUDA;
  } else if (!int8_encode_operand(enc, &in, w_in, S * f, d, d, 128)) {
    return SWAPMOE_ERR_CUDA;
  }
  if (!int8_encode_operand(enc, &outm, w_out, S * d, f, f, 128)) return SWAPMOE_ERR_CUDA;
  b->w_in = static_cast<const int8_t*>(w_in); b->w_out = static_cast<const int8_t*>(w_out);
  b->map_in = in; b->map_out = outm; b->in_scales = in_scales; b->out_scales = out_scales;
  b->bound = true;
  return SWAPMOE_OK;
}

int32_t swapmoe_expert_bank_forward(swapmoe_expert_bank_t* b, const void* x, int64_t x_stride, const float* x_scales, const int32_t* slots,
                                    const float* weights, void* out, int64_t out_stride, int32_t T, void* stream) {
  if (!b || T < 0) return SWAPMOE_ERR_INVALID_ARG;
  if (T == 0) return SWAPMOE_OK;
  const swapmoe_expert_bank_config_t& c = b->cfg;
  if (!x || !x_scales || !slots || !weights || !out || x_stride < c.d_model || out_stride < c.d_model) return SWAPMOE_ERR_INVALID_ARG;
  const size_t elem = c.dtype == SWAPMOE_BF16 ? 2 : 4;
  if (!rows_aligned(x, T, x_stride, 1, 16) || misaligned(out, elem) || misaligned(x_scales, 4) || misaligned(slots, 4) || misaligned(weights, 4))
    return SWAPMOE_ERR_INVALID_ARG;
  if (!b->bound) return SWAPMOE_ERR_NOT_READY;
  if (T > c.max_tokens) return SWAPMOE_ERR_TOO_MANY_TOKENS;
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev != b->dev.id) {
    cudaGetLastError();
    return SWAPMOE_ERR_INVALID_ARG;
  }
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool pdl = standalone_pdl(), swiglu = c.act == SWAPMOE_ACT_SWIGLU;
  const int P = T * c.top_k, pairs = b->dev.pairs;
  cudaError_t e = cudaSuccess;
  // Few pairs on small experts: two launches that take the weights straight to registers.  us, that form / the general one: 512 x 704 top-2 20
  // pairs 11.9 / 17.9, 32 pairs 13.1 / 18.6, 48 pairs 16.9 / 18.3; 1024 x 512 top-4 24 pairs 14.4 / 20.8, 40 pairs 21.8 / 24.9, 64 pairs 27.0 / 25.2; 512 x
  // 256 top-8 64 pairs 13.4 / 22.9, 128 pairs 24.7 / 23.9; 768 x 2112 top-2 12 pairs 18.1 / 29.2, 22 pairs 32 / 28; 2048 x 1024 top-4 16 pairs 25.2 / 29.7;
  // 1024 x 4096 top-2 8 pairs 23.0 / 29.5.
  const int share = kStreamMaxPairs / c.top_k, fit = kBankOutRowBytes / (c.top_k * bank_row_bytes(c.d_ff));       // tokens that a CTA may take
  if (P <= kStreamPairs && fit > 0 && 3ll * P * c.d_model * c.d_ff <= (P <= 16 ? 100ll : 68ll) << 20) {
    BankStreamArgs q;
    q.x8 = static_cast<const int8_t*>(x); q.w_in = b->w_in; q.w_out = b->w_out; q.x_scales = x_scales; q.in_scales = b->in_scales;
    q.out_scales = b->out_scales; q.weights = weights; q.slots = slots; q.h = b->h; q.largest = b->largest; q.out = out;
    q.x_stride = x_stride; q.out_stride = out_stride; q.P = P; q.S = c.n_slots; q.k = c.top_k; q.d = c.d_model; q.F = c.d_ff; q.T = T;
    q.in_tokens = share;
    // the second kernel's CTAs take fewer tokens where that keeps more SMs at work, one CTA on each and with 64 KB of weights at least
    const long long groups = std::max(1ll, std::min<long long>(b->dev.sms / (c.d_model / 16), (long long)P * 16 * c.d_ff >> 16));
    q.out_tokens = std::min(std::min(share, fit), (int)((T + groups - 1) / groups));
    e = bank_stream_in(q, swiglu, st, pdl);
    if (e == cudaSuccess) e = c.dtype == SWAPMOE_BF16 ? bank_stream_out<bf16>(q, st, pdl) : bank_stream_out<float>(q, st, pdl);
    return launched(e);
  }
  BankArgs a;
  a.x8 = static_cast<const int8_t*>(x); a.x_scales = x_scales; a.slots = slots; a.rows8 = b->rows8; a.row_scales = b->row_scales;
  a.row_pair = b->row_pair; a.pair_row = b->pair_row; a.largest = b->row_largest; a.counts = b->counts; a.cta_base = b->cta_base; a.tiles = b->tiles;
  a.n_tiles = b->n_tiles;
  a.x_stride = x_stride; a.P = P; a.S = c.n_slots; a.k = c.top_k; a.d = c.d_model;
  a.cols[0] = (c.d_ff + (swiglu ? 127 : 255)) / (swiglu ? 128 : 256); a.k_blocks[0] = (c.d_model + kI8BK - 1) / kI8BK;
  a.cols[1] = (c.d_model + 255) / 256; a.k_blocks[1] = (c.d_ff + kI8BK - 1) / kI8BK; a.pairs = pairs;
  if (P <= kBankDirectPairs) {
    a.per_cta = kBankDirectWarps;
    e = launch_kernel(bank_gather_direct_kernel, dim3((P + a.per_cta - 1) / a.per_cta + 1), dim3(kBankThreads), 0, st, pdl, a);
  } else {
    a.per_cta = std::max(8, (P + 2 * b->dev.sms - 1) / (2 * b->dev.sms));
    const int ctas = (P + a.per_cta - 1) / a.per_cta;
    if (ctas > kBankMaxCtas) return SWAPMOE_ERR_UNSUPPORTED;
    e = launch_kernel(bank_count_kernel, dim3(ctas), dim3(kBankThreads), 0, st, pdl, a);
    if (e == cudaSuccess) e = launch_kernel(bank_gather_kernel, dim3(ctas), dim3(kBankThreads), 0, st, pdl, a);
  }

  const long long rows = std::min<long long>(b->max_rows, (P + 31ll * std::min(P, c.n_slots) + 31) / 32 * 32);
  const long long max_tiles = (P + 63) / 64 + std::min(P, c.n_slots);
  I8GemmArgs g = {};
  g.tiles = b->tiles; g.n_tiles = b->n_tiles; g.height = 256; g.early = 1; g.row_group = row_group(P, c.d_model, 256);
  g.C = b->h; g.x_scales = b->row_scales; g.w_scales = b->in_scales; g.ldc = c.d_ff; g.n_cols = c.d_ff; g.largest = b->row_largest;
  g.n_col_tiles = a.cols[0]; g.k_blocks = a.k_blocks[0]; g.w_rows = c.d_ff;
  const int epi = swiglu ? kI8Swiglu : kI8Relu;
  long long work = max_tiles * g.n_col_tiles;
  if (e == cudaSuccess)
    e = launch_kernel(int8_gemm_kernel(epi), dim3(2 * (unsigned)std::min<long long>(work, pairs)), dim3(kI8Threads), int8_smem_bytes(epi), st, pdl,
                      b->map_in, b->map_x[0], b->map_x[1], b->map_x[2], b->map_x[3], b->map_h_out, g);
  BankQuantizeArgs q;
  q.h = b->h; q.largest = b->row_largest; q.row_pair = b->row_pair; q.pair_row = b->pair_row; q.n_tiles = b->n_tiles;
  q.h8 = reinterpret_cast<uint8_t*>(b->h8); q.h_scales = b->h_scales;
  const int turns = c.d_ff < 1024 ? 4 : 8;
  q.F = c.d_ff; q.by_pair = P < rows / 2; q.n = q.by_pair ? P : (int)rows; q.parts = (c.d_ff + 128 * turns - 1) / (128 * turns);
  const dim3 units((unsigned)(((long long)q.n * q.parts + kBankThreads / 32 - 1) / (kBankThreads / 32)));
  if (e == cudaSuccess)
    e = turns == 4 ? launch_kernel(bank_quantize_kernel<4>, units, dim3(kBankThreads), 0, st, pdl, q)
                   : launch_kernel(bank_quantize_kernel<8>, units, dim3(kBankThreads), 0, st, pdl, q);
  g.C = b->y; g.x_scales = b->h_scales; g.w_scales = b->out_scales; g.ldc = c.d_model; g.n_cols = c.d_model; g.largest = nullptr; g.early = 2; g.row_group = row_group(P, c.d_ff, 256);
  g.n_col_tiles = a.cols[1]; g.k_blocks = a.k_blocks[1]; g.w_rows = c.d_model;
  work = max_tiles * g.n_col_tiles;
  if (e == cudaSuccess)
    e = launch_kernel(int8_gemm_kernel(kI8F32), dim3(2 * (unsigned)std::min<long long>(work, pairs)), dim3(kI8Threads), int8_smem_bytes(kI8F32), st,
                      pdl, b->map_out, b->map_h[0], b->map_h[1], b->map_h[2], b->map_h[3], b->map_y_out, g);
  BankCombineArgs m;
  m.y = b->y; m.pair_row = b->pair_row; m.weights = weights; m.counts = b->counts; m.out = out; m.out_stride = out_stride;
  m.T = T; m.k = c.top_k; m.d = c.d_model; m.S = c.n_slots; m.vec = rows_aligned(out, T, out_stride, elem, 4 * elem);
  if (e == cudaSuccess) e = c.dtype == SWAPMOE_BF16 ? bank_combine_launch<bf16>(m, st, pdl) : bank_combine_launch<float>(m, st, pdl);
  if (e != cudaSuccess) cudaMemsetAsync(b->counts, 0, kBankMaxSlots * 4, st);          // what the last kernel would have left
  return launched(e);
}

}  // extern "C"
