// Rows to 8-bit integers with a scale each:
//   y = x,  relu(x),  or silu(x[0 .. d)) * x[d .. 2 d);  scale = max |y| / 127,  q = y / scale, rounded to nearest, ties to even.
// The scale is the quotient rounded to fp32, and q the quotient by that scale rounded to an integer, as IEEE division gives both.
//
// Bound by HBM: a team of warps holds a row in registers between its maximum and its rounding.
#pragma once
#include "block_norm.cuh"

namespace swapmoe {

enum { kQuantNone = 0, kQuantRelu = 1, kQuantSwiglu = 2 };
constexpr int kQuantMaxWidth = kNormChunk * kNormMaxWarps * 4;

struct QuantizeArgs {
  const void* x;
  uint8_t* out8;
  float* scales;
  const int32_t *row_pair, *n_rows;      // a row whose entry is negative, or behind n_rows[0], is left out (nullptr: none is)
  long long x_stride, out8_stride;       // elements
  int T, d, act;
  int warps_per_row, rows_per_cta;
};

// v / scale rounded to an integer as the division would be.  v * (1 / scale) is off by less than 2^-22 of itself, 4e-5 of a step at
// 127: only a product that lies nearer to the middle of two integers can be rounded to the wrong one, and is divided.
__device__ __forceinline__ float quotient8(float v, float scale, float inverse) {
  const float t = v * inverse, r = rintf(t);
  return fabsf(fabsf(t - r) - 0.5f) < 1e-4f ? rintf(__fdiv_rn(v, scale)) : t;
}

template <typename T, int kChunks, bool kVec>
__global__ void __launch_bounds__(kNormMaxWarps * 32) quantize_rows_kernel(const __grid_constant__ QuantizeArgs a) {
  __shared__ float s_max[kNormMaxWarps];
  const int lane = threadIdx.x & 31, wr = threadIdx.x >> 5, team = threadIdx.y;       // a team per row: blockDim.x threads
  const long long row = (long long)blockIdx.x * a.rows_per_cta + team;
  pdl_wait();
  pdl_trigger();
  const bool active = row < a.T && (a.row_pair == nullptr || (row < __ldcg(a.n_rows) && a.row_pair[row] >= 0));
  const int d = active ? a.d : 0;        // a team without a row computes on zeros and stores nothing
  auto first = [&](int j) { return (wr + j * a.warps_per_row) * kNormChunk; };
  const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
  float y[kChunks][8], most = 0.f;
#pragma unroll
  for (int j = 0; j < kChunks; ++j) norm_load8<kVec>(x, first(j), lane, d, y[j]);
  if (a.act == kQuantRelu) {
#pragma unroll
    for (int j = 0; j < kChunks; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) y[j][i] = y[j][i] < 0.f ? 0.f : y[j][i];                   // NaN stays NaN
  } else if (a.act == kQuantSwiglu) {
#pragma unroll
    for (int j = 0; j < kChunks; ++j) {
      float u[8];
      norm_load8<kVec>(x + a.d, first(j), lane, d, u);
#pragma unroll
      for (int i = 0; i < 8; ++i) y[j][i] = silu_from_exp(y[j][i], __expf(-y[j][i])) * u[i];
    }
  }
#pragma unroll
  for (int j = 0; j < kChunks; ++j) most = max_magnitude(most, largest8(y[j]), 0.f);
  most = warp_largest(most);
  if (a.warps_per_row > 1) {
    if (lane == 0) s_max[team * a.warps_per_row + wr] = most;
    __syncthreads();
    for (int w = 0; w < a.warps_per_row; ++w) most = max_magnitude(most, s_max[team * a.warps_per_row + w], 0.f);
  }
  // a row of zeros has scale 0 and zeros; other scales are at least 2^-120, so that the reciprocal is finite
  const float quotient = __fdiv_rn(most, kInt8Max), scale = quotient < kNormMinScale ? kNormMinScale : quotient;
  const float inverse = __frcp_rn(scale);
  if (active && wr == 0 && lane == 0) a.scales[row] = most == 0.f ? 0.f : scale;
  uint8_t* q = a.out8 + row * a.out8_stride;
#pragma unroll
  for (int j = 0; j < kChunks; ++j) {
#pragma unroll
    for (int i = 0; i < 8; ++i) y[j][i] = quotient8(y[j][i], scale, inverse);
    store8_int8<kVec>(q, first(j), lane, d, y[j]);
  }
}

template <typename T>
inline cudaError_t quantize_rows_launch(QuantizeArgs a, bool vec, int sm_count, cudaStream_t st, bool pdl) {
  const int chunks = (a.d + kNormChunk - 1) / kNormChunk;
  // as in the norms; rows of more than 64 chunks: four per warp
  const bool few = (long long)a.T * chunks <= 8ll * sm_count && chunks <= kNormMaxWarps;
  const int per_warp = few ? 1 : chunks <= 2 * kNormMaxWarps ? 2 : 4;
  a.warps_per_row = (chunks + per_warp - 1) / per_warp;
  a.rows_per_cta = few || a.warps_per_row >= 8 ? 1 : 8 / a.warps_per_row;
  const dim3 grid((unsigned)(((long long)a.T + a.rows_per_cta - 1) / a.rows_per_cta)), block(32 * a.warps_per_row, a.rows_per_cta);
  auto go = [&](auto kernel) { return launch_kernel(kernel, grid, block, 0, st, pdl, a); };
  if (vec) return per_warp == 1 ? go(quantize_rows_kernel<T, 1, true>) : per_warp == 2 ? go(quantize_rows_kernel<T, 2, true>) : go(quantize_rows_kernel<T, 4, true>);
  return per_warp == 1 ? go(quantize_rows_kernel<T, 1, false>) : per_warp == 2 ? go(quantize_rows_kernel<T, 2, false>) : go(quantize_rows_kernel<T, 4, false>);
}

}  // namespace swapmoe
