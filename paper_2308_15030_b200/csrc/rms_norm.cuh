// The residual's addition and the root-mean-square norm in front of a layer:
//   h = x + residual,  residual_out = round(h),  y = h * w / sqrt(mean(h^2) + eps),
// y as rows of the layer's dtype, as e4m3 rows with scales (q = y / s, s = max |y| / 448 over a row or a group of columns), or both.
// The norm is taken of the sum before it is rounded, in fp32; every output is rounded once.
//
// Bound by HBM: each row is read once, kept in registers between the sum of squares and the scaling, and written once.  A team
// of warps holds a row, eight columns per lane and chunk of 256.  y is computed as (h w) s: multiplying by the row's positive
// factor keeps the order of magnitudes, so the largest |y| of a row is the largest |h w| times s to the last bit and is found in
// the same exchange between the warps as the sum of squares.
#pragma once
#include <cuda_fp8.h>
#include <math_constants.h>

#include "common.cuh"
#include "launch.cuh"

namespace swapmoe {

constexpr int kNormChunk = 256;          // columns of a warp's chunk: eight per lane
constexpr int kNormMaxWarps = 32;
constexpr int kNormMaxWidth = kNormChunk * kNormMaxWarps * 2;
constexpr float kE4m3Max = 448.f;
// A scale other than 0 is at least this: its reciprocal stays finite.  (A row whose largest value is below 448 x 2^-120 then uses
// fewer of the 8-bit type's values.)
constexpr float kNormMinScale = 0x1p-120f;

struct RmsNormArgs {
  const void *x, *residual, *weight;
  void *residual_out, *out;
  uint8_t* out8;
  float* scales;
  long long x_stride, residual_stride, residual_out_stride, out_stride, out8_stride, scales_stride;   // elements
  int T, d, group;                       // group: columns per scale (0: one scale per row)
  float eps;
  int warps_per_row, rows_per_cta;
};

__device__ __forceinline__ float norm_load(const float* p) { return *p; }
__device__ __forceinline__ float norm_load(const bf16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void norm_store(float* p, float v) { *p = v; }
__device__ __forceinline__ void norm_store(bf16* p, float v) { *p = __float2bfloat16_rn(v); }

// Eight of a row's columns.  kVec: 16-byte pieces, lane l holds columns 8 l ... 8 l + 7 of the chunk; else columns l, l + 32, ...
// (a row that starts anywhere, of any width), so that a warp's loads still cover consecutive columns.
template <bool kVec, typename T>
__device__ __forceinline__ void norm_load8(const T* row, int c0, int lane, int d, float (&v)[8]) {
  if constexpr (kVec) {
    if (c0 + lane * 8 < d) {
      load4(row + c0 + lane * 8, v);
      load4(row + c0 + lane * 8 + 4, v + 4);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = 0.f;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c0 + i * 32 + lane < d ? norm_load(row + c0 + i * 32 + lane) : 0.f;
  }
}
template <bool kVec, typename T>
__device__ __forceinline__ void norm_store8(T* row, int c0, int lane, int d, const float (&v)[8]) {
  if constexpr (kVec) {
    if (c0 + lane * 8 < d) store8(row + c0 + lane * 8, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c0 + i * 32 + lane < d) norm_store(row + c0 + i * 32 + lane, v[i]);
  }
}
// Two values to e4m3, values beyond the type's range to its ends (NaN stays NaN).
__device__ __forceinline__ uint32_t pack_e4m3x2(float lo, float hi) {
  return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
}
template <bool kVec>
__device__ __forceinline__ void norm_store8_e4m3(uint8_t* row, int c0, int lane, int d, const float (&v)[8]) {
  if constexpr (kVec) {
    if (c0 + lane * 8 < d)
      *reinterpret_cast<uint2*>(row + c0 + lane * 8) = make_uint2(pack_e4m3x2(v[0], v[1]) | pack_e4m3x2(v[2], v[3]) << 16,
                                                                  pack_e4m3x2(v[4], v[5]) | pack_e4m3x2(v[6], v[7]) << 16);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c0 + i * 32 + lane < d) row[c0 + i * 32 + lane] = (uint8_t)pack_e4m3x2(v[i], 0.f);
  }
}
// Magnitudes as integers: their order is that of the values, with NaN above infinity.
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// Scale of the largest magnitude, and its reciprocal (0 for a row or group of zeros, whose 8-bit values are zeros).
__device__ __forceinline__ float norm_scale(float largest, float* inverse) {
  const float s = largest > 0.f ? fmaxf(largest / kE4m3Max, kNormMinScale) : largest;     // NaN stays NaN
  *inverse = s > 0.f ? 1.f / s : s;
  return s;
}

// T: rows and weight; R: the residual's rows; kChunks: chunks per warp.
template <typename T, typename R, int kChunks, bool kVec>
__global__ void __launch_bounds__(kNormMaxWarps * 32) rms_norm_kernel(const RmsNormArgs a) {
  __shared__ float s_sum[kNormMaxWarps];
  __shared__ uint32_t s_max[kNormMaxWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int team = warp / a.warps_per_row, wr = warp - team * a.warps_per_row;
  const long long row = (long long)blockIdx.x * a.rows_per_cta + team;
  const bool active = row < a.T;
  const int d = active ? a.d : 0;        // a team without a row computes on zeros and stores nothing
  float h[kChunks][8], p[kChunks][8];
  pdl_wait();
  pdl_trigger();
  const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
#pragma unroll
  for (int j = 0; j < kChunks; ++j) norm_load8<kVec>(x, (wr + j * a.warps_per_row) * kNormChunk, lane, d, h[j]);
  if (a.residual != nullptr) {
    const R* r = static_cast<const R*>(a.residual) + row * a.residual_stride;
#pragma unroll
    for (int j = 0; j < kChunks; ++j) norm_load8<kVec>(r, (wr + j * a.warps_per_row) * kNormChunk, lane, d, p[j]);
#pragma unroll
    for (int j = 0; j < kChunks; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) h[j][i] += p[j][i];
    if (a.residual_out != nullptr) {
      R* ro = static_cast<R*>(a.residual_out) + row * a.residual_out_stride;
#pragma unroll
      for (int j = 0; j < kChunks; ++j) norm_store8<kVec>(ro, (wr + j * a.warps_per_row) * kNormChunk, lane, d, h[j]);
    }
  }
  if (a.out == nullptr && a.out8 == nullptr) return;                  // the same for the whole grid
  float sum = 0.f;
  uint32_t most = 0u;
#pragma unroll
  for (int j = 0; j < kChunks; ++j) {
    norm_load8<kVec>(static_cast<const T*>(a.weight), (wr + j * a.warps_per_row) * kNormChunk, lane, d, p[j]);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      sum = fmaf(h[j][i], h[j][i], sum);
      p[j][i] *= h[j][i];
      most = max(most, magnitude(p[j][i]));
    }
  }
  sum = warp_sum(sum);
  most = __reduce_max_sync(0xffffffffu, most);
  if (lane == 0) { s_sum[warp] = sum; s_max[warp] = most; }
  // squares that leave the range of fp32 (rows of 1e18 and more, or below 1e-15 with next to no eps), infinities, NaN
  const bool rare = !(sum < 1e36f) || most >= 0x7f800000u || (sum < 1e-28f && a.eps < 1e-25f);
  const bool slow = __syncthreads_or(rare) != 0;
  float total = 0.f;
  uint32_t largest = 0u;
  for (int w = 0; w < a.warps_per_row; ++w) {
    total += s_sum[team * a.warps_per_row + w];
    largest = max(largest, s_max[team * a.warps_per_row + w]);
  }
  float s = rsqrtf(total / (float)a.d + a.eps);
  if (slow) {
    // the same with the row divided by its largest magnitude m: h / sqrt(mean(h^2) + eps) = (h / m) / sqrt(mean((h / m)^2) + eps / m^2)
    most = 0u;
#pragma unroll
    for (int j = 0; j < kChunks; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) most = max(most, magnitude(h[j][i]));
    most = __reduce_max_sync(0xffffffffu, most);
    __syncthreads();
    if (lane == 0) s_max[warp] = most;
    __syncthreads();
    for (int w = 0; w < a.warps_per_row; ++w) most = max(most, s_max[team * a.warps_per_row + w]);
    const float m = __uint_as_float(most);
    const bool scaled = most > 0u && most < 0x7f800000u;
    sum = 0.f;
    most = 0u;
#pragma unroll
    for (int j = 0; j < kChunks; ++j) {
      norm_load8<kVec>(static_cast<const T*>(a.weight), (wr + j * a.warps_per_row) * kNormChunk, lane, d, p[j]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (scaled) h[j][i] /= m;
        sum = fmaf(h[j][i], h[j][i], sum);
      }
    }
    sum = warp_sum(sum);
    __syncthreads();
    if (lane == 0) s_sum[warp] = sum;
    __syncthreads();
    total = 0.f;
    for (int w = 0; w < a.warps_per_row; ++w) total += s_sum[team * a.warps_per_row + w];
    s = rsqrtf(total / (float)a.d + (scaled ? a.eps / m / m : a.eps));
    // the row's factor goes into the products at once: an infinity among them would be none behind it
#pragma unroll
    for (int j = 0; j < kChunks; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        p[j][i] *= h[j][i] * s;
        most = max(most, magnitude(p[j][i]));
      }
    s = 1.f;
    most = __reduce_max_sync(0xffffffffu, most);
    __syncthreads();
    if (lane == 0) s_max[warp] = most;
    __syncthreads();
    largest = 0u;
    for (int w = 0; w < a.warps_per_row; ++w) largest = max(largest, s_max[team * a.warps_per_row + w]);
  }
#pragma unroll
  for (int j = 0; j < kChunks; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i) p[j][i] *= s;
  if (a.out != nullptr) {
    T* o = static_cast<T*>(a.out) + row * a.out_stride;
#pragma unroll
    for (int j = 0; j < kChunks; ++j) norm_store8<kVec>(o, (wr + j * a.warps_per_row) * kNormChunk, lane, d, p[j]);
  }
  if (a.out8 == nullptr) return;
  uint8_t* q = a.out8 + row * a.out8_stride;
  float* sc = a.scales + row * a.scales_stride;
  if (a.group == 0) {
    float inv;
    const float scale = norm_scale(__uint_as_float(largest) * s, &inv);
    if (active && wr == 0 && lane == 0) sc[0] = scale;
#pragma unroll
    for (int j = 0; j < kChunks; ++j) {
#pragma unroll
      for (int i = 0; i < 8; ++i) p[j][i] *= inv;
      norm_store8_e4m3<kVec>(q, (wr + j * a.warps_per_row) * kNormChunk, lane, d, p[j]);
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < kChunks; ++j) {
    const int c0 = (wr + j * a.warps_per_row) * kNormChunk;
    if constexpr (kVec) {
      // a group is group / 8 neighbouring lanes
      uint32_t m = 0u;
#pragma unroll
      for (int i = 0; i < 8; ++i) m = max(m, magnitude(p[j][i]));
      for (int o = a.group >> 4; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
      float inv;
      const float scale = norm_scale(__uint_as_float(m), &inv);
      const int c = c0 + lane * 8;
      if (c < d && (c & (a.group - 1)) == 0) sc[c / a.group] = scale;
#pragma unroll
      for (int i = 0; i < 8; ++i) p[j][i] *= inv;
    } else {
      // a group is group / 32 of the lanes' columns, over all lanes
      uint32_t m[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) m[i] = __reduce_max_sync(0xffffffffu, magnitude(p[j][i]));
#pragma unroll
      for (int o = 1; o < 8; o <<= 1)
        if (a.group >= 64 * o) {
          uint32_t t[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) t[i] = max(m[i], m[i ^ o]);
#pragma unroll
          for (int i = 0; i < 8; ++i) m[i] = t[i];
        }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float inv;
        const float scale = norm_scale(__uint_as_float(m[i]), &inv);
        const int c = c0 + i * 32;
        if (lane == 0 && c < d && (c & (a.group - 1)) == 0) sc[c / a.group] = scale;
        p[j][i] *= inv;
      }
    }
    norm_store8_e4m3<kVec>(q, c0, lane, d, p[j]);
  }
}

template <typename T, typename R>
inline cudaError_t rms_norm_launch_typed(RmsNormArgs a, bool vec, int sm_count, cudaStream_t st, bool pdl) {
  const int chunks = (a.d + kNormChunk - 1) / kNormChunk;
  // Few rows: a row over as many warps as it has chunks, for the shortest chain.  Else two chunks per warp.
  const bool few = (long long)a.T * chunks <= 8ll * sm_count && chunks <= kNormMaxWarps;
  const int per_warp = few ? 1 : 2;
  a.warps_per_row = (chunks + per_warp - 1) / per_warp;
  a.rows_per_cta = few || a.warps_per_row >= 8 ? 1 : 8 / a.warps_per_row;
  const dim3 grid((unsigned)((a.T + a.rows_per_cta - 1) / a.rows_per_cta)), block(32 * a.warps_per_row * a.rows_per_cta);
  auto go = [&](auto kernel) { return launch_kernel(kernel, grid, block, 0, st, pdl, a); };
  if (vec) return per_warp == 1 ? go(rms_norm_kernel<T, R, 1, true>) : go(rms_norm_kernel<T, R, 2, true>);
  return per_warp == 1 ? go(rms_norm_kernel<T, R, 1, false>) : go(rms_norm_kernel<T, R, 2, false>);
}

}  // namespace swapmoe
