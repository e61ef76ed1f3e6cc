// The residual's addition and the root-mean-square norm in front of a layer:
//   h = x + residual,  residual_out = round(h),  y = h * w / sqrt(mean(h^2) + eps),
// y as rows of the layer's dtype, as e4m3 rows with scales (q = y / s, s = max |y| / 448 over a row or a group of columns), or both.
// The norm is taken of the sum before it is rounded, in fp32; every output is rounded once.
//
// Bound by HBM, and next to it by instructions: each row is read once, kept in registers between the sum of squares and the scaling,
// and written once.  A team of warps holds a row, eight columns per lane and chunk of 256; fp32 arithmetic goes two values at a
// time (f32x2).  Where 8-bit rows have one scale y is computed as (h w) s: multiplying by the row's positive factor keeps the order
// of magnitudes, so the largest |y| of a row is the largest |h w| times s to the last bit and is found in the same exchange
// between the warps as the sum of squares.
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

constexpr float kNormLift = 0x1p56f;

struct RmsNormArgs {
  const void *x, *residual, *weight;
  void *residual_out, *out;
  uint8_t* out8;
  float* scales;
  long long x_stride, residual_stride, residual_out_stride, out_stride, out8_stride, scales_stride;   // elements
  int T, d, group;                       // group: columns per scale (0: one scale per row)
  float eps, per_column;                 // per_column: 1 / d
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
      if constexpr (sizeof(T) == 2) {
        const uint4 u = *reinterpret_cast<const uint4*>(row + c0 + lane * 8);
        const uint32_t q[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(q[i] << 16); v[2 * i + 1] = __uint_as_float(q[i] & 0xffff0000u); }
      } else {
        load4(row + c0 + lane * 8, v);
        load4(row + c0 + lane * 8 + 4, v + 4);
      }
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
// Two products, sums at a time.
__device__ __forceinline__ void mul2(float& a, float& b, float c, float d) {
  asm("{\n .reg .b64 x, y;\n mov.b64 x, {%0, %1};\n mov.b64 y, {%2, %3};\n mul.rn.f32x2 x, x, y;\n mov.b64 {%0, %1}, x;\n}"
      : "+f"(a), "+f"(b) : "f"(c), "f"(d));
}
__device__ __forceinline__ void add2(float& a, float& b, float c, float d) {
  asm("{\n .reg .b64 x, y;\n mov.b64 x, {%0, %1};\n mov.b64 y, {%2, %3};\n add.rn.f32x2 x, x, y;\n mov.b64 {%0, %1}, x;\n}"
      : "+f"(a), "+f"(b) : "f"(c), "f"(d));
}
__device__ __forceinline__ void square2(float& a, float& b, float c, float d) {      // a += c c, b += d d
  asm("{\n .reg .b64 x, y;\n mov.b64 x, {%0, %1};\n mov.b64 y, {%2, %3};\n fma.rn.f32x2 x, y, y, x;\n mov.b64 {%0, %1}, x;\n}"
      : "+f"(a), "+f"(b) : "f"(c), "f"(d));
}
// The largest of m, |a|, |b|; NaN if one of them is.
__device__ __forceinline__ float max_magnitude(float m, float a, float b) {
  asm("max.NaN.f32 %0, %0, %1, %2;" : "+f"(m) : "f"(fabsf(a)), "f"(fabsf(b)));
  return m;
}
__device__ __forceinline__ float largest8(const float (&v)[8]) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 8; i += 2) m = max_magnitude(m, v[i], v[i + 1]);
  return m;
}
// (values that are not negative, infinities and NaN among them, are ordered as their bits)
__device__ __forceinline__ float warp_largest(float m) {
  return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(m) & 0x7fffffffu));
}

// Scale of the largest magnitude, and its reciprocal (0 for a row or group of zeros, whose 8-bit values are zeros; NaN for NaN).
__device__ __forceinline__ float norm_scale(float largest, float* inverse) {
  const float s = largest == 0.f ? 0.f : largest * (1.f / kE4m3Max);
  const float t = s < kNormMinScale ? kNormMinScale : s;                // NaN stays NaN
  *inverse = __fdividef(1.f, t);                                       // (t is below 2^119)
  return largest == 0.f ? 0.f : t;
}

// T: rows and weight; R: the residual's rows; kChunks: chunks per warp; kRow8: 8-bit rows with one scale each.
template <typename T, typename R, int kChunks, bool kVec, bool kRow8>
__global__ void __launch_bounds__(kNormMaxWarps * 32) rms_norm_kernel(const __grid_constant__ RmsNormArgs a) {
  __shared__ __align__(16) float s_sum[kNormMaxWarps], s_max[kNormMaxWarps];
  const int lane = threadIdx.x & 31, wr = threadIdx.x >> 5, team = threadIdx.y;       // a team per row: blockDim.x threads
  const int team0 = team * a.warps_per_row, warp = team0 + wr;
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
      for (int i = 0; i < 8; i += 2) add2(h[j][i], h[j][i + 1], p[j][i], p[j][i + 1]);
    if (a.residual_out != nullptr) {
      R* ro = static_cast<R*>(a.residual_out) + row * a.residual_out_stride;
#pragma unroll
      for (int j = 0; j < kChunks; ++j) norm_store8<kVec>(ro, (wr + j * a.warps_per_row) * kNormChunk, lane, d, h[j]);
    }
  }
  if (a.out == nullptr && a.out8 == nullptr) return;                  // the same for the whole grid
  float sum = 0.f, sum1 = 0.f, most = 0.f;
#pragma unroll
  for (int j = 0; j < kChunks; ++j) {
    norm_load8<kVec>(static_cast<const T*>(a.weight), (wr + j * a.warps_per_row) * kNormChunk, lane, d, p[j]);
#pragma unroll
    for (int i = 0; i < 8; i += 2) square2(sum, sum1, h[j][i], h[j][i + 1]);
    if constexpr (kRow8) {
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        float u = h[j][i], v = h[j][i + 1];
        mul2(u, v, kNormLift, kNormLift);
        mul2(p[j][i], p[j][i + 1], u, v);                             // h w 2^56
        most = max_magnitude(most, p[j][i], p[j][i + 1]);
      }
    }
  }
  sum = warp_sum(sum + sum1);
  if constexpr (kRow8) most = warp_largest(most);
  if (lane == 0) {
    s_sum[warp] = sum;
    if constexpr (kRow8) s_max[warp] = most;
  }
  // squares that leave the range of fp32 (rows of 1e18 and more, or below 1e-15 with next to no eps), infinities, NaN
  const bool rare = !(sum < 1e36f) || (kRow8 && !(most < 3e38f)) || (sum < 1e-28f && a.eps < 1e-25f);
  const bool slow = __syncthreads_or(rare) != 0;
  float total = 0.f, largest = 0.f;
  int w = 0;
  for (; w + 4 <= a.warps_per_row && team0 % 4 == 0; w += 4) {
    const float4 t = *reinterpret_cast<const float4*>(s_sum + team0 + w);
    total += (t.x + t.y) + (t.z + t.w);
    if constexpr (kRow8) {
      const float4 m = *reinterpret_cast<const float4*>(s_max + team0 + w);
      largest = fmaxf(largest, fmaxf(fmaxf(m.x, m.y), fmaxf(m.z, m.w)));
    }
  }
  for (; w < a.warps_per_row; ++w) {
    total += s_sum[team0 + w];
    if constexpr (kRow8) largest = fmaxf(largest, s_max[team0 + w]);
  }
  float s = rsqrtf(total * a.per_column + a.eps) * (kRow8 ? 1.f / kNormLift : 1.f);
  if (slow) {
    // For the rows that are rare (a CTA's other rows keep what they have: a row hangs on itself) the same with the row divided by m, the
    // power of two below the larger one of its largest magnitude and sqrt(eps), so that neither square leaves the range:
    // h / sqrt(mean(h^2) + eps) = (h / m) / sqrt(mean((h / m)^2) + eps / m^2)
    auto over_team = [&](float v, bool add) {
      __syncthreads();
      if (lane == 0) s_sum[warp] = v;
      __syncthreads();
      float t = s_sum[team0];
      for (int w = 1; w < a.warps_per_row; ++w) t = add ? t + s_sum[team0 + w] : max_magnitude(t, s_sum[team0 + w], 0.f);
      return t;
    };
    const bool mine = over_team(rare ? 1.f : 0.f, false) > 0.f;
    most = 0.f;
#pragma unroll
    for (int j = 0; j < kChunks; ++j) most = max_magnitude(most, largest8(h[j]), 0.f);
    const float top = over_team(warp_largest(most), false);
    const bool scaled = mine && top > 0.f && top < CUDART_INF_F;
    const uint32_t exponent = __float_as_uint(fmaxf(top, sqrtf(a.eps))) >> 23;                  // (below 2^-126: m = 2^-127)
    const float inverse_m = __uint_as_float(exponent < 254u ? (254u - exponent) << 23 : 0x400000u);
    const float by = scaled ? inverse_m : 1.f;
    sum = 0.f;
    most = 0.f;
#pragma unroll
    for (int j = 0; j < kChunks; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        h[j][i] *= by;
        sum = fmaf(h[j][i], h[j][i], sum);
      }
    total = over_team(warp_sum(sum), true);
    if (mine) s = rsqrtf(total * a.per_column + a.eps * by * by);
    if constexpr (kRow8) {
      // the row's factor goes into the products at once: an infinity among them would be none behind it
      if (mine)
#pragma unroll
        for (int j = 0; j < kChunks; ++j) {
          norm_load8<kVec>(static_cast<const T*>(a.weight), (wr + j * a.warps_per_row) * kNormChunk, lane, d, p[j]);
#pragma unroll
          for (int i = 0; i < 8; ++i) p[j][i] *= h[j][i] * s;
          most = max_magnitude(most, largest8(p[j]), 0.f);
        }
      const float t = over_team(warp_largest(most), false);
      if (mine) {
        s = 1.f;
        largest = t;
      }
    }
  }
  float (&y)[kChunks][8] = kRow8 ? p : h;
#pragma unroll
  for (int j = 0; j < kChunks; ++j)
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      mul2(y[j][i], y[j][i + 1], s, s);
      if constexpr (!kRow8) mul2(y[j][i], y[j][i + 1], p[j][i], p[j][i + 1]);
    }
  if (a.out != nullptr) {
    T* o = static_cast<T*>(a.out) + row * a.out_stride;
#pragma unroll
    for (int j = 0; j < kChunks; ++j) norm_store8<kVec>(o, (wr + j * a.warps_per_row) * kNormChunk, lane, d, y[j]);
  }
  if (a.out8 == nullptr) return;
  uint8_t* q = a.out8 + row * a.out8_stride;
  float* sc = a.scales + row * a.scales_stride;
  if constexpr (kRow8) {
    float inv;
    const float scale = norm_scale(largest * s, &inv);
    if (active && wr == 0 && lane == 0) sc[0] = scale;
#pragma unroll
    for (int j = 0; j < kChunks; ++j) {
#pragma unroll
      for (int i = 0; i < 8; i += 2) mul2(y[j][i], y[j][i + 1], inv, inv);
      norm_store8_e4m3<kVec>(q, (wr + j * a.warps_per_row) * kNormChunk, lane, d, y[j]);
    }
  } else {
    const int shift = 31 - __clz(a.group);
#pragma unroll
    for (int j = 0; j < kChunks; ++j) {
      const int c0 = (wr + j * a.warps_per_row) * kNormChunk;
      if constexpr (kVec) {
        // a group is group / 8 neighbouring lanes
        float m = largest8(y[j]);
        for (int o = a.group >> 4; o > 0; o >>= 1) m = max_magnitude(m, __shfl_xor_sync(0xffffffffu, m, o), 0.f);
        float inv;
        const float scale = norm_scale(m, &inv);
        const int c = c0 + lane * 8;
        if (c < d && (c & (a.group - 1)) == 0) sc[c >> shift] = scale;
#pragma unroll
        for (int i = 0; i < 8; i += 2) mul2(y[j][i], y[j][i + 1], inv, inv);
      } else {
        // a group is group / 32 of the lanes' columns, over all lanes
        float m[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) m[i] = warp_largest(y[j][i]);
#pragma unroll
        for (int o = 1; o < 8; o <<= 1)
          if (a.group >= 64 * o) {
            float t[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) t[i] = max_magnitude(m[i], m[i ^ o], 0.f);
#pragma unroll
            for (int i = 0; i < 8; ++i) m[i] = t[i];
          }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float inv;
          const float scale = norm_scale(m[i], &inv);
          const int c = c0 + i * 32;
          if (lane == 0 && c < d && (c & (a.group - 1)) == 0) sc[c >> shift] = scale;
          y[j][i] *= inv;
        }
      }
      norm_store8_e4m3<kVec>(q, c0, lane, d, y[j]);
    }
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
  const dim3 grid((unsigned)(((long long)a.T + a.rows_per_cta - 1) / a.rows_per_cta)), block(32 * a.warps_per_row, a.rows_per_cta);
  a.per_column = 1.f / (float)a.d;
  auto go = [&](auto kernel) { return launch_kernel(kernel, grid, block, 0, st, pdl, a); };
  const bool row8 = a.out8 != nullptr && a.group == 0;
  if (vec && row8) return few ? go(rms_norm_kernel<T, R, 1, true, true>) : go(rms_norm_kernel<T, R, 2, true, true>);
  if (vec) return few ? go(rms_norm_kernel<T, R, 1, true, false>) : go(rms_norm_kernel<T, R, 2, true, false>);
  if (row8) return few ? go(rms_norm_kernel<T, R, 1, false, true>) : go(rms_norm_kernel<T, R, 2, false, true>);
  return few ? go(rms_norm_kernel<T, R, 1, false, false>) : go(rms_norm_kernel<T, R, 2, false, false>);
}

}  // namespace swapmoe
