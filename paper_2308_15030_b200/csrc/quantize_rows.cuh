// Rows to 8-bit integers with a scale each:
//   y = x,  relu(x),  or silu(x[0 .. d)) * x[d .. 2 d);  scale = max |y| / 127,  q = y / scale, rounded to nearest, ties to even.
// The scale is the quotient rounded to fp32, and q the quotient by that scale rounded to an integer, as IEEE division gives both.
//
// Bound by HBM and, next to it, by instructions.  A team of warps holds a row in registers between its maximum and its rounding, bf16 rows
// as they are stored, two values a register: a team of eight warps then holds rows of 16384, and as many teams fit an SM as keep
// enough bytes in flight.  A value costs five instructions: products, sums and maxima go two at a time, rounding is the addition of 1.5 2^23, whose
// sum has the integer in its lowest byte.  8192 rows of 14336 bf16: 62 us, 5.7 TB/s (a plain copy 6.5), while few quotients lie next to the middle of two
// integers.  bf16 rows can have many that lie right there, each of which makes its warp divide: one in 200 of normal values without an outlier, 85 us;
// values that are uniform in [0, 1) 110.  With ReLU 137 us, with SwiGLU 191 (normal values; the products keep fp32, half the rows fit an SM).  61 rows of 4096
// 2.0 us.
#pragma once
#include <type_traits>

#include "block_norm.cuh"

namespace swapmoe {

enum { kQuantNone = 0, kQuantRelu = 1, kQuantSwiglu = 2 };
constexpr int kQuantMaxWidth = 32768;

struct QuantizeArgs {
  const void* x;
  uint8_t* out8;
  float* scales;
  long long x_stride, out8_stride;       // elements
  int T, d, act;
  int warps_per_row, rows_per_cta;
};

// The largest magnitude of eight values; NaN if there is one.
__device__ __forceinline__ float largest_of(const RowPiece<float>& p) { return largest8(p.v); }
__device__ __forceinline__ float largest_of(const RowPiece<bf16>& p) {
  uint32_t a, b;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(p.v[0] & 0x7fff7fffu), "r"(p.v[1] & 0x7fff7fffu));
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(b) : "r"(p.v[2] & 0x7fff7fffu), "r"(p.v[3] & 0x7fff7fffu));
  asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(a) : "r"(b));
  return max_magnitude(__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u), 0.f);
}

// silu(x) in fp32, the same bits in every kernel that makes hidden values of it: which of two integers a value next to their border becomes must not
// hang on the form that a call takes.  The exponential is within 2 + 1.17 |x| steps of 2^-23, the quotient as a division rounds it (silu_from_exp).
__device__ __forceinline__ float silu(float x) { return silu_from_exp(x, __expf(-x)); }

// Scale of a row whose largest magnitude is `most`: rows of zeros are divided by 2^-120 and have scale 0.
__device__ __forceinline__ float quantize_divisor(float most) {
  const float q = __fdiv_rn(most, kInt8Max);
  return q < kNormMinScale ? kNormMinScale : q;                        // NaN stays NaN
}

__device__ __forceinline__ void fma2(float& a, float& b, float c, float d, float e, float f) {      // a = c e + a, b = d f + b
  asm("{\n .reg .b64 x, y, z;\n mov.b64 x, {%0, %1};\n mov.b64 y, {%2, %3};\n mov.b64 z, {%4, %5};\n fma.rn.f32x2 x, y, z, x;\n mov.b64 {%0, %1}, x;\n}"
      : "+f"(a), "+f"(b) : "f"(c), "f"(d), "f"(e), "f"(f));
}

// v / scale rounded to integers as the division would be, in the lowest bytes of q.  v * (1 / scale) is off by less than 2^-22 of
// itself, 3e-5 at 127: only a value that lies as near as that to the middle of two integers can be rounded to the wrong one, and then the
// eight are divided (and where the scale is not finite: NaN becomes 0).
__device__ __forceinline__ void quotients8(float (&v)[8], float scale, float inverse, uint32_t (&q)[8]) {
  constexpr float kShift = 12582912.f;   // 1.5 2^23: the sum's last bit is the unit
  float off = 0.f;
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    float a = kShift, b = kShift;
    fma2(a, b, v[i], v[i + 1], inverse, inverse);
    q[i] = __float_as_uint(a); q[i + 1] = __float_as_uint(b);
    add2(a, b, -kShift, -kShift);
    float e = -a, f = -b;
    fma2(e, f, v[i], v[i + 1], inverse, inverse);
    off = max_magnitude(off, e, f);
  }
  if (!(off < 0.5f - 1e-4f)) {
#pragma unroll 1
    for (int i = 0; i < 8; ++i) {
      // (indices known only at run time would put the arrays into memory: they rotate instead)
      const uint32_t r = (uint32_t)__float2int_rn(__fdiv_rn(v[0], scale));
#pragma unroll
      for (int j = 0; j < 7; ++j) { v[j] = v[j + 1]; q[j] = q[j + 1]; }
      q[7] = r;
    }
  }
}
// The lowest bytes of four integers.
__device__ __forceinline__ uint32_t pack_bytes(const uint32_t* q) {
  return __byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410);
}
template <bool kVec>
__device__ __forceinline__ void store8_bytes(uint8_t* row, int c0, int lane, int d, const uint32_t (&q)[8]) {
  if constexpr (kVec) {
    if (c0 + lane * 8 < d) *reinterpret_cast<uint2*>(row + c0 + lane * 8) = make_uint2(pack_bytes(q), pack_bytes(q + 4));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c0 + i * 32 + lane < d) row[c0 + i * 32 + lane] = (uint8_t)q[i];
  }
}

// T: rows; kChunks: chunks per warp; kAct: an activation stands in front.
template <typename T, int kChunks, bool kVec, bool kAct>
__global__ void __launch_bounds__(kChunks == 1 ? 1024 : 512) quantize_rows_kernel(const __grid_constant__ QuantizeArgs a) {
  typedef typename std::conditional<kAct, float, T>::type Kept;
  __shared__ float s_max[kNormMaxWarps];
  const int lane = threadIdx.x & 31, wr = threadIdx.x >> 5, team = threadIdx.y;       // a team per row: blockDim.x threads
  const long long row = (long long)blockIdx.x * a.rows_per_cta + team;
  pdl_wait();
  pdl_trigger();
  const bool active = row < a.T;
  const int d = active ? a.d : 0;        // a team without a row computes on zeros and stores nothing
  auto first = [&](int j) { return (wr + j * a.warps_per_row) * kNormChunk; };
  const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
  RowPiece<Kept> y[kChunks];
  float most = 0.f;
  if constexpr (kAct) {
#pragma unroll
    for (int j = 0; j < kChunks; ++j) norm_load8<kVec>(x, first(j), lane, d, y[j].v);
    if (a.act == kQuantRelu) {
#pragma unroll
      for (int j = 0; j < kChunks; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) y[j].v[i] = y[j].v[i] < 0.f ? 0.f : y[j].v[i];           // NaN stays NaN
    } else {
#pragma unroll
      for (int j = 0; j < kChunks; ++j) {
        float u[8];
        norm_load8<kVec>(x + a.d, first(j), lane, d, u);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[j].v[i] = silu(y[j].v[i]) * u[i];
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < kChunks; ++j) y[j].template load<kVec>(x, first(j), lane, d);
  }
#pragma unroll
  for (int j = 0; j < kChunks; ++j) most = max_magnitude(most, largest_of(y[j]), 0.f);
  most = warp_largest(most);
  if (a.warps_per_row > 1) {
    if (lane == 0) s_max[team * a.warps_per_row + wr] = most;
    __syncthreads();
    for (int w = 0; w < a.warps_per_row; ++w) most = max_magnitude(most, s_max[team * a.warps_per_row + w], 0.f);
  }
  const float scale = quantize_divisor(most);
  const float inverse = __frcp_rn(scale);
  if (active && wr == 0 && lane == 0) a.scales[row] = most == 0.f ? 0.f : scale;
  uint8_t* q = a.out8 + row * a.out8_stride;
#pragma unroll
  for (int j = 0; j < kChunks; ++j) {
    float v[8];
    uint32_t b[8];
    y[j].get(v);
    quotients8(v, scale, inverse, b);
    store8_bytes<kVec>(q, first(j), lane, d, b);
  }
}

template <typename T, bool kAct>
inline cudaError_t quantize_rows_launch_typed(QuantizeArgs a, bool vec, int sm_count, cudaStream_t st, bool pdl) {
  const int chunks = (a.d + kNormChunk - 1) / kNormChunk;
  // Few rows: a row over as many warps as it has chunks, for the shortest chain.  Else as many chunks per warp as leave a row eight warps
  // (16 where they are kept as fp32, and for the widest ones), at least two.
  constexpr int kWarps = sizeof(T) == 2 && !kAct ? 8 : 16;
  int per_warp = 2;
  if ((long long)a.T * chunks <= 8ll * sm_count && chunks <= kNormMaxWarps) per_warp = 1;
  else while (per_warp < 8 && chunks > kWarps * per_warp) per_warp *= 2;
  a.warps_per_row = (chunks + per_warp - 1) / per_warp;
  a.rows_per_cta = per_warp == 1 || a.warps_per_row >= 8 ? 1 : 8 / a.warps_per_row;
  const dim3 grid((unsigned)(((long long)a.T + a.rows_per_cta - 1) / a.rows_per_cta)), block(32 * a.warps_per_row, a.rows_per_cta);
  auto go = [&](auto kernel) { return launch_kernel(kernel, grid, block, 0, st, pdl, a); };
  if (per_warp == 1) return vec ? go(quantize_rows_kernel<T, 1, true, kAct>) : go(quantize_rows_kernel<T, 1, false, kAct>);
  if (per_warp == 2) return vec ? go(quantize_rows_kernel<T, 2, true, kAct>) : go(quantize_rows_kernel<T, 2, false, kAct>);
  if (per_warp == 4) return vec ? go(quantize_rows_kernel<T, 4, true, kAct>) : go(quantize_rows_kernel<T, 4, false, kAct>);
  return vec ? go(quantize_rows_kernel<T, 8, true, kAct>) : go(quantize_rows_kernel<T, 8, false, kAct>);
}

template <typename T>
inline cudaError_t quantize_rows_launch(const QuantizeArgs& a, bool vec, int sm_count, cudaStream_t st, bool pdl) {
  return a.act == kQuantNone ? quantize_rows_launch_typed<T, false>(a, vec, sm_count, st, pdl) : quantize_rows_launch_typed<T, true>(a, vec, sm_count, st, pdl);
}

}  // namespace swapmoe
