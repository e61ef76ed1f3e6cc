// The norms behind and in front of a block, with the block's gate and residual scale between them:
//   p = x * wp / sqrt(mean(x^2) + eps_p),  h = residual + scale * gate * p,  residual_out = round(h),
//   y = h * w / sqrt(mean(h^2) + eps),
// y as rows of the layer's dtype, in 8 bits (e4m3 or integers) with scales, or both.  All in fp32; every output is rounded once, and the
// second norm is taken of the sum before it is rounded.
//
// Bound by HBM, and next to it by the chain of a row: loads, an exchange between the warps for each sum, weights, stores.  A team of warps
// holds a row, eight columns per lane and chunk of 256, and an SM as many teams as its registers hold; x and a bf16 residual stay packed until
// they are added.  Four CTAs of eight warps an SM, 64 registers a thread: at five the kernel spills 28 to 36 bytes a thread (16384 x 4096 bf16 on an fp32
// residual, gate, rows out 131 us, 124 with four; e4m3 by groups 142, 135; integers with one scale 143, 138).  Where 8-bit rows have one scale, the largest |h w| of the
// row is found in the same exchange as the second sum: the largest |y| is that times the row's positive factor, to three roundings (y is (h s) w).
// 8-bit values are products with the scale's reciprocal: dividing instead, as quantize_rows does, takes longer (16384 rows of 4096 to integers
// with one scale 138 -> 148 us), for integers that differ where y's own error decides.
// 16384 rows of 4096, bf16 on an fp32 residual, to 8-bit groups of 128: 133 us, 5.6 TB/s (a plain copy 6.5); one row of 4096 2.4 us.
#pragma once
#include "rms_norm.cuh"

namespace swapmoe {

constexpr float kInt8Max = 127.f;
constexpr int kBlockNormCtas = 4;        // CTAs of eight warps an SM

struct BlockNormArgs {
  const void *x, *residual, *post_weight, *gate, *weight;
  void *residual_out, *out;
  uint8_t* out8;
  float* scales;
  long long x_stride, residual_stride, gate_stride, residual_out_stride, out_stride, out8_stride, scales_stride;   // elements
  int T, d, group;                       // group: columns per scale (0: one scale per row)
  int int8;                              // 8-bit rows are integers (else e4m3)
  float eps, post_eps, scale, per_column;
  int warps_per_row, rows_per_cta;
};

// Four values to 8-bit integers (nearest, ties to even; NaN: 0).
__device__ __forceinline__ uint32_t pack_int8x4(float a, float b, float c, float d) {
  const uint32_t lo = __byte_perm(__float2int_rn(a), __float2int_rn(b), 0x0040);
  return __byte_perm(lo, __byte_perm(__float2int_rn(c), __float2int_rn(d), 0x0040), 0x5410);
}
template <bool kVec>
__device__ __forceinline__ void store8_int8(uint8_t* row, int c0, int lane, int d, const float (&v)[8]) {
  if constexpr (kVec) {
    if (c0 + lane * 8 < d)
      *reinterpret_cast<uint2*>(row + c0 + lane * 8) = make_uint2(pack_int8x4(v[0], v[1], v[2], v[3]), pack_int8x4(v[4], v[5], v[6], v[7]));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c0 + i * 32 + lane < d) row[c0 + i * 32 + lane] = (uint8_t)__float2int_rn(v[i]);
  }
}
// Scale of the largest magnitude (two roundings from the quotient), and the factor that takes values to the 8-bit type (0 for zeros, NaN for NaN).
__device__ __forceinline__ float scale8(float largest, float inverse_max, float* inverse) {
  const float s = largest * inverse_max, t = s < kNormMinScale ? kNormMinScale : s;         // NaN stays NaN
  *inverse = __fdividef(1.f, t);                                       // (t is below 2^122)
  return largest == 0.f ? 0.f : t;
}

// What the warps of a row's team agree on.  Every thread of the CTA takes each step.
struct NormTeam {
  float *s_sum, *s_max;
  int lane, warp, first, n;              // this warp and its team's first one in the CTA; warps of the team

  // Sums and maxima of the team; returns whether any row of the CTA is rare.
  template <bool kMax>
  __device__ __forceinline__ bool exchange(float& sum, float& most, bool rare_most, float eps, bool* rare) const {
    sum = warp_sum(sum);
    if constexpr (kMax) most = warp_largest(most);
    // squares that leave the range of fp32 (rows of 1e18 and more, or below 1e-15 with next to no eps), infinities, NaN
    *rare = !(sum < 1e36f) || (sum < 1e-28f && eps < 1e-25f);
    if constexpr (kMax) *rare = *rare || (rare_most && (!(most < 1e36f) || (most < 1e-25f && most > 0.f)));
    __syncthreads();                     // the exchange before has been read
    if (lane == 0) {
      s_sum[warp] = sum;
      if constexpr (kMax) s_max[warp] = most;
    }
    const bool any = __syncthreads_or(*rare) != 0;
    float t = 0.f, m = 0.f;
    int w = 0;
    for (; w + 4 <= n && first % 4 == 0; w += 4) {
      const float4 u = *reinterpret_cast<const float4*>(s_sum + first + w);
      t += (u.x + u.y) + (u.z + u.w);
      if constexpr (kMax) {
        const float4 v = *reinterpret_cast<const float4*>(s_max + first + w);
        m = fmaxf(m, fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w)));
      }
    }
    for (; w < n; ++w) {
      t += s_sum[first + w];
      if constexpr (kMax) m = fmaxf(m, s_max[first + w]);
    }
    sum = t;
    if constexpr (kMax) most = m;
    return any;
  }
  __device__ __forceinline__ float over(float v, bool add) const {
    __syncthreads();
    if (lane == 0) s_sum[warp] = v;
    __syncthreads();
    float t = s_sum[first];
    for (int w = 1; w < n; ++w) t = add ? t + s_sum[first + w] : max_magnitude(t, s_sum[first + w], 0.f);
    return t;
  }
  // The factors of a rare row (others keep theirs: a row hangs on itself): values are multiplied by `by` first, the reciprocal of the power of
  // two m below the larger one of their largest magnitude and sqrt(eps), so that neither square leaves the range:
  // v / sqrt(mean(v^2) + eps) = (v / m) / sqrt(mean((v / m)^2) + eps / m^2)
  template <int kChunks, typename Values>
  __device__ __forceinline__ bool rescale(Values values, bool rare, float eps, float per_column, float* by, float* s) const {
    const bool mine = over(rare ? 1.f : 0.f, false) > 0.f;
    float most = 0.f, v[8];
#pragma unroll 1
    for (int j = 0; j < kChunks; ++j) {
      values(j, v);
      most = max_magnitude(most, largest8(v), 0.f);
    }
    const float top = over(warp_largest(most), false);
    const uint32_t exponent = __float_as_uint(fmaxf(top, sqrtf(eps))) >> 23;                    // (below 2^-126: m = 2^-127)
    const float f = mine && top > 0.f && top < CUDART_INF_F ? __uint_as_float(exponent < 254u ? (254u - exponent) << 23 : 0x400000u) : 1.f;
    float sum = 0.f;
#pragma unroll 1
    for (int j = 0; j < kChunks; ++j) {
      values(j, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fmaf(v[i] * f, v[i] * f, sum);
    }
    const float total = over(warp_sum(sum), true);
    if (mine) {
      *by = f;
      *s = rsqrtf(total * per_column + eps * f * f);
    }
    return mine;
  }
};

// Eight values of a row as they are stored.
template <typename S> struct RowPiece;
template <> struct RowPiece<float> {
  float v[8];
  template <bool kVec>
  __device__ __forceinline__ void load(const float* row, int c0, int lane, int d) { norm_load8<kVec>(row, c0, lane, d, v); }
  __device__ __forceinline__ void get(float (&f)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = v[i];
  }
};
template <> struct RowPiece<bf16> {
  uint32_t v[4];
  template <bool kVec>
  __device__ __forceinline__ void load(const bf16* row, int c0, int lane, int d) {
    if constexpr (kVec) {
      const uint4 u = c0 + lane * 8 < d ? *reinterpret_cast<const uint4*>(row + c0 + lane * 8) : make_uint4(0u, 0u, 0u, 0u);
      v[0] = u.x; v[1] = u.y; v[2] = u.z; v[3] = u.w;
    } else {
      const uint16_t* r = reinterpret_cast<const uint16_t*>(row);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int c = c0 + 2 * i * 32 + lane;
        v[i] = (c < d ? r[c] : 0u) | (c + 32 < d ? (uint32_t)r[c + 32] << 16 : 0u);
      }
    }
  }
  __device__ __forceinline__ void get(float (&f)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(v[i] << 16); f[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u); }
  }
};

// T: x, weights, gate, out; R: the residual's rows; kChunks: chunks per warp; kRow8: 8-bit rows with one scale each; kThreads, kCtas: most
// threads of a CTA, CTAs that an SM is to hold.
template <typename T, typename R, int kChunks, bool kVec, bool kRow8, int kThreads, int kCtas>
__global__ void __launch_bounds__(kThreads, kCtas) block_norm_kernel(const __grid_constant__ BlockNormArgs a) {
  __shared__ __align__(16) float s_sum[kNormMaxWarps], s_max[kNormMaxWarps];
  const int lane = threadIdx.x & 31, wr = threadIdx.x >> 5, team = threadIdx.y;       // a team per row: blockDim.x threads
  const NormTeam tm = {s_sum, s_max, lane, team * a.warps_per_row + wr, team * a.warps_per_row, a.warps_per_row};
  const long long row = (long long)blockIdx.x * a.rows_per_cta + team;
  const bool active = row < a.T;
  const int d = active ? a.d : 0;        // a team without a row computes on zeros and stores nothing
  auto first = [&](int j) { return (wr + j * a.warps_per_row) * kNormChunk; };
  RowPiece<T> x[kChunks];
  RowPiece<R> r[kChunks];
  float h[kChunks][8];
  pdl_wait();
  pdl_trigger();
  {
    const T* xs = static_cast<const T*>(a.x) + row * a.x_stride;
    const R* rs = static_cast<const R*>(a.residual) + row * a.residual_stride;
#pragma unroll
    for (int j = 0; j < kChunks; ++j) x[j].template load<kVec>(xs, first(j), lane, d);
#pragma unroll
    for (int j = 0; j < kChunks; ++j) r[j].template load<kVec>(rs, first(j), lane, a.residual != nullptr ? d : 0);
  }
  bool rare;
  float s = 1.f, by = 1.f, none = 0.f;
  if (a.post_weight != nullptr) {
    float sum = 0.f, sum1 = 0.f;
#pragma unroll
    for (int j = 0; j < kChunks; ++j) {
      float v[8];
      x[j].get(v);
#pragma unroll
      for (int i = 0; i < 8; i += 2) square2(sum, sum1, v[i], v[i + 1]);
    }
    sum += sum1;
    const bool slow = tm.exchange<false>(sum, none, false, a.post_eps, &rare);
    s = rsqrtf(sum * a.per_column + a.post_eps);
    if (slow) {
      auto block = [&](int j, float (&v)[8]) {
#pragma unroll
        for (int k = 0; k < kChunks; ++k)
          if (k == j) x[k].get(v);
      };
      tm.rescale<kChunks>(block, rare, a.post_eps, a.per_column, &by, &s);
    }
  }
  const T* gate = static_cast<const T*>(a.gate) + row * a.gate_stride;
  R* ro = static_cast<R*>(a.residual_out) + row * a.residual_out_stride;
#pragma unroll
  for (int j = 0; j < kChunks; ++j) {
    float v[8], w[8];
    x[j].get(v);
    if (a.post_weight != nullptr) {
      norm_load8<kVec>(static_cast<const T*>(a.post_weight), first(j), lane, d, w);
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        mul2(v[i], v[i + 1], by, by);
        mul2(v[i], v[i + 1], s, s);
        mul2(v[i], v[i + 1], w[i], w[i + 1]);
      }
    }
    if (a.gate != nullptr) {
      norm_load8<kVec>(gate, first(j), lane, d, w);
#pragma unroll
      for (int i = 0; i < 8; i += 2) mul2(v[i], v[i + 1], w[i], w[i + 1]);
    }
    r[j].get(h[j]);
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      mul2(v[i], v[i + 1], a.scale, a.scale);
      add2(h[j][i], h[j][i + 1], v[i], v[i + 1]);
    }
    if (a.residual_out != nullptr) norm_store8<kVec>(ro, first(j), lane, d, h[j]);
  }
  if (a.out == nullptr && a.out8 == nullptr) return;                  // the same for the whole grid
  float sum = 0.f, sum1 = 0.f, most = 0.f;
#pragma unroll
  for (int j = 0; j < kChunks; ++j) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) square2(sum, sum1, h[j][i], h[j][i + 1]);
    if constexpr (kRow8) {
      float w[8];
      norm_load8<kVec>(static_cast<const T*>(a.weight), first(j), lane, d, w);
#pragma unroll
      for (int i = 0; i < 8; i += 2) most = max_magnitude(most, h[j][i] * w[i], h[j][i + 1] * w[i + 1]);
    }
  }
  sum += sum1;
  const bool slow = tm.exchange<kRow8>(sum, most, true, a.eps, &rare);
  s = rsqrtf(sum * a.per_column + a.eps);
  by = 1.f;
  float largest = most * s;
  bool mine = false;
  if (slow) {
    auto stream = [&](int j, float (&v)[8]) {
#pragma unroll
      for (int k = 0; k < kChunks; ++k)
        if (k == j)
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = h[k][i];
    };
    mine = tm.rescale<kChunks>(stream, rare, a.eps, a.per_column, &by, &s);
  }
  T* o = static_cast<T*>(a.out) + row * a.out_stride;
#pragma unroll
  for (int j = 0; j < kChunks; ++j) {
    float w[8];
    norm_load8<kVec>(static_cast<const T*>(a.weight), first(j), lane, d, w);
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      if (slow) mul2(h[j][i], h[j][i + 1], by, by);
      mul2(h[j][i], h[j][i + 1], s, s);
      mul2(h[j][i], h[j][i + 1], w[i], w[i + 1]);                     // y
    }
    if (a.out != nullptr) norm_store8<kVec>(o, first(j), lane, d, h[j]);
  }
  if (a.out8 == nullptr) return;
  if constexpr (kRow8) {
    if (slow) {
      most = 0.f;
#pragma unroll
      for (int j = 0; j < kChunks; ++j) most = max_magnitude(most, largest8(h[j]), 0.f);
      const float t = tm.over(warp_largest(most), false);
      if (mine) largest = t;
    }
  }
  uint8_t* q = a.out8 + row * a.out8_stride;
  float* sc = a.scales + row * a.scales_stride;
  const float inverse_max = a.int8 ? 1.f / kInt8Max : 1.f / kE4m3Max;
  auto store = [&](int c0, float (&v)[8]) {
    if (a.int8) store8_int8<kVec>(q, c0, lane, d, v);
    else norm_store8_e4m3<kVec>(q, c0, lane, d, v);
  };
  if constexpr (kRow8) {
    float inv;
    const float scale = scale8(largest, inverse_max, &inv);
    if (active && wr == 0 && lane == 0) sc[0] = scale;
#pragma unroll
    for (int j = 0; j < kChunks; ++j) {
#pragma unroll
      for (int i = 0; i < 8; i += 2) mul2(h[j][i], h[j][i + 1], inv, inv);
      store(first(j), h[j]);
    }
  } else {
    const int shift = 31 - __clz(a.group);
    if constexpr (kVec) {
      // a group is group / 8 neighbouring lanes; the chunks' exchanges go side by side
      float m[kChunks];
#pragma unroll
      for (int j = 0; j < kChunks; ++j) m[j] = largest8(h[j]);
#pragma unroll 1
      for (int o = a.group >> 4; o > 0; o >>= 1)
#pragma unroll
        for (int j = 0; j < kChunks; ++j) m[j] = max_magnitude(m[j], __shfl_xor_sync(0xffffffffu, m[j], o), 0.f);
#pragma unroll
      for (int j = 0; j < kChunks; ++j) {
        float inv;
        const float scale = scale8(m[j], inverse_max, &inv);
        const int c = first(j) + lane * 8;
        if (c < d && (c & (a.group - 1)) == 0) sc[c >> shift] = scale;
#pragma unroll
        for (int i = 0; i < 8; i += 2) mul2(h[j][i], h[j][i + 1], inv, inv);
        store(first(j), h[j]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < kChunks; ++j) {
        // a group is group / 32 of the lanes' columns, over all lanes
        float m[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) m[i] = warp_largest(h[j][i]);
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
          const float scale = scale8(m[i], inverse_max, &inv);
          const int c = first(j) + i * 32;
          if (lane == 0 && c < d && (c & (a.group - 1)) == 0) sc[c >> shift] = scale;
          h[j][i] *= inv;
        }
        store(first(j), h[j]);
      }
    }
  }
}

template <typename T, typename R>
inline cudaError_t block_norm_launch_typed(BlockNormArgs a, bool vec, int sm_count, cudaStream_t st, bool pdl) {
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
  constexpr int kWide = 32 * kNormMaxWarps, kCtas = kBlockNormCtas;
  if (vec && few) return row8 ? go(block_norm_kernel<T, R, 1, true, true, kWide, 1>) : go(block_norm_kernel<T, R, 1, true, false, kWide, 1>);
  if (vec && a.warps_per_row <= 8)
    return row8 ? go(block_norm_kernel<T, R, 2, true, true, 256, kCtas>) : go(block_norm_kernel<T, R, 2, true, false, 256, kCtas>);
  if (vec) return row8 ? go(block_norm_kernel<T, R, 2, true, true, kWide, 1>) : go(block_norm_kernel<T, R, 2, true, false, kWide, 1>);
  if (few) return row8 ? go(block_norm_kernel<T, R, 1, false, true, kWide, 1>) : go(block_norm_kernel<T, R, 1, false, false, kWide, 1>);
  return row8 ? go(block_norm_kernel<T, R, 2, false, true, kWide, 1>) : go(block_norm_kernel<T, R, 2, false, false, kWide, 1>);
}

}  // namespace swapmoe
