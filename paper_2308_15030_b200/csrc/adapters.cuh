// Low-rank adapters of many requests beside a projection that all of them share:
//   out[t] = y[t] + scale_a * B_a (A_a x[t]),  a = ids[t]  (no adapter: out[t] = y[t]),
// A_a [rank, d_in], B_a [d_out, rank], y the shared projection's row.
//
// Bound by bytes: x, y and out once, the adapters that are asked for once per tile of tokens; the products are rank * 2 operations
// per element of x and out.  One launch does both products.  Tokens of one adapter form tiles of up to 32; a cluster of 1 to 8 CTAs
// takes a tile and splits the columns of x, then those of out.  All operands go from global memory straight to the registers of
// the warp that multiplies them (warp-level mma, tokens as mma rows), 64 contiguous bytes of eight rows per load:
//  - first product: the contraction is dealt out to the warps in steps of 64 bytes, so that a step's x and A belong to one warp
//    (two or four warps share x from rank 40 on).  Within a step a lane's 16-byte piece holds its operands of two (bf16) mma: the
//    contraction index is permuted the same way on both sides.  The warps' sums are added in shared memory, the CTAs' through
//    distributed shared memory, in a fixed order.
//  - second product: a warp owns 64 bytes of columns of all the tile's rows; the columns are dealt out to the mma's column tiles
//    so that a lane's results are 16 contiguous bytes of a row, and y is read and out written from registers.
// (With chunks of x and y staged in shared memory by bulk copies of 256 bytes, 8192 x 4096 at rank 64 took 229 us: issuing
// 768 such copies per CTA takes longer than moving them.)
#pragma once
#include <cuda_fp8.h>

#include "common.cuh"
#include "launch.cuh"

namespace swapmoe {

constexpr int kAdMaxRank = 128, kAdMaxCount = 4096, kAdMaxWidth = 1 << 16;
constexpr int kAdThreads = 256, kAdWarps = kAdThreads / 32;
constexpr int kAdMaxCtas = 8;              // most CTAs per cluster
constexpr int kAdTile = 32, kAdMT = kAdTile / 16;   // tokens of a tile; mma row tiles
constexpr int kAdDirect = 64;              // up to this many tokens every cluster finds its tile itself

struct AdapterTile { int32_t adapter, first, rows, pad; };   // tokens perm[first] ... perm[first + rows - 1]; adapter -1: none

struct AdapterArgs {
  const void* x;            // [T, d] rows of T or e4m3
  const float* x_scales;    // [T] with e4m3 rows
  const int32_t* ids;       // [T]
  const void* y;            // [T, n] or nullptr (zeros)
  void* out;                // [T, n]
  const void *A, *B;        // [count, r, d], [count, n, r]
  const float* scale;       // [count] or nullptr (ones)
  long long x_stride, y_stride, out_stride;
  int T, d, n, r, count;
  int ctas;                 // CTAs per cluster
  int32_t* perm;            // [T]            } written by the plan kernel, for more than kAdDirect tokens
  AdapterTile* tiles;       // [max tiles]    }
  int32_t* n_tiles;         // [1]            }
};

// ----------------------------------------------------------------------------- plan
constexpr int kAdPlanThreads = 1024;

// Groups the tokens by adapter and cuts the groups into tiles of at most `tile_rows`.  One CTA: counts per adapter, their
// exclusive scans, then every token takes a place in its group.  (Which place is left to the order of atomics; a row's result does
// not depend on it.)
__global__ void __launch_bounds__(kAdPlanThreads) adapters_plan_kernel(const AdapterArgs a, int tile_rows) {
  __shared__ int32_t s_cursor[kAdMaxCount + 1];
  __shared__ int32_t s_warp[2][32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_wait();
  pdl_trigger();
  const int groups = a.count + 1;                           // the last one: tokens without an adapter
  for (int g = tid; g < groups; g += kAdPlanThreads) s_cursor[g] = 0;
  __syncthreads();
  auto group_of = [&](int t) {
    const int id = a.ids[t];
    return id < 0 || id >= a.count ? a.count : id;
  };
  for (int t0 = warp * 32; t0 < a.T; t0 += kAdPlanThreads) {
    const int g = t0 + lane < a.T ? group_of(t0 + lane) : -1;
    const uint32_t same = __match_any_sync(0xffffffffu, g);  // runs of one adapter: one atomic per warp
    if (g >= 0 && __ffs(same) - 1 == lane) atomicAdd(&s_cursor[g], __popc(same));
  }
  __syncthreads();
  // thread i owns groups i * per ... : sums, scan over the threads, then first rows and tiles of its groups
  const int per = (groups + kAdPlanThreads - 1) / kAdPlanThreads, g0 = tid * per;
  int rows = 0, tiles = 0;
  for (int g = g0; g < min(groups, g0 + per); ++g) {
    rows += s_cursor[g];
    tiles += (s_cursor[g] + tile_rows - 1) / tile_rows;
  }
  int row_incl = rows, tile_incl = tiles;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, row_incl, o), v = __shfl_up_sync(0xffffffffu, tile_incl, o);
    if (lane >= o) { row_incl += u; tile_incl += v; }
  }
  if (lane == 31) { s_warp[0][warp] = row_incl; s_warp[1][warp] = tile_incl; }
  __syncthreads();
  int row = row_incl - rows, tile = tile_incl - tiles;
  for (int w = 0; w < warp; ++w) { row += s_warp[0][w]; tile += s_warp[1][w]; }
  for (int g = g0; g < min(groups, g0 + per); ++g) {
    const int n = s_cursor[g], cut = (n + tile_rows - 1) / tile_rows;
    const int each = cut > 0 ? (n + cut - 1) / cut : 0;     // tiles of equal height
    for (int i = 0; i < cut; ++i)
      a.tiles[tile + i] = {g < a.count ? g : -1, row + i * each, min(each, n - i * each), 0};
    s_cursor[g] = row;
    row += n;
    tile += cut;
  }
  if (tid == kAdPlanThreads - 1) *a.n_tiles = tile;
  __syncthreads();
  for (int t0 = warp * 32; t0 < a.T; t0 += kAdPlanThreads) {
    const int t = t0 + lane, g = t < a.T ? group_of(t) : -1;
    const uint32_t same = __match_any_sync(0xffffffffu, g);
    const int leader = __ffs(same) - 1;
    int base = 0;
    if (g >= 0 && leader == lane) base = atomicAdd(&s_cursor[g], __popc(same));
    base = __shfl_sync(0xffffffffu, base, leader);
    if (g >= 0) a.perm[base + __popc(same & ((1u << lane) - 1))] = t;
  }
}

// ----------------------------------------------------------------------------- fragments and products
__device__ __forceinline__ void mma_bf16_16x8x16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                                 uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ad_mma_tf32(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                            uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// x = hi + lo, both TF32, each rounded to nearest: what is lost is below 2^-22 of x.
__device__ __forceinline__ void ad_split(uint32_t x, uint32_t& hi, uint32_t& lo) {
  asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(hi) : "f"(__uint_as_float(x)));
  asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(lo) : "f"(__uint_as_float(x) - __uint_as_float(hi)));
}
// c += one step of 64 bytes: rows g and g + 8 of the left operand (pieces p, p8), row g of the right one (w).
__device__ __forceinline__ void ad_step(float (&c)[4], const uint4& p, const uint4& p8, const uint4& w, bf16) {
  mma_bf16_16x8x16(c, p.x, p8.x, p.y, p8.y, w.x, w.y);
  mma_bf16_16x8x16(c, p.z, p8.z, p.w, p8.w, w.z, w.w);
}
__device__ __forceinline__ void ad_step(float (&c)[4], const uint4& p, const uint4& p8, const uint4& w, float) {
  // fp32 products as three of TF32 pieces (lo * lo is below 2^-22)
  auto two = [&](uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    uint32_t h[6], l[6];
    ad_split(a0, h[0], l[0]); ad_split(a1, h[1], l[1]); ad_split(a2, h[2], l[2]); ad_split(a3, h[3], l[3]);
    ad_split(b0, h[4], l[4]); ad_split(b1, h[5], l[5]);
    ad_mma_tf32(c, l[0], l[1], l[2], l[3], h[4], h[5]);
    ad_mma_tf32(c, h[0], h[1], h[2], h[3], l[4], l[5]);
    ad_mma_tf32(c, h[0], h[1], h[2], h[3], h[4], h[5]);
  };
  two(p.x, p8.x, p.y, p8.y, w.x, w.y);
  two(p.z, p8.z, p.w, p8.w, w.z, w.w);
}
// Two e4m3 values as two bf16 (exact).
__device__ __forceinline__ uint32_t e4m3x2_to_bf16x2(uint32_t v) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(v & 0xffffu), __NV_E4M3);
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
  return pack_bf16x2(f.x, f.y);
}
// A lane's piece of a row of x as it is loaded, and as an operand.
template <typename X> struct AdPiece { typedef uint4 type; };
template <> struct AdPiece<__nv_fp8_e4m3> { typedef uint2 type; };
__device__ __forceinline__ uint4 ad_operand(const uint4& v) { return v; }
__device__ __forceinline__ uint4 ad_operand(const uint2& v) {
  return make_uint4(e4m3x2_to_bf16x2(v.x), e4m3x2_to_bf16x2(v.x >> 16), e4m3x2_to_bf16x2(v.y), e4m3x2_to_bf16x2(v.y >> 16));
}
__device__ __forceinline__ void ad_zero(uint4& v) { v = make_uint4(0u, 0u, 0u, 0u); }
__device__ __forceinline__ void ad_zero(uint2& v) { v = make_uint2(0u, 0u); }
__device__ __forceinline__ void ad_store_u(float* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }
__device__ __forceinline__ void ad_store_u(bf16* p, float4 v) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
}
// Two neighbouring values of y, plus the sums, rounded once.
__device__ __forceinline__ uint32_t ad_add2(uint32_t y, float d0, float d1) {
  return pack_bf16x2(__uint_as_float(y << 16) + d0, __uint_as_float(y & 0xffff0000u) + d1);
}
// A lane's 16 bytes of out from those of y and its accumulators of a row (columns 2 h, 2 h + 1 in tile h).
__device__ __forceinline__ uint4 ad_finish(const uint4& y, const float (&c)[4][4], int e, bf16) {
  return make_uint4(ad_add2(y.x, c[0][e], c[0][e + 1]), ad_add2(y.y, c[1][e], c[1][e + 1]), ad_add2(y.z, c[2][e], c[2][e + 1]),
                    ad_add2(y.w, c[3][e], c[3][e + 1]));
}
__device__ __forceinline__ uint4 ad_finish(const uint4& y, const float (&c)[2][4], int e, float) {
  return make_uint4(__float_as_uint(__uint_as_float(y.x) + c[0][e]), __float_as_uint(__uint_as_float(y.y) + c[0][e + 1]),
                    __float_as_uint(__uint_as_float(y.z) + c[1][e]), __float_as_uint(__uint_as_float(y.w) + c[1][e + 1]));
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
__device__ __forceinline__ float4 ld_cluster4(const float* mine, int cta) {        // the same place in that CTA's shared memory
  uint32_t at;
  float4 v;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(mine)), "r"(cta));
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
  return v;
}

// Rank tiles (of eight ranks) that a warp accumulates, warps side by side over the ranks, warps over the contraction.
__host__ __device__ constexpr int ad_rank_warps(int r, int rtw) {
  const int w = (r / 8 + rtw - 1) / rtw;
  return w <= 1 ? 1 : w <= 2 ? 2 : 4;
}
__host__ __device__ constexpr int ad_rtw(int r) { return r <= 8 ? 1 : r <= 16 ? 2 : 4; }
// Pitch of u in shared memory: fragments (lanes g, q read piece q of row g) are free of bank conflicts at 64 bytes modulo 128.
__host__ __device__ constexpr int ad_u_pitch(int r, int elem) {
  const int b = (r * elem + 63) & ~63;
  return b % 128 == 0 ? b + 64 : b;
}
__host__ __device__ constexpr int ad_part_bytes(int r) { return kAdWarps / ad_rank_warps(r, ad_rtw(r)) * kAdTile * r * 4; }
__host__ __device__ constexpr int ad_smem_bytes(int r, int elem) { return ad_part_bytes(r) + kAdTile * ad_u_pitch(r, elem) + kAdTile * 4 + 16; }

// The tile of cluster i without a plan: it has one if token i is the first, or the 32nd, ... of its adapter; then its tokens
// are the next 32 of that adapter from i on.  By one warp; T <= 64: lane l holds tokens l and l + 32.
__device__ __forceinline__ int ad_direct_tile(const AdapterArgs& a, int i, int32_t* list, int* adapter) {
  const int lane = threadIdx.x & 31;
  int id[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int t = lane + 32 * h;
    id[h] = t < a.T ? a.ids[t] : -2;
    if (t < a.T && (id[h] < 0 || id[h] >= a.count)) id[h] = -1;
  }
  const int mine = __shfl_sync(0xffffffffu, i < 32 ? id[0] : id[1], i & 31);
  const unsigned long long all = (unsigned long long)__ballot_sync(0xffffffffu, id[1] == mine) << 32 |
                                 __ballot_sync(0xffffffffu, id[0] == mine);
  const unsigned long long below = (1ull << i) - 1;
  *adapter = mine;
  if (__popcll(all & below) % kAdTile != 0) return 0;
  const unsigned long long rest = all & ~below;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int t = lane + 32 * h, at = __popcll(rest & ((1ull << t) - 1));
    if ((rest >> t) & 1 && at < kAdTile) list[at] = t;
  }
  return min(kAdTile, __popcll(rest));
}

// X: rows of x (T or e4m3), T: everything else, RTW: rank tiles per warp.
template <typename X, typename T, int RTW>
__global__ void __launch_bounds__(kAdThreads, 2) adapters_kernel(const AdapterArgs a) {
  constexpr int kElem = (int)sizeof(T);
  constexpr int P = 16 / kElem;                  // values of a lane's piece; a step or unit is 4 P values
  constexpr int NT = P / 2;                      // column tiles of a unit of out
  typedef typename AdPiece<X>::type XPiece;
  extern __shared__ __align__(128) unsigned char smem[];
  const int r = a.r, rank_tiles = r / 8, u_pitch = ad_u_pitch(r, kElem);
  const int rank_warps = ad_rank_warps(r, RTW), slices = kAdWarps / rank_warps;
  float* part = reinterpret_cast<float*>(smem);                                 // [slices][tile][r]
  unsigned char* us = smem + ad_part_bytes(r);                                  // [tile] rows of u in T
  int32_t* list = reinterpret_cast<int32_t*>(us + kAdTile * u_pitch);           // [tile] tokens
  volatile int* ctl = list + kAdTile;                                           // rows, adapter
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), g = lane >> 2, q = lane & 3;
  const int C = a.ctas, cta = blockIdx.x % C, cluster = blockIdx.x / C, n_clusters = gridDim.x / C;
  pdl_wait();
  pdl_trigger();
  const bool direct = a.T <= kAdDirect;
  const int n_tiles = direct ? a.T : *a.n_tiles;
  const X* x = static_cast<const X*>(a.x);
  const T* y = static_cast<const T*>(a.y);
  T* out = static_cast<T*>(a.out);
  bool owe_wait = false;                         // this CTA has told the others that it has read their parts
#pragma unroll 1
  for (int tile = cluster; tile < n_tiles; tile += n_clusters) {
    __syncthreads();                             // the tile in front is done with the list
    if (direct) {
      if (warp == 0) {
        int adapter;
        const int rows = ad_direct_tile(a, tile, list, &adapter);
        if (lane == 0) { ctl[0] = rows; ctl[1] = adapter; }
      }
    } else {
      const AdapterTile td = a.tiles[tile];
      if (tid < td.rows) list[tid] = a.perm[td.first + tid];
      if (tid == 0) { ctl[0] = td.rows; ctl[1] = td.adapter; }
    }
    __syncthreads();
    const int rows = ctl[0], adapter = ctl[1];
    if (rows == 0) continue;                     // the same for the whole cluster
    const int mt = (rows + 15) >> 4;
    const bool work = adapter >= 0;
    // the lane's rows: g + 8 i; a row that the tile does not have repeats the first one and is not stored
    int token[2 * kAdMT];
#pragma unroll
    for (int i = 0; i < 2 * kAdMT; ++i) token[i] = list[g + 8 * i < rows ? g + 8 * i : 0];
    if (work) {
      // ---- first product
      const T* A = static_cast<const T*>(a.A) + (long long)adapter * r * a.d;
      const int slice = warp / rank_warps, rt0 = (warp % rank_warps) * RTW;
      float acc[RTW][kAdMT][4];
#pragma unroll
      for (int h = 0; h < RTW; ++h)
#pragma unroll
        for (int m = 0; m < kAdMT; ++m)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[h][m][e] = 0.f;
      struct Step { XPiece x[2 * kAdMT]; uint4 w[RTW]; };
      auto load = [&](Step& s, int c) {          // c: the lane's first column
        const bool in = c < a.d;
#pragma unroll
        for (int i = 0; i < 2 * kAdMT; ++i) {
          ad_zero(s.x[i]);
          if (in && i < 2 * mt) s.x[i] = *reinterpret_cast<const XPiece*>(x + (long long)token[i] * a.x_stride + c);
        }
#pragma unroll
        for (int h = 0; h < RTW; ++h) {
          ad_zero(s.w[h]);
          if (in && rt0 + h < rank_tiles) s.w[h] = __ldg(reinterpret_cast<const uint4*>(A + (long long)((rt0 + h) * 8 + g) * a.d + c));
        }
      };
      auto multiply = [&](const Step& s) {
#pragma unroll
        for (int m = 0; m < kAdMT; ++m) {
          if (m >= mt) break;
          const uint4 p = ad_operand(s.x[2 * m]), p8 = ad_operand(s.x[2 * m + 1]);
#pragma unroll
          for (int h = 0; h < RTW; ++h) ad_step(acc[h][m], p, p8, s.w[h], T());
        }
      };
      const int step = C * slices * 4 * P;
      Step s0, s1;
      int c = (cta * slices + slice) * 4 * P + q * P;
      const int end = a.d + q * P;               // the same number of turns for all lanes
      load(s0, c);
#pragma unroll 1
      for (; c < end; c += 2 * step) {
        load(s1, c + step);
        multiply(s0);
        if (c + step >= end) break;
        load(s0, c + 2 * step);
        multiply(s1);
      }
      if (owe_wait) cluster_wait();              // everybody has read the parts of the tile in front
      owe_wait = false;
#pragma unroll
      for (int h = 0; h < RTW; ++h) {
        if (rt0 + h >= rank_tiles) break;
#pragma unroll
        for (int m = 0; m < kAdMT; ++m) {
          if (m >= mt) break;
          float* p = part + (slice * kAdTile + m * 16 + g) * r + (rt0 + h) * 8 + 2 * q;
          *reinterpret_cast<float2*>(p) = make_float2(acc[h][m][0], acc[h][m][1]);
          *reinterpret_cast<float2*>(p + 8 * r) = make_float2(acc[h][m][2], acc[h][m][3]);
        }
      }
      __syncthreads();
    }
    // ---- second product: the first unit's y is requested before the sums are exchanged
    const T* B = static_cast<const T*>(a.B) + (long long)(work ? adapter : 0) * a.n * r;
    const int n_units = (a.n + 4 * P - 1) / (4 * P);
    uint4 yv[2 * kAdMT];
    auto load_y = [&](int unit) {
      const int c = (unit * 4 + q) * P;
#pragma unroll
      for (int i = 0; i < 2 * kAdMT; ++i) {
        ad_zero(yv[i]);
        if (y != nullptr && c < a.n && i < 2 * mt) yv[i] = *reinterpret_cast<const uint4*>(y + (long long)token[i] * a.y_stride + c);
      }
    };
    int unit = cta * kAdWarps + warp;
    load_y(unit);
    if (work) {
      const float sc = a.scale != nullptr ? a.scale[adapter] : 1.f;
      const int total = rows * r;
      auto finish = [&](int i, float4 s) {
        const int t = i / r, j = i - t * r;
        float f = sc;
        if (a.x_scales != nullptr) f *= a.x_scales[list[t]];
        ad_store_u(reinterpret_cast<T*>(us + t * u_pitch) + j, make_float4(s.x * f, s.y * f, s.z * f, s.w * f));
      };
      for (int i = tid * 4; i < total; i += kAdThreads * 4) {
        float4 s = *reinterpret_cast<const float4*>(part + i);
        for (int k = 1; k < slices; ++k) {
          const float4 v = *reinterpret_cast<const float4*>(part + k * kAdTile * r + i);
          s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
        if (C > 1) *reinterpret_cast<float4*>(part + i) = s;
        else finish(i, s);
      }
      if (C > 1) {
        cluster_arrive();
        cluster_wait();
        for (int i = tid * 4; i < total; i += kAdThreads * 4) {
          float4 s = ld_cluster4(part + i, 0);
#pragma unroll
          for (int k = 1; k < kAdMaxCtas; ++k) {
            if (k >= C) break;
            const float4 v = ld_cluster4(part + i, k);
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
          }
          finish(i, s);
        }
        cluster_arrive();
        owe_wait = true;
      }
      __syncthreads();                           // u is complete
    }
#pragma unroll 1
    for (; unit < n_units; unit += C * kAdWarps) {
      const int c0 = unit * 4 * P;
      float acc[kAdMT][NT][4];
#pragma unroll
      for (int m = 0; m < kAdMT; ++m)
#pragma unroll
        for (int h = 0; h < NT; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[m][h][e] = 0.f;
      if (work) {
#pragma unroll 2
        for (int k0 = 0; k0 < r; k0 += 4 * P) {
          const int k = k0 + q * P;
          uint4 w[NT];
#pragma unroll
          for (int h = 0; h < NT; ++h) {
            const int c = c0 + P * (g >> 1) + 2 * h + (g & 1);
            ad_zero(w[h]);
            if (k < r && c < a.n) w[h] = __ldg(reinterpret_cast<const uint4*>(B + (long long)c * r + k));
          }
#pragma unroll
          for (int m = 0; m < kAdMT; ++m) {
            if (m >= mt) break;
            uint4 p, p8;
            ad_zero(p);
            ad_zero(p8);
            if (k < r) {
              p = *reinterpret_cast<const uint4*>(us + (m * 16 + g) * u_pitch + k * kElem);
              p8 = *reinterpret_cast<const uint4*>(us + (m * 16 + g + 8) * u_pitch + k * kElem);
            }
#pragma unroll
            for (int h = 0; h < NT; ++h) ad_step(acc[m][h], p, p8, w[h], T());
          }
        }
      }
      uint4 res[2 * kAdMT];
#pragma unroll
      for (int i = 0; i < 2 * kAdMT; ++i) res[i] = work ? ad_finish(yv[i], acc[i >> 1], (i & 1) * 2, T()) : yv[i];
      load_y(unit + C * kAdWarps);
      const int c = c0 + q * P;
#pragma unroll
      for (int i = 0; i < 2 * kAdMT; ++i)
        if (c < a.n && g + 8 * i < rows) *reinterpret_cast<uint4*>(out + (long long)token[i] * a.out_stride + c) = res[i];
    }
  }
  if (owe_wait) cluster_wait();                  // nobody leaves while others read its part
}

// Most tiles that T tokens on `count` adapters can make.
inline int ad_max_tiles(int T, int count) { return T / kAdTile + (T < count + 1 ? T : count + 1); }
constexpr int kAdMaxClusters = 2048;

template <typename X, typename T>
inline cudaError_t adapters_launch(AdapterArgs a, int sm_count, cudaStream_t st, bool pdl) {
  int tiles = a.T;
  if (a.T > kAdDirect) {
    const cudaError_t e = launch_kernel(adapters_plan_kernel, dim3(1), dim3(kAdPlanThreads), 0, st, pdl, a, kAdTile);
    if (e != cudaSuccess) return e;
    tiles = ad_max_tiles(a.T, a.count);
  }
  // CTAs per cluster: as many as it takes to fill the chip
  a.ctas = 1;
  while (a.ctas < kAdMaxCtas && tiles * a.ctas < 3 * sm_count) a.ctas *= 2;
  const dim3 grid(a.ctas * (tiles < kAdMaxClusters ? tiles : kAdMaxClusters));
  auto go = [&](auto kernel) {
    return launch_cluster(kernel, a.ctas, grid, dim3(kAdThreads), ad_smem_bytes(a.r, (int)sizeof(T)), st, pdl, a);
  };
  return ad_rtw(a.r) == 1 ? go(adapters_kernel<X, T, 1>) : ad_rtw(a.r) == 2 ? go(adapters_kernel<X, T, 2>) : go(adapters_kernel<X, T, 4>);
}
// Raises the kernels' limit of dynamic shared memory where the default does not do.
inline cudaError_t adapters_set_limits() {
  cudaError_t e = cudaSuccess;
  auto raise = [&](auto kernel, int elem) {
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, ad_smem_bytes(kAdMaxRank, elem));
  };
  raise(adapters_kernel<float, float, 4>, 4);
  raise(adapters_kernel<bf16, bf16, 4>, 2);
  raise(adapters_kernel<__nv_fp8_e4m3, bf16, 4>, 2);
  return e;
}

}  // namespace swapmoe
