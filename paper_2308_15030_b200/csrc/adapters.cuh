// Low-rank adapters of many requests beside a projection that all of them share:
//   out[t] = y[t] + scale_a * B_a (A_a x[t]),  a = ids[t]  (no adapter: out[t] = y[t]),
// A_a [rank, d_in], B_a [d_out, rank], y the shared projection's row.
//
// Bound by bytes: x, y and out once, the adapters that are asked for once per tile of tokens; the products are rank * 2 operations
// per element of x and out, warp-level mma with tokens as mma rows.  One launch does both products: tokens of one adapter form
// tiles, a cluster of 1 to 8 CTAs takes a tile and splits the columns of x, then those of out; the CTAs' parts of A x are
// added through distributed shared memory, in a fixed order.  Two forms:
//  - up to 128 tokens (fp32 at high ranks: fewer; adapters_few_kernel, tiles of 16): all operands go from global memory straight to
//    the registers of the warp that multiplies them, 64 contiguous bytes of eight rows per load; clusters find their tiles themselves.
//  - more (adapters_tile_kernel, tiles of 64, a plan kernel in front that groups the tokens by adapter): x, A, y and B run through
//    a ring in shared memory, so A and B are fetched once per 64 tokens and the loads run ahead of the products.
// In the second product the columns are dealt out to the mma's column tiles so that a lane's results are 16 contiguous bytes of a
// row: out is written from registers.
#pragma once
#include <cuda_fp8.h>
#include <math_constants.h>

#include "common.cuh"
#include "launch.cuh"

namespace swapmoe {

constexpr int kAdMaxRank = 128, kAdMaxCount = 4096, kAdMaxWidth = 1 << 16;
constexpr int kAdThreads = 256, kAdWarps = kAdThreads / 32;
constexpr int kAdMaxCtas = 8;              // most CTAs per cluster
constexpr int kAdTile = 16;                // tokens of a tile: one mma row tile
constexpr int kAdDirect = 128;             // up to this many tokens every cluster finds its tile itself (see ad_direct_tokens)

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
constexpr int kAdPlanIds = 8;              // tokens whose ids a thread keeps

// Groups the tokens by adapter and cuts the groups into tiles of at most `tile_rows`.  One CTA: counts per adapter, their
// exclusive scans, then every token takes a place in its group.  (Which place is left to the order of atomics; a row's result does
// not depend on it.)  A chain of latencies: ids are read once, in one go, runs of one adapter cost one atomic per warp.
__global__ void __launch_bounds__(kAdPlanThreads) adapters_plan_kernel(const AdapterArgs a, int tile_rows) {
  __shared__ int32_t s_cursor[kAdMaxCount + 1];
  __shared__ int32_t s_warp[2][32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x;
  const int groups = a.count + 1;                           // the last one: tokens without an adapter
  for (int g = tid; g < groups; g += threads) s_cursor[g] = 0;
  pdl_wait();
  pdl_trigger();
  auto group_of = [&](int t) {
    if (t >= a.T) return -1;
    const int id = a.ids[t];
    return id < 0 || id >= a.count ? a.count : id;
  };
  int kept[kAdPlanIds];
#pragma unroll
  for (int i = 0; i < kAdPlanIds; ++i) kept[i] = group_of(tid + i * threads);
  __syncthreads();
  auto count = [&](int g) {
    const uint32_t same = __match_any_sync(0xffffffffu, g);
    if (g >= 0 && __ffs(same) - 1 == lane) atomicAdd(&s_cursor[g], __popc(same));
  };
#pragma unroll
  for (int i = 0; i < kAdPlanIds; ++i)
    if (i * threads < a.T) count(kept[i]);
  for (int t0 = kAdPlanIds * threads; t0 < a.T; t0 += threads) count(group_of(t0 + tid));
  __syncthreads();
  // thread i owns groups i * per ... : sums, scan over the threads, then first rows and tiles of its groups
  const int per = (groups + threads - 1) / threads, g0 = tid * per;
  int rows = 0, tiles = 0;
  for (int g = g0; g < min(groups, g0 + per); ++g) {
    rows += s_cursor[g];
    tiles += (s_cursor[g] + tile_rows - 1) / tile_rows;
  }
  auto scan = [&](int& u, int& v) {                         // inclusive, over the lanes
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, u, o), y = __shfl_up_sync(0xffffffffu, v, o);
      if (lane >= o) { u += x; v += y; }
    }
  };
  int row_incl = rows, tile_incl = tiles;
  scan(row_incl, tile_incl);
  if (lane == 31) { s_warp[0][warp] = row_incl; s_warp[1][warp] = tile_incl; }
  __syncthreads();
  int row_base = lane < threads / 32 ? s_warp[0][lane] : 0, tile_base = lane < threads / 32 ? s_warp[1][lane] : 0;
  scan(row_base, tile_base);
  const int row_front = __shfl_sync(0xffffffffu, row_base, max(warp - 1, 0)), tile_front = __shfl_sync(0xffffffffu, tile_base, max(warp - 1, 0));
  const int all_tiles = __shfl_sync(0xffffffffu, tile_base, 31);
  int row = row_incl - rows + (warp > 0 ? row_front : 0), tile = tile_incl - tiles + (warp > 0 ? tile_front : 0);
  if (tid == 0) *a.n_tiles = all_tiles;
  for (int g = g0; g < min(groups, g0 + per); ++g) {
    const int n = s_cursor[g], cut = (n + tile_rows - 1) / tile_rows;
    const int each = cut > 0 ? (n + cut - 1) / cut : 0;     // tiles of equal height
    for (int i = 0; i < cut; ++i)
      a.tiles[tile + i] = {g < a.count ? g : -1, row + i * each, min(each, n - i * each), 0};
    s_cursor[g] = row;
    row += n;
    tile += cut;
  }
  __syncthreads();
  auto place = [&](int g, int t) {
    const uint32_t same = __match_any_sync(0xffffffffu, g);
    const int leader = __ffs(same) - 1;
    int base = 0;
    if (g >= 0 && leader == lane) base = atomicAdd(&s_cursor[g], __popc(same));
    base = __shfl_sync(0xffffffffu, base, leader);
    if (g >= 0) a.perm[base + __popc(same & ((1u << lane) - 1))] = t;
  };
#pragma unroll
  for (int i = 0; i < kAdPlanIds; ++i)
    if (i * threads < a.T) place(kept[i], tid + i * threads);
  for (int t0 = kAdPlanIds * threads; t0 < a.T; t0 += threads) place(group_of(t0 + tid), t0 + tid);
}

// ----------------------------------------------------------------------------- fragments and products
__device__ __forceinline__ void mma_bf16_16x8x16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                                 uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Two fp32 values as three pairs of bf16 pieces, each rounded to nearest from what the ones in front left: 24 bits in all.
__device__ __forceinline__ void ad_split(uint32_t x, uint32_t y, uint32_t& hi, uint32_t& mid, uint32_t& lo) {
  float a = __uint_as_float(x), b = __uint_as_float(y);
  hi = pack_bf16x2(a, b);
  a -= __uint_as_float(hi << 16);
  b -= __uint_as_float(hi & 0xffff0000u);
  mid = pack_bf16x2(a, b);
  lo = pack_bf16x2(a - __uint_as_float(mid << 16), b - __uint_as_float(mid & 0xffff0000u));
}
// The left operand of a step of 64 bytes: rows g and g + 8 (pieces p, p8); fp32 ones in their bf16 pieces, once for all column tiles.
template <typename T> struct AdLeft;
template <> struct AdLeft<bf16> {
  uint4 p, p8;
  __device__ __forceinline__ AdLeft(const uint4& a, const uint4& b) : p(a), p8(b) {}
};
template <> struct AdLeft<float> {
  uint32_t v[3][4];                          // pieces of a mma's operand
  __device__ __forceinline__ AdLeft(const uint4& p, const uint4& p8) {
    ad_split(p.x, p.y, v[0][0], v[1][0], v[2][0]);
    ad_split(p8.x, p8.y, v[0][1], v[1][1], v[2][1]);
    ad_split(p.z, p.w, v[0][2], v[1][2], v[2][2]);
    ad_split(p8.z, p8.w, v[0][3], v[1][3], v[2][3]);
  }
};
// c += one step: row g of the right operand (w).
__device__ __forceinline__ void ad_step(float (&c)[4], const AdLeft<bf16>& a, const uint4& w) {
  mma_bf16_16x8x16(c, a.p.x, a.p8.x, a.p.y, a.p8.y, w.x, w.y);
  mma_bf16_16x8x16(c, a.p.z, a.p8.z, a.p.w, a.p8.w, w.z, w.w);
}
__device__ __forceinline__ void ad_step(float (&c)[4], const AdLeft<float>& a, const uint4& w) {
  // fp32 products as six of bf16 pieces, the small ones first (the others are below 2^-25 together).  Three products of TF32 pieces
  // are as many mma, two steps of 8 in depth each, and slower: 1531 tokens of 768 -> 2240 18.8 us with them and 17.8 so, 400 of 2048 at
  // rank 128 75.3 and 72.1.  The tensor core's sums truncate, so a step's six are added to c by an ordinary addition: over d_in
  // 4096 in one accumulator they drift by 3e-5 of the result.
  uint32_t b[3][2];
  ad_split(w.x, w.y, b[0][0], b[1][0], b[2][0]);
  ad_split(w.z, w.w, b[0][1], b[1][1], b[2][1]);
  float t[4] = {0.f, 0.f, 0.f, 0.f};
  auto product = [&](int i, int j) { mma_bf16_16x8x16(t, a.v[i][0], a.v[i][1], a.v[i][2], a.v[i][3], b[j][0], b[j][1]); };
  product(2, 0);
  product(0, 2);
  product(1, 1);
  product(1, 0);
  product(0, 1);
  product(0, 0);
#pragma unroll
  for (int e = 0; e < 4; ++e) c[e] += t[e];
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
// What lies between the products, u = scale * A x, is kept in fp32 (fp32 banks) or in two bf16 pieces, to 2^-16: rounded to one, it
// alone brought as much error as the rounding of the results.  The first piece is cut off, not rounded, and the second one is never 0
// where the first is not (2^-24 of it in place of a 0): pieces of one sign, whose products with an infinity of B are
// infinities of one sign too.  An infinite u has two infinite pieces.  `lo`: bytes from the first piece to the second.
__device__ __forceinline__ float ad_rest(float v, float first) {
  const float rest = v - first;
  return fabsf(rest) > 0.f ? rest : first * 0x1p-24f;
}
__device__ __forceinline__ void ad_pieces(float a, float b, uint32_t& hi, uint32_t& lo) {
  const uint32_t x = __float_as_uint(a) & 0xffff0000u, y = __float_as_uint(b) & 0xffff0000u;
  hi = x >> 16 | y;
  lo = pack_bf16x2(ad_rest(a, __uint_as_float(x)), ad_rest(b, __uint_as_float(y)));
}
__device__ __forceinline__ void ad_store_u(float* p, float4 v, int) { *reinterpret_cast<float4*>(p) = v; }
__device__ __forceinline__ void ad_store_u(bf16* p, float4 v, int lo) {
  uint2 h, l;
  ad_pieces(v.x, v.y, h.x, l.x);
  ad_pieces(v.z, v.w, h.y, l.y);
  *reinterpret_cast<uint2*>(p) = h;
  *reinterpret_cast<uint2*>(reinterpret_cast<unsigned char*>(p) + lo) = l;
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
// fp32: sums of bf16 pieces that are not finite say little: an infinity's second piece is inf - inf, and a finite value beyond bf16's
// largest has an infinite one.  What such a sum belongs to is computed again by plain multiply-adds, out of line (never taken
// with finite results).
template <int N>
__device__ __forceinline__ bool ad_finite(const float (&c)[N][4], int e) {
  float m = 0.f;
#pragma unroll
  for (int h = 0; h < N; ++h) m += fabsf(c[h][e]) + fabsf(c[h][e + 1]);
  return m < CUDART_INF_F;
}
// Two neighbouring ranks of A x: x a row, w the first rank's row of A.
static __device__ __noinline__ float2 ad_again_u(const float* x, const float* w, int d) {
  float2 s = make_float2(0.f, 0.f);
#pragma unroll 4
  for (int c = 0; c < d; ++c) {
    s.x = fmaf(x[c], w[c], s.x);
    s.y = fmaf(x[c], w[d + c], s.y);
  }
  return s;
}
// 16 bytes of out: u a row of the low-rank side, w the first column's row of B.
static __device__ __noinline__ uint4 ad_again_out(const float* u, const float* w, int r, uint4 y) {
  float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
  for (int j = 0; j < r; ++j)
#pragma unroll
    for (int c = 0; c < 4; ++c) s[c] = fmaf(u[j], w[c * r + j], s[c]);
  return make_uint4(__float_as_uint(__uint_as_float(y.x) + s[0]), __float_as_uint(__uint_as_float(y.y) + s[1]),
                    __float_as_uint(__uint_as_float(y.z) + s[2]), __float_as_uint(__uint_as_float(y.w) + s[3]));
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
// bf16 rows of u are two: the first pieces and the second ones.  Up to rank 16 both are halves of one row of 64 bytes, a step of the
// second product, whose other operand then is B twice: no more products than for one piece.
__host__ __device__ constexpr bool ad_u_halves(int r, int elem) { return elem == 2 && r <= 16; }
__host__ __device__ constexpr int ad_u_bytes(int r, int elem) { return kAdTile * ad_u_pitch(r, elem) * (elem == 2 && !ad_u_halves(r, elem) ? 2 : 1); }
__host__ __device__ constexpr int ad_smem_bytes(int r, int elem) { return ad_part_bytes(r) + ad_u_bytes(r, elem) + kAdTile * 4 + 16; }

// The tile of cluster i without a plan: it has one if token i is the first, or the 17th, ... of its adapter; then its tokens
// are the next 16 of that adapter from i on.  By one warp: lane l holds tokens l, l + 32, ...
__device__ __forceinline__ int ad_direct_tile(const AdapterArgs& a, int i, int32_t* list, int* adapter) {
  constexpr int kWords = kAdDirect / 32;
  const int lane = threadIdx.x & 31;
  int id[kWords], mine = 0;
#pragma unroll
  for (int w = 0; w < kWords; ++w) {
    const int t = lane + 32 * w;
    id[w] = t < a.T ? a.ids[t] : -2;
    if (t < a.T && (id[w] < 0 || id[w] >= a.count)) id[w] = -1;
  }
#pragma unroll
  for (int w = 0; w < kWords; ++w) {
    const int v = __shfl_sync(0xffffffffu, id[w], i & 31);
    if (w == i >> 5) mine = v;
  }
  *adapter = mine;
  int before = 0, at = 0;                        // tokens of the adapter in front of i; from i on, in front of word w
  uint32_t rest[kWords];
#pragma unroll
  for (int w = 0; w < kWords; ++w) {
    const uint32_t same = __ballot_sync(0xffffffffu, id[w] == mine);
    const uint32_t front = w < i >> 5 ? 0xffffffffu : w == i >> 5 ? (1u << (i & 31)) - 1 : 0u;
    before += __popc(same & front);
    rest[w] = same & ~front;
  }
  if (before % kAdTile != 0) return 0;
#pragma unroll
  for (int w = 0; w < kWords; ++w) {
    const int place = at + __popc(rest[w] & ((1u << lane) - 1));
    if ((rest[w] >> lane) & 1 && place < kAdTile) list[place] = lane + 32 * w;
    at += __popc(rest[w]);
  }
  return min(kAdTile, at);
}

// First product: the contraction is dealt out to the warps in steps of 64 bytes (two or four warps share x from rank 40 on), and their
// sums are added in shared memory.  Within a step a lane's 16-byte piece holds its operands of two (bf16) mma: the contraction
// index is permuted the same way on both sides.  Second product: a warp owns 64 bytes of columns of all the tile's rows.
// X: rows of x (T or e4m3), T: everything else, RTW: rank tiles per warp.
template <typename X, typename T, int RTW>
__global__ void __launch_bounds__(kAdThreads, 2) adapters_few_kernel(const AdapterArgs a) {
  constexpr int kElem = (int)sizeof(T);
  constexpr bool kHalves = kElem == 2 && RTW <= 2;      // ad_u_halves of the ranks that come here
  constexpr int P = 16 / kElem;                  // values of a lane's piece; a step or unit is 4 P values
  constexpr int NT = P / 2;                      // column tiles of a unit of out
  typedef typename AdPiece<X>::type XPiece;
  extern __shared__ __align__(128) unsigned char smem[];
  const int r = a.r, rank_tiles = r / 8, u_pitch = ad_u_pitch(r, kElem);
  const int rank_warps = ad_rank_warps(r, RTW), slices = kAdWarps / rank_warps;
  float* part = reinterpret_cast<float*>(smem);                                 // [slices][tile][r]
  unsigned char* us = smem + ad_part_bytes(r);                                  // [tile] rows of u in T, and their second pieces
  int32_t* list = reinterpret_cast<int32_t*>(us + ad_u_bytes(r, kElem));        // [tile] tokens
  volatile int* ctl = list + kAdTile;                                           // rows, adapter
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), g = lane >> 2, q = lane & 3;
  const int C = a.ctas, cta = blockIdx.x % C;
  pdl_wait();
  pdl_trigger();
  const X* x = static_cast<const X*>(a.x);
  const T* y = static_cast<const T*>(a.y);
  T* out = static_cast<T*>(a.out);
  if (warp == 0) {
    int adapter;
    const int rows = ad_direct_tile(a, blockIdx.x / C, list, &adapter);
    if (lane == 0) { ctl[0] = rows; ctl[1] = adapter; }
  }
  __syncthreads();
  const int rows = ctl[0], adapter = ctl[1];
  if (rows == 0) return;                         // the same for the whole cluster
  const bool work = adapter >= 0;
  // the lane's rows: g, g + 8; a row that the tile does not have repeats its first one and is not stored
  int token[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) token[i] = list[g + 8 * i < rows ? g + 8 * i : 0];
  if (work) {
    // ---- first product, kDepth steps on their way.  Rank tiles that the warp does not have repeat the last one and are not stored:
    // no load of a full step has a condition of its own.
    constexpr int kDepth = RTW <= 2 ? 4 : 2;
    const char* A = reinterpret_cast<const char*>(static_cast<const T*>(a.A) + (long long)adapter * r * a.d);
    const int slice = warp / rank_warps, rt0 = (warp % rank_warps) * RTW;
    const char* xp[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) xp[i] = reinterpret_cast<const char*>(x + (long long)token[i] * a.x_stride);
    uint32_t ap[RTW];
#pragma unroll
    for (int h = 0; h < RTW; ++h) ap[h] = (uint32_t)((min(rt0 + h, rank_tiles - 1) * 8 + g) * a.d) * kElem;
    float acc[RTW][4];
#pragma unroll
    for (int h = 0; h < RTW; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[h][e] = 0.f;
    struct Step { XPiece x[2]; uint4 w[RTW]; };
    auto load = [&](Step& s, uint32_t c) {     // c: the lane's first column
#pragma unroll
      for (int i = 0; i < 2; ++i) s.x[i] = *reinterpret_cast<const XPiece*>(xp[i] + c * (uint32_t)sizeof(X));
#pragma unroll
      for (int h = 0; h < RTW; ++h) s.w[h] = __ldg(reinterpret_cast<const uint4*>(A + (ap[h] + c * kElem)));
    };
    auto multiply = [&](const Step& s) {
      const AdLeft<T> left(ad_operand(s.x[0]), ad_operand(s.x[1]));
#pragma unroll
      for (int h = 0; h < RTW; ++h) ad_step(acc[h], left, s.w[h]);
    };
    const int step = C * slices * 4 * P, first = (cta * slices + slice) * 4 * P;
    const int n_full = first + 4 * P <= a.d ? (a.d - 4 * P - first) / step + 1 : 0;     // steps all of whose pieces exist
    Step s[kDepth];
#pragma unroll
    for (int i = 0; i < kDepth; ++i)
      if (i < n_full) load(s[i], first + i * step + q * P);
#pragma unroll 1
    for (int n = 0; n < n_full; n += kDepth) {
#pragma unroll
      for (int i = 0; i < kDepth; ++i) {
        if (n + i >= n_full) break;
        multiply(s[i]);
        if (n + i + kDepth < n_full) load(s[i], first + (n + i + kDepth) * step + q * P);
      }
    }
    const int c0 = first + n_full * step;
    if (c0 < a.d) {                            // the last step of the rows
#pragma unroll
      for (int i = 0; i < 2; ++i) ad_zero(s[0].x[i]);
#pragma unroll
      for (int h = 0; h < RTW; ++h) ad_zero(s[0].w[h]);
      if (c0 + q * P < a.d) load(s[0], c0 + q * P);
      multiply(s[0]);
    }
#pragma unroll
    for (int h = 0; h < RTW; ++h) {
      if (rt0 + h >= rank_tiles) break;
      float* p = part + (slice * kAdTile + g) * r + (rt0 + h) * 8 + 2 * q;
      *reinterpret_cast<float2*>(p) = make_float2(acc[h][0], acc[h][1]);
      *reinterpret_cast<float2*>(p + 8 * r) = make_float2(acc[h][2], acc[h][3]);
    }
    __syncthreads();
  }
  // ---- second product, two units at a time: y and the first step of B are requested before the sums are exchanged, and those of
  // the next two units before this pair is stored
  constexpr int kUnits = 2;
  const char* B = reinterpret_cast<const char*>(static_cast<const T*>(a.B) + (long long)(work ? adapter : 0) * a.n * r);
  const int n_units = (a.n + 4 * P - 1) / (4 * P), stride = C * kAdWarps;
  const char* yp[2];
  char* op[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    yp[i] = reinterpret_cast<const char*>(y + (long long)token[i] * a.y_stride) + q * 16;
    op[i] = reinterpret_cast<char*>(out + (long long)token[i] * a.out_stride) + q * 16;
  }
  uint4 yv[kUnits][2], wb[kUnits][NT];
#pragma unroll
  for (int v = 0; v < kUnits; ++v)
#pragma unroll
    for (int i = 0; i < 2; ++i) ad_zero(yv[v][i]);
  auto load_y = [&](uint4 (&d)[2], int unit) {
    if (y != nullptr && (unit * 4 + q) * P < a.n) {
#pragma unroll
      for (int i = 0; i < 2; ++i) d[i] = *reinterpret_cast<const uint4*>(yp[i] + (uint32_t)unit * 64u);
    }
  };
  // lane's row of B in column tile h of a unit: P (g / 2) + 2 h + g % 2
  const int b_col = P * (g >> 1) + (g & 1);
  const uint32_t b_row = (uint32_t)(r * kElem);
  const int qr = kHalves ? q & 1 : q;            // the lane's piece of the ranks
  auto load_b = [&](uint4 (&w)[NT], int unit, int k0) {
    const int c = unit * 4 * P + b_col;
#pragma unroll
    for (int h = 0; h < NT; ++h) {
      ad_zero(w[h]);
      if (k0 + qr * P < r && c + 2 * h < a.n)
        w[h] = __ldg(reinterpret_cast<const uint4*>(B + ((uint32_t)(c + 2 * h) * b_row + k0 * kElem + qr * 16)));
    }
  };
  int unit = cta * kAdWarps + warp;
#pragma unroll
  for (int v = 0; v < kUnits; ++v) {
    load_y(yv[v], unit + v * stride);
    if (work) load_b(wb[v], unit + v * stride, 0);
  }
  if (work) {
    const float sc = a.scale != nullptr ? a.scale[adapter] : 1.f;
    const int total = rows * r;
    auto finish = [&](int i, float4 s) {
      const int t = i / r, j = i - t * r;
      if constexpr (kElem == 4)
        if (!(fabsf(s.x) + fabsf(s.y) + fabsf(s.z) + fabsf(s.w) < CUDART_INF_F)) {
          const X* row = x + (long long)list[t] * a.x_stride;
          const T* w = static_cast<const T*>(a.A) + ((long long)adapter * r + j) * a.d;
          const float2 lo = ad_again_u(row, w, a.d), hi = ad_again_u(row, w + 2ll * a.d, a.d);
          s = make_float4(lo.x, lo.y, hi.x, hi.y);
        }
      float f = sc;
      if (a.x_scales != nullptr) f *= a.x_scales[list[t]];
      ad_store_u(reinterpret_cast<T*>(us + t * u_pitch) + j, make_float4(s.x * f, s.y * f, s.z * f, s.w * f), kHalves ? 32 : kAdTile * u_pitch);
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
    }
    __syncthreads();                           // u is complete
  }
  auto operand_u = [&](uint4& p, int row, int k0) {
    ad_zero(p);
    if (k0 + qr * P < r) p = *reinterpret_cast<const uint4*>(us + row * u_pitch + k0 * kElem + q * 16);
  };
#pragma unroll 1
  for (; unit < n_units; unit += kUnits * stride) {
    uint4 res[kUnits][2];
#pragma unroll
    for (int v = 0; v < kUnits; ++v) {
      if (work) {
        float acc[NT][4];
#pragma unroll
        for (int h = 0; h < NT; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[h][e] = 0.f;
        for (int k0 = 0; k0 < r; k0 += 4 * P) {
          uint4 p, p8;
          operand_u(p, g, k0);
          operand_u(p8, g + 8, k0);
          const AdLeft<T> left(p, p8);
          if (k0 > 0) load_b(wb[v], unit + v * stride, k0);
          if constexpr (kElem == 2 && !kHalves) {        // the second pieces first
            operand_u(p, g + kAdTile, k0);
            operand_u(p8, g + 8 + kAdTile, k0);
            const AdLeft<T> rest(p, p8);
#pragma unroll
            for (int h = 0; h < NT; ++h) ad_step(acc[h], rest, wb[v][h]);
          }
#pragma unroll
          for (int h = 0; h < NT; ++h) ad_step(acc[h], left, wb[v][h]);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          res[v][i] = ad_finish(yv[v][i], acc, 2 * i, T());
          if constexpr (kElem == 4) {
            const int c = ((unit + v * stride) * 4 + q) * P, row = g + 8 * i;
            if (!ad_finite(acc, 2 * i) && c < a.n && row < rows)
              res[v][i] = ad_again_out(reinterpret_cast<const T*>(us + row * u_pitch), reinterpret_cast<const T*>(B) + (long long)c * r, r,
                                       yv[v][i]);
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) res[v][i] = yv[v][i];
      }
    }
#pragma unroll
    for (int v = 0; v < kUnits; ++v) {
      const int next = unit + (kUnits + v) * stride;
      load_y(yv[v], next);
      if (work && next < n_units) load_b(wb[v], next, 0);
    }
#pragma unroll
    for (int v = 0; v < kUnits; ++v) {
      const int at = unit + v * stride;
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if ((at * 4 + q) * P < a.n && g + 8 * i < rows) *reinterpret_cast<uint4*>(op[i] + (uint32_t)at * 64u) = res[v][i];
    }
  }
  if (C > 1 && work) cluster_wait();              // nobody leaves while others read its part
}

// ----------------------------------------------------------------------------- many tokens
constexpr int kAdTM = 64;                  // tokens of a tile
constexpr int kAdChunk = 256;              // bytes of a row of x (bf16, fp32), A, y and out that a CTA takes at a time
constexpr int kAdMaxStages = 6;
// A stage holds the tile's rows of a chunk of x and the same columns of A, or the rows of a chunk of y and the rows of B behind its
// columns: the same number of bytes.  The 16-byte pieces of a row trade places by an exclusive or with ad_swap of the row, so that
// the lanes that are served together meet different banks: eight rows' pieces of one index (ldmatrix), and two rows of four pieces
// (operands that are converted on the way).
__host__ __device__ constexpr int ad_swap(int row) { return (row & 1) << 2 | (row >> 1 & 3); }
// The same for rows of B, of `pieces` pieces: eight rows of one column tile lie at 8 a + b, a < 4, b < 2 (see from_b).
__host__ __device__ constexpr int ad_swap_b(int row, int pieces) {
  return pieces >= 8 ? (row & 1) << 2 | (row >> 3 & 3) : row >> 3 & (pieces - 1);
}
__host__ __device__ constexpr int ad_rank_up(int r) { return r <= 16 ? 16 : r <= 32 ? 32 : r <= 64 ? 64 : 128; }
__host__ __device__ constexpr int ad_stage_bytes(int r) { return kAdTM * kAdChunk + kAdChunk * r; }
// A row of u: bf16 ones are first pieces, then second pieces, which trade places as above, by ad_swap_u of the row.
__host__ __device__ constexpr int ad_tile_u_pitch(int r, int elem) { return elem == 2 ? r * 4 : ad_u_pitch(r, elem); }
__host__ __device__ constexpr int ad_swap_u(int row, int pitch) { return pitch == 64 ? row >> 1 & 3 : row & 7; }
// What lies behind the stages: rows of u, for small ranks the CTA's part of u (else it takes the stage that was multiplied last,
// which is then not free before the other CTAs have read it), the list of tokens.
__host__ __device__ constexpr bool ad_own_part(int r) { return r <= 32; }
__host__ __device__ constexpr int ad_tile_rest(int r, int elem) {
  return kAdTM * ad_tile_u_pitch(r, elem) + (ad_own_part(r) ? kAdTM * r * 4 : 0) + kAdTM * 4 + 512;
}
// Stages: as many as fit with two CTAs per SM (228 KB, of which each CTA costs 1), or, where that leaves fewer than three, with one.
constexpr int kAdTwoBytes = 113 * 1024, kAdOneBytes = 227 * 1024;
inline int ad_stages(int r, int elem) {
  const int two = (kAdTwoBytes - ad_tile_rest(r, elem)) / ad_stage_bytes(r);
  const int n = two >= 3 ? two : (kAdOneBytes - ad_tile_rest(r, elem)) / ad_stage_bytes(r);
  return n < kAdMaxStages ? n : kAdMaxStages;
}
template <int kBytes>
__device__ __forceinline__ void ad_copy(uint32_t d, const void* src) {               // to shared memory
  if constexpr (kBytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(d), "l"(src) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(d), "l"(src) : "memory");
}
template <int kBytes>
__device__ __forceinline__ void ad_clear(uint32_t d) {
  if constexpr (kBytes == 16) asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(d), "r"(0) : "memory");
  else asm volatile("st.shared.v2.b32 [%0], {%1, %1};" ::"r"(d), "r"(0) : "memory");
}
__device__ __forceinline__ void ad_copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void ad_copy_wait(int pending) {            // at most `pending` groups are still on their way
  switch (pending) {
    case 0: asm volatile("cp.async.wait_group 0;" ::: "memory"); break;
    case 1: asm volatile("cp.async.wait_group 1;" ::: "memory"); break;
    case 2: asm volatile("cp.async.wait_group 2;" ::: "memory"); break;
    case 3: asm volatile("cp.async.wait_group 3;" ::: "memory"); break;
    default: asm volatile("cp.async.wait_group 4;" ::: "memory"); break;
  }
}
__device__ __forceinline__ void ad_store_u2(float* p, float a, float b, int) { *reinterpret_cast<float2*>(p) = make_float2(a, b); }
__device__ __forceinline__ void ad_store_u2(bf16* p, float a, float b, int lo) {
  uint32_t h, l;
  ad_pieces(a, b, h, l);
  *reinterpret_cast<uint32_t*>(p) = h;
  *reinterpret_cast<uint32_t*>(reinterpret_cast<unsigned char*>(p) + lo) = l;
}

__device__ __forceinline__ uint4 ad_lds(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
  return v;
}
__device__ __forceinline__ uint4 ad_lds8(uint32_t at) {             // eight e4m3 values as bf16
  uint2 v;
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at));
  return ad_operand(v);
}

__device__ __forceinline__ void ad_ldmatrix(uint32_t (&v)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(at));
}
__device__ __forceinline__ void ad_ldmatrix(uint32_t (&v)[2], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x2.shared.b16 {%0, %1}, [%2];" : "=r"(v[0]), "=r"(v[1]) : "r"(at));
}

// Tile `which` of the plan that adapters_plan_kernel would make, found by a CTA for itself, for up to kAdHere tokens: rows and adapter
// in ctl (no rows: there is no such tile), tokens in list.  Tokens of a group are taken in their order, so that all CTAs agree.
// scratch: count + 1 + 96 words.
constexpr int kAdHere = kAdPlanIds * kAdThreads;
__device__ __forceinline__ void ad_tile_here(const AdapterArgs& a, int which, int32_t* scratch, int32_t* list, int32_t* ctl) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, groups = a.count + 1;
  int32_t *cursor = scratch, *front = scratch + groups, *per_warp = front + 64;
  int kept[kAdPlanIds];
#pragma unroll
  for (int i = 0; i < kAdPlanIds; ++i) {
    const int t = tid + i * kAdThreads;
    kept[i] = -1;
    if (t < a.T) {
      const int id = a.ids[t];
      kept[i] = id < 0 || id >= a.count ? a.count : id;
    }
  }
  for (int g = tid; g < groups; g += kAdThreads) cursor[g] = 0;
  if (tid == 0) ctl[0] = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kAdPlanIds; ++i) {
    if (i * kAdThreads >= a.T) break;
    const uint32_t same = __match_any_sync(0xffffffffu, kept[i]);
    if (kept[i] >= 0 && __ffs(same) - 1 == lane) atomicAdd(&cursor[kept[i]], __popc(same));
  }
  __syncthreads();
  const int per = (groups + kAdThreads - 1) / kAdThreads, g0 = tid * per;
  int tiles = 0;
  for (int g = g0; g < min(groups, g0 + per); ++g) tiles += (cursor[g] + kAdTM - 1) / kAdTM;
  int incl = tiles;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += v;
  }
  if (lane == 31) per_warp[warp] = incl;
  __syncthreads();
  int tile = incl - tiles;
  for (int w = 0; w < warp; ++w) tile += per_warp[w];
  for (int g = g0; g < min(groups, g0 + per); ++g) {
    const int n = cursor[g], cut = (n + kAdTM - 1) / kAdTM;
    if (which >= tile && which < tile + cut) {
      const int each = (n + cut - 1) / cut;
      ctl[2] = (which - tile) * each;                        // first place in the group
      ctl[1] = g;
      ctl[0] = min(each, n - ctl[2]);
    }
    tile += cut;
  }
  __syncthreads();
  const int rows = ctl[0], group = ctl[1], first = ctl[2];
  if (rows == 0) return;
#pragma unroll
  for (int i = 0; i < kAdPlanIds; ++i) {
    const uint32_t m = __ballot_sync(0xffffffffu, kept[i] == group);
    if (lane == 0) front[i * kAdWarps + warp] = __popc(m);
  }
  __syncthreads();
  if (warp == 0) {                                           // exclusive scan of the 64 counts, in the tokens' order
    const int u = front[2 * lane], v = front[2 * lane + 1];
    int sum = u + v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int w = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += w;
    }
    front[2 * lane] = sum - u - v;
    front[2 * lane + 1] = sum - v;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kAdPlanIds; ++i) {
    const uint32_t m = __ballot_sync(0xffffffffu, kept[i] == group);
    const int at = front[i * kAdWarps + warp] + __popc(m & ((1u << lane) - 1)) - first;
    if (kept[i] == group && at >= 0 && at < rows) list[at] = tid + i * kAdThreads;
  }
  __syncthreads();
}

// Tiles of up to 64 tokens from the plan; a cluster takes a tile and deals its chunks of x, then of y, out to its CTAs.  The
// chunks of both products run through one ring of stages, so the first of y and B are on their way while x is still multiplied; one
// barrier per chunk.  Warp w multiplies 16 tokens (w % 4) by half the ranks, then by half the chunk's columns of out.
// RP: the rank rounded up (16, 32, 64, 128), so that all places in shared memory are constants (places that hang on the rank
// itself: 8192 x 4096 at rank 64 80 us, constants 67).  bf16 operands come by ldmatrix, whose four registers are an operand as it is;
// from two rows' 16-byte pieces it has to be put together, which took more instructions than the products.
template <typename X, typename T, int RP>
__global__ void __launch_bounds__(kAdThreads, 2) adapters_tile_kernel(const __grid_constant__ AdapterArgs a, int stages, int here) {
  constexpr int kElem = (int)sizeof(T), P = 16 / kElem, NT = P / 2;
  constexpr int kCols = kAdChunk / kElem;                    // columns of a chunk
  constexpr int kXPiece = sizeof(X) == 1 ? 8 : 16;           // bytes of a lane's piece of x: P values
  constexpr int kXRow = 16 * kXPiece;                        // bytes of a row of a chunk of x
  constexpr int NTH = RP / 16;                               // rank tiles per warp
  constexpr int kBRow = RP * kElem, kBPieces = kBRow / 16;   // a row of B in a stage
  constexpr int kUPitch = ad_tile_u_pitch(RP, kElem);
  constexpr uint32_t kStage = (uint32_t)ad_stage_bytes(RP), kW = kAdTM * kAdChunk;
  constexpr bool kMatrixX = sizeof(X) == 2, kMatrixB = kElem == 2;     // operands of the two products by ldmatrix
  extern __shared__ __align__(128) unsigned char smem_raw[];
  // (a step's piece is found by an exclusive or with its index: stages start at multiples of the longest row)
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 511) & ~static_cast<uintptr_t>(511));
  const int r = a.r;
  unsigned char* us = smem + stages * kStage;
  float* own_part = reinterpret_cast<float*>(us + kAdTM * kUPitch);
  int32_t* list = reinterpret_cast<int32_t*>(us + kAdTM * kUPitch + (ad_own_part(RP) ? kAdTM * RP * 4 : 0));
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), g = lane >> 2, q = lane & 3;
  const int mw = warp & 3, nh = warp >> 2;
  const int C = a.ctas, cta = blockIdx.x % C, cluster = blockIdx.x / C, n_clusters = gridDim.x / C;
  const int x_chunks = (a.d + kCols - 1) / kCols, y_chunks = (a.n + kCols - 1) / kCols;
  const int x_iters = (x_chunks + C - 1) / C, y_iters = (y_chunks + C - 1) / C;     // the same for all CTAs of a cluster
  const int per_row = r / P;                                 // pieces of a row of B
  const uint32_t stage0 = (uint32_t)__cvta_generic_to_shared(smem), us0 = stage0 + stages * kStage;
  // What a thread copies: piece tid % 16 of rows tid / 16 + 16 k of x, y and A; of B pieces tid + 256 k.
  const int crow = tid >> 4, cpiece = tid & 15;
  const uint32_t to_row = crow * 256 + ((cpiece ^ ad_swap(crow)) << 4);
  const uint32_t to_x = kXPiece == 16 ? to_row : crow * 128 + ((cpiece ^ ((crow & 3) << 2)) << 3);
  const uint32_t to_b = (uint32_t)(tid ^ ad_swap_b(tid / kBPieces, kBPieces)) * 16;
  // Operands: the lane's places in a stage at contraction index 0 (further ones by an exclusive or with the piece's index)
  const int row0 = mw * 16 + g, col = nh * (kCols / 2);      // the lane's first token, the warp's first column in a chunk of out
  const int l8 = lane & 7, l1 = lane >> 3 & 1, l2 = lane >> 4;
  const uint32_t from_x = kMatrixX ? (mw * 16 + l8 + 8 * l1) * 256 + ((l2 ^ ad_swap(l8)) << 4)
                                   : kXPiece == 16 ? row0 * 256 + ((q ^ ad_swap(g)) << 4) : row0 * 128 + ((q ^ ((g & 3) << 2)) << 3);
  const uint32_t from_a = kW + (kMatrixX ? (nh * NTH * 8 + l2 * 8 + l8) * 256 + ((l1 ^ ad_swap(l8)) << 4)
                                         : (nh * NTH * 8 + g) * 256 + ((q ^ ad_swap(g)) << 4));
  const int b_row = kMatrixB ? 8 * (l8 >> 1) + 2 * l2 + (l8 & 1) : P * (g >> 1) + (g & 1);      // (in column tile 0 of unit 0)
  const uint32_t from_b = kW + (col + b_row) * kBRow + (((kMatrixB ? l1 : q) ^ ad_swap_b(b_row, kBPieces)) << 4);
  const uint32_t from_u = us0 + (kMatrixB ? (mw * 16 + l8 + 8 * l1) * kUPitch + ((l2 ^ ad_swap_u(l8, kUPitch)) << 4) : row0 * kUPitch + q * 16);
  // ranks j, j + 1, ... of row t of u, and the bytes from there to the second pieces
  auto u_at = [&](int t, int j) {
    return reinterpret_cast<T*>(us + t * kUPitch + (kMatrixB ? (((j >> 3) ^ ad_swap_u(t, kUPitch)) << 4) + (j & 7) * 2 : j * 4));
  };
  auto u_lo = [&](int t, int j) { return (((j >> 3 ^ ad_swap_u(t, kUPitch)) & RP / 8) ? -1 : 1) * (RP * 2); };
  const uint32_t from_y = row0 * 256 + (((col / P + q) ^ ad_swap(g)) << 4);
  pdl_wait();
  pdl_trigger();
  int n_tiles = cluster + 1;                                 // `here`: a tile for every cluster
  if (here) ad_tile_here(a, cluster, reinterpret_cast<int32_t*>(smem), list, list + kAdTM);
  else n_tiles = *a.n_tiles;
  const X* x = static_cast<const X*>(a.x);
  const T* y = static_cast<const T*>(a.y);
  T* out = static_cast<T*>(a.out);
#pragma unroll 1
  for (int tile = cluster; tile < n_tiles; tile += n_clusters) {
    int rows, adapter;
    if (here) {
      rows = list[kAdTM];
      adapter = list[kAdTM + 1] < a.count ? list[kAdTM + 1] : -1;
      if (rows == 0) break;                                  // the same for the whole cluster
    } else {
      const AdapterTile td = a.tiles[tile];
      rows = td.rows;
      adapter = td.adapter;
      __syncthreads();                                       // the tile in front is done with the list and the stages
      if (tid < rows) list[tid] = a.perm[td.first + tid];
      __syncthreads();
    }
    if (adapter < 0) {                                       // no adapter: rows of y as they are, two chunks at a time
      if (y == out && a.y_stride == a.out_stride) continue;
      constexpr int kRows = kAdTM / 16;
      const T* from[kRows];
      T* to[kRows];
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
        const long long t = list[min(crow + 16 * k, rows - 1)];
        from[k] = y + t * a.y_stride + cpiece * P;
        to[k] = out + t * a.out_stride + cpiece * P;
      }
      for (int c = cta * kCols; c < a.n; c += 2 * C * kCols) {
        uint4 v[2][kRows];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int k = 0; k < kRows; ++k) {
            ad_zero(v[h][k]);
            const int at = c + h * C * kCols;
            if (y != nullptr && at + cpiece * P < a.n && crow + 16 * k < rows) v[h][k] = *reinterpret_cast<const uint4*>(from[k] + at);
          }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int k = 0; k < kRows; ++k) {
            const int at = c + h * C * kCols;
            if (at + cpiece * P < a.n && crow + 16 * k < rows) *reinterpret_cast<uint4*>(to[k] + at) = v[h][k];
          }
      }
      continue;
    }
    // sources of the next chunk: they move on by C chunks with every request
    const char *xp[kAdTM / 16], *yp[kAdTM / 16];
#pragma unroll
    for (int k = 0; k < kAdTM / 16; ++k) {
      const long long t = list[min(crow + 16 * k, rows - 1)];
      xp[k] = reinterpret_cast<const char*>(x + t * a.x_stride) + cpiece * kXPiece + cta * kXRow;
      yp[k] = reinterpret_cast<const char*>(y + t * a.y_stride) + cpiece * 16 + cta * kAdChunk;
    }
    const char* ap = reinterpret_cast<const char*>(static_cast<const T*>(a.A) + ((long long)adapter * r + crow) * a.d) + cpiece * 16 +
                     cta * kAdChunk;
    const char* bp = reinterpret_cast<const char*>(static_cast<const T*>(a.B) + ((long long)adapter * a.n + cta * kCols) * r);
    const int a_step = 16 * a.d * kElem;
    const int n_rows = (rows - crow + 15) >> 4, n_ranks = (r - crow + 15) >> 4;      // rows crow + 16 k below rows, r
    int cx = cta * kCols, cy = cta * kCols;                  // first column of the next chunk of x, of y
    auto request_x = [&](uint32_t stage) {
      if (cx + cpiece * P < a.d) {
#pragma unroll
        for (int k = 0; k < kAdTM / 16; ++k) {
          if (k < n_rows) ad_copy<kXPiece>(stage + to_x + k * (16 * kXRow), xp[k]);
          xp[k] += C * kXRow;
        }
#pragma unroll
        for (int k = 0; k < NTH; ++k)
          if (k < n_ranks) ad_copy<16>(stage + kW + to_row + k * 4096, ap + k * a_step);
        ap += C * kAdChunk;
      } else if (cx < a.d) {                                 // beyond the rows: zeros
#pragma unroll
        for (int k = 0; k < kAdTM / 16; ++k) ad_clear<kXPiece>(stage + to_x + k * (16 * kXRow));
#pragma unroll
        for (int k = 0; k < NTH; ++k)
          if (k < n_ranks) ad_clear<16>(stage + kW + to_row + k * 4096);
      }
      cx += C * kCols;
    };
    auto request_y = [&](uint32_t stage) {
      if (y != nullptr && cy + cpiece * P < a.n) {
#pragma unroll
        for (int k = 0; k < kAdTM / 16; ++k) {
          if (k < n_rows) ad_copy<16>(stage + to_row + k * 4096, yp[k]);
          yp[k] += C * kAdChunk;
        }
      }
      const int pieces = min(kCols, a.n - cy) * kBPieces;
      if (r == RP) {
#pragma unroll
        for (int k = 0; k < NTH; ++k)                        // 16 r pieces in all
          if (tid + kAdThreads * k < pieces)
            ad_copy<16>(stage + kW + (to_b ^ (ad_swap_b(kAdThreads * k / kBPieces, kBPieces) << 4)) + k * 4096, bp + (tid + kAdThreads * k) * 16);
      } else {                                               // ranks that B does not have: zeros
        for (int p = tid; p < pieces; p += kAdThreads) {
          const int c = p / kBPieces, j = p % kBPieces;
          const uint32_t at = stage + kW + c * kBRow + ((j ^ ad_swap_b(c, kBPieces)) << 4);
          if (j < per_row) ad_copy<16>(at, bp + (c * per_row + j) * 16);
          else ad_clear<16>(at);
        }
      }
      bp += (long long)C * kCols * r * kElem;
      cy += C * kCols;
    };
    const int items = x_iters + y_iters;
    for (int i = 0; i < stages - 1; ++i) {
      if (i < x_iters) request_x(stage0 + i * kStage);
      else if (i < items) request_y(stage0 + i * kStage);
      ad_copy_commit();
    }
    uint32_t at = 0, before = (stages - 1) * kStage;         // stages of item i and of item i - 1
    const bool mine = mw * 16 < rows;                        // the warp has tokens
    float acc[NTH][4];
#pragma unroll
    for (int h = 0; h < NTH; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[h][e] = 0.f;
    T* op[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) op[i] = out + (long long)list[min(row0 + 8 * i, rows - 1)] * a.out_stride + cta * kCols + col + q * P;
    // ---- first product.  (Ranks beyond r are multiplied too: whatever their rows of A hold goes into results nobody reads.)
#pragma unroll 1
    for (int i = 0; i < x_iters; ++i) {
      ad_copy_wait(stages - 2);
      __syncthreads();
      if (i + stages - 1 < x_iters) request_x(stage0 + before);
      else if (i + stages - 1 < items) request_y(stage0 + before);
      ad_copy_commit();
      const uint32_t st = stage0 + at;
      before = at;
      at = at + kStage == stages * kStage ? 0u : at + kStage;
      if (!mine || (cta + i * C) * kCols >= a.d) continue;
      if constexpr (kMatrixX) {
#pragma unroll
        for (int s = 0; s < 8; ++s) {                        // 16 columns
          uint32_t p[4];
          ad_ldmatrix(p, (st + from_x) ^ (s * 32));
          if constexpr (NTH == 1) {
            uint32_t w[2];
            ad_ldmatrix(w, (st + from_a) ^ (s * 32));
            mma_bf16_16x8x16(acc[0], p[0], p[1], p[2], p[3], w[0], w[1]);
          } else {
#pragma unroll
            for (int h = 0; h + 1 < NTH; h += 2) {
              uint32_t w[4];
              ad_ldmatrix(w, ((st + from_a) ^ (s * 32)) + h * 2048);
              mma_bf16_16x8x16(acc[h], p[0], p[1], p[2], p[3], w[0], w[1]);
              mma_bf16_16x8x16(acc[h + 1], p[0], p[1], p[2], p[3], w[2], w[3]);
            }
          }
        }
      } else {
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          uint4 p, p8;
          if constexpr (kXPiece == 16) {
            p = ad_lds((st + from_x) ^ (s * 64));
            p8 = ad_lds(((st + from_x) ^ (s * 64)) + 8 * kXRow);
          } else {
            p = ad_lds8((st + from_x) ^ (s * 32));
            p8 = ad_lds8(((st + from_x) ^ (s * 32)) + 8 * kXRow);
          }
          const AdLeft<T> left(p, p8);
#pragma unroll
          for (int h = 0; h < NTH; ++h) ad_step(acc[h], left, ad_lds(((st + from_a) ^ (s * 64)) + h * 2048));
        }
      }
    }
    ad_copy_wait(stages - 2);
    __syncthreads();
    {
      // ---- u = scale * A x: the CTAs' parts are added in their order
      const float sc = a.scale != nullptr ? a.scale[adapter] : 1.f;
      if (C == 1) {
        if (mine) {
          float f[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) f[e] = a.x_scales != nullptr ? sc * a.x_scales[list[min(row0 + 8 * e, rows - 1)]] : sc;
#pragma unroll
          for (int h = 0; h < NTH; ++h) {
            if ((nh * NTH + h) * 8 >= r)                     // ranks that A does not have
              acc[h][0] = acc[h][1] = acc[h][2] = acc[h][3] = 0.f;
            if constexpr (kElem == 4) {
#pragma unroll
              for (int e = 0; e < 2; ++e)
                if (!(fabsf(acc[h][2 * e]) + fabsf(acc[h][2 * e + 1]) < CUDART_INF_F) && row0 + 8 * e < rows) {
                  const float2 u = ad_again_u(x + (long long)list[row0 + 8 * e] * a.x_stride,
                                              static_cast<const T*>(a.A) + ((long long)adapter * r + (nh * NTH + h) * 8 + 2 * q) * a.d, a.d);
                  acc[h][2 * e] = u.x;
                  acc[h][2 * e + 1] = u.y;
                }
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int t = row0 + 8 * e, j = (nh * NTH + h) * 8 + 2 * q;
              ad_store_u2(u_at(t, j), acc[h][2 * e] * f[e], acc[h][2 * e + 1] * f[e], u_lo(t, j));
            }
          }
        }
      } else {
        float* part = ad_own_part(RP) ? own_part : reinterpret_cast<float*>(smem + before);   // (the stage just multiplied)
        if (mine) {
#pragma unroll
          for (int h = 0; h < NTH; ++h) {
            float* p = part + row0 * RP + (nh * NTH + h) * 8 + 2 * q;
            *reinterpret_cast<float2*>(p) = make_float2(acc[h][0], acc[h][1]);
            *reinterpret_cast<float2*>(p + 8 * RP) = make_float2(acc[h][2], acc[h][3]);
          }
        }
        cluster_arrive();
        cluster_wait();
        for (int k = tid * 4; k < rows * RP; k += kAdThreads * 4) {
          const int t = k / RP, j = k % RP;
          float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
          if (j < r) {                                       // (ranks that A does not have: zeros)
            s = ld_cluster4(part + k, 0);
#pragma unroll
            for (int c = 1; c < kAdMaxCtas; ++c) {
              if (c >= C) break;
              const float4 v = ld_cluster4(part + k, c);
              s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
            }
            if constexpr (kElem == 4)
              if (!(fabsf(s.x) + fabsf(s.y) + fabsf(s.z) + fabsf(s.w) < CUDART_INF_F)) {
                const X* row = x + (long long)list[t] * a.x_stride;
                const T* w = static_cast<const T*>(a.A) + ((long long)adapter * r + j) * a.d;
                const float2 lo = ad_again_u(row, w, a.d), hi = ad_again_u(row, w + 2ll * a.d, a.d);
                s = make_float4(lo.x, lo.y, hi.x, hi.y);
              }
          }
          const float f = a.x_scales != nullptr ? sc * a.x_scales[list[t]] : sc;
          ad_store_u(u_at(t, j), make_float4(s.x * f, s.y * f, s.z * f, s.w * f), u_lo(t, j));
        }
        cluster_arrive();
        if (!ad_own_part(RP)) cluster_wait();                // the stage is free again
      }
      __syncthreads();
    }
    // ---- second product: out = y + u B, two units of four lanes' pieces of columns
    int c0 = cta * kCols;
#pragma unroll 1
    for (int i = x_iters; i < items; ++i) {
      if (i > x_iters) {
        ad_copy_wait(stages - 2);
        __syncthreads();
      }
      if (i + stages - 1 < items) request_y(stage0 + before);
      ad_copy_commit();
      const uint32_t st = stage0 + at;
      before = at;
      at = at + kStage == stages * kStage ? 0u : at + kStage;
      if (mine && c0 < a.n) {
        float d[2][NT][4];
#pragma unroll
        for (int v = 0; v < 2; ++v)
#pragma unroll
          for (int h = 0; h < NT; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) d[v][h][e] = 0.f;
        if constexpr (kMatrixB) {
#pragma unroll
          for (int k = 0; k < RP / 16; ++k) {
            uint32_t p[4], rest[4], w[2][2][4];
            ad_ldmatrix(p, from_u ^ (k * 32));
            ad_ldmatrix(rest, from_u ^ (RP * 2 + k * 32));
#pragma unroll
            for (int v = 0; v < 2; ++v)
#pragma unroll
              for (int h = 0; h < 2; ++h) ad_ldmatrix(w[v][h], ((st + from_b) ^ (k * 32)) + (v * 4 * P + 4 * h) * kBRow);
            // the second pieces first, eight products between two that add to the same sums (8192 tokens of 4096 at rank 64: two
            // between 67.8 us, four 65.8, eight 64.6; one piece 59.9)
            auto product = [&](const uint32_t (&u)[4]) {
#pragma unroll
              for (int v = 0; v < 2; ++v)
#pragma unroll
                for (int h = 0; h < NT; ++h)
                  mma_bf16_16x8x16(d[v][h], u[0], u[1], u[2], u[3], w[v][h / 2][h % 2 * 2], w[v][h / 2][h % 2 * 2 + 1]);
            };
            product(rest);
            product(p);
          }
        } else {
#pragma unroll
          for (int k = 0; k < kBPieces; k += 4) {
            const AdLeft<T> left(ad_lds(from_u + k * 16), ad_lds(from_u + 8 * kUPitch + k * 16));
#pragma unroll
            for (int v = 0; v < 2; ++v)
#pragma unroll
              for (int h = 0; h < NT; ++h)
                ad_step(d[v][h], left, ad_lds(((st + from_b) ^ (k * 16 ^ ad_swap_b(v * 4 * P, kBPieces) << 4)) + (v * 4 * P + 2 * h) * kBRow));
          }
        }
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          if (c0 + col + v * 4 * P + q * P >= a.n) continue;
          uint4 y0, y8;
          ad_zero(y0);
          ad_zero(y8);
          if (y != nullptr) {
            y0 = ad_lds((st + from_y) ^ (v * 64));
            y8 = ad_lds(((st + from_y) ^ (v * 64)) + 8 * 256);
          }
          auto store = [&](T* to, int row, const uint4& yr, int e) {
            uint4 o = ad_finish(yr, d[v], e, T());
            if constexpr (kElem == 4)
              if (!ad_finite(d[v], e))
                o = ad_again_out(reinterpret_cast<const T*>(us + row * kUPitch),
                                 static_cast<const T*>(a.B) + ((long long)adapter * a.n + c0 + col + v * 4 * P + q * P) * r, r, yr);
            *reinterpret_cast<uint4*>(to + v * 4 * P) = o;
          };
          if (row0 < rows) store(op[0], row0, y0, 0);
          if (row0 + 8 < rows) store(op[1], row0 + 8, y8, 2);
        }
      }
      op[0] += C * kCols;
      op[1] += C * kCols;
      c0 += C * kCols;
    }
    ad_copy_wait(0);
    if (ad_own_part(RP) && C > 1) cluster_wait();            // the others have read the CTA's part
  }
}

// Most tiles that T tokens on `count` adapters can make.
inline int ad_max_tiles(int T, int count) { return T / kAdTM + (T < count + 1 ? T : count + 1); }
constexpr int kAdMaxClusters = 2048;

// Most tokens of adapters_few_kernel.  us for 100 tokens of 2048 with 12 adapters, in it and in adapters_tile_kernel, every token with an
// adapter of its own / runs of 50: bf16 at rank 16 5.7 (65 tokens) and 8.0, 72 13.7 and 13.2 / 14.4 and 18.8, 128 16.5 and 13.2 / 16.7 and
// 19.4; fp32 at rank 40 27.3 and 25.5 / 27.0 and 28.9, 64 30.1 and 25.1 / 30.5 and 28.4, 128 69.6 and 42.0 / 56.3 and 47.5.  fp32
// at rank 64, 72 tokens (clusters of four, two of them per SM; beyond half the SMs there are only two CTAs in each) 19.9 and 24.9.
template <typename T>
inline int ad_direct_tokens(int r, int sm_count) {
  return sizeof(T) == 4 && r > 40 && sm_count / 2 < kAdDirect ? sm_count / 2 : kAdDirect;
}

template <typename X, typename T>
inline cudaError_t adapters_launch(AdapterArgs a, int sm_count, cudaStream_t st, bool pdl, int* kernels) {
  const int elem = (int)sizeof(T);
  *kernels = 1;
  if (a.T <= ad_direct_tokens<T>(a.r, sm_count)) {
    a.ctas = 1;
    // CTAs per cluster: until every SM has one or a CTA's warps one step each.  us, 61 tokens of 4096 with 64 adapters of rank 16:
    // 1 CTA 13.5, 2 11.1, 4 8.2, 8 11.2; one token of 1024: 5.0, 4.3, 4.4, 4.7.
    while (a.ctas < kAdMaxCtas && a.T * a.ctas < sm_count && a.ctas * kAdWarps * (64 / elem) < (a.d > a.n ? a.d : a.n)) a.ctas *= 2;
    auto go = [&](auto kernel) {
      return launch_cluster(kernel, a.ctas, dim3(a.ctas * a.T), dim3(kAdThreads), ad_smem_bytes(a.r, elem), st, pdl, a);
    };
    return ad_rtw(a.r) == 1 ? go(adapters_few_kernel<X, T, 1>) : ad_rtw(a.r) == 2 ? go(adapters_few_kernel<X, T, 2>)
                                                                                  : go(adapters_few_kernel<X, T, 4>);
  }
  const int tiles = ad_max_tiles(a.T, a.count), rp = ad_rank_up(a.r), stages = ad_stages(rp, elem);
  // us, 8192 tokens of 4096 at rank 64: 1 CTA 76, 2 64, 4 73, 8 109 (two CTAs fit an SM, a second round costs as much as the first);
  // 1531 of 768 -> 2240 in fp32 at rank 8: 1 53, 2 31, 4 23, 8 18.
  const int smem = stages * ad_stage_bytes(rp) + ad_tile_rest(rp, elem);
  const int at_once = smem <= kAdTwoBytes ? 2 * sm_count : sm_count;
  a.ctas = 1;
  while (a.ctas < kAdMaxCtas && 10 * tiles * a.ctas <= 6 * at_once) a.ctas *= 2;      // (`tiles` is an upper bound)
  // A plan of its own per CTA where all CTAs run at once (later rounds would pay for it again): us, 1531 tokens, with the plan kernel
  // 20.2, without 18.4.
  const int here = a.T <= kAdHere && tiles * a.ctas <= at_once;
  if (!here) {
    const cudaError_t e = launch_kernel(adapters_plan_kernel, dim3(1), dim3(a.T <= 2048 ? 256 : kAdPlanThreads), 0, st, pdl, a, kAdTM);
    if (e != cudaSuccess) return e;
    *kernels = 2;
  }
  const dim3 grid(a.ctas * (tiles < kAdMaxClusters ? tiles : kAdMaxClusters));
  auto go = [&](auto kernel) {
    return launch_cluster(kernel, a.ctas, grid, dim3(kAdThreads), smem, st, pdl, a, stages, here);
  };
  return rp == 16 ? go(adapters_tile_kernel<X, T, 16>) : rp == 32 ? go(adapters_tile_kernel<X, T, 32>)
       : rp == 64 ? go(adapters_tile_kernel<X, T, 64>) : go(adapters_tile_kernel<X, T, 128>);
}
// Raises the kernels' limit of dynamic shared memory where the default does not do.
template <typename X, typename T>
inline cudaError_t adapters_set_limits() {
  cudaError_t e = cudaSuccess;
  auto raise = [&](auto kernel, int bytes) {
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  };
  raise(adapters_few_kernel<X, T, 4>, ad_smem_bytes(kAdMaxRank, (int)sizeof(T)));
  raise(adapters_tile_kernel<X, T, 16>, kAdOneBytes);
  raise(adapters_tile_kernel<X, T, 32>, kAdOneBytes);
  raise(adapters_tile_kernel<X, T, 64>, kAdOneBytes);
  raise(adapters_tile_kernel<X, T, 128>, kAdOneBytes);
  return e;
}

}  // namespace swapmoe
