// Low-rank adapters of many requests beside a projection that all of them share:
//   out[t] = y[t] + scale_a * B_a (A_a x[t]),  a = ids[t]  (no adapter: out[t] = y[t]),
// A_a [rank, d_in], B_a [d_out, rank], y the shared projection's row.
//
// Bound by bytes: x, y and out once, the adapters that are asked for once per tile of tokens; the products are rank * 2 operations
// per element of x and out.  One launch does both products.  Tokens of one adapter form tiles of up to TM; a cluster of eight
// CTAs takes a tile: CTA c multiplies every eighth 256-byte chunk of the rows of x by A (warp-level mma, tokens as mma rows), the
// CTAs exchange their parts of A x through distributed shared memory, and CTA c adds B (A x) to every eighth chunk of the rows of y.
// Rows of x and y come in, and rows of out leave, by bulk copies of 256 bytes from and to wherever the token sits; the first chunks
// of y are requested with those of x.  A and B go from L2 to registers: no two warps of a CTA need the same piece.
//
// Within a step of 64 bytes a thread's 16-byte piece holds its operands of two (bf16) mma: the contraction index is permuted
// the same way for both operands.
#pragma once
#include <cuda_fp8.h>

#include "common.cuh"
#include "launch.cuh"
#include "ptx.cuh"

namespace swapmoe {

constexpr int kAdMaxRank = 128, kAdMaxCount = 4096, kAdMaxWidth = 1 << 16;
constexpr int kAdCtas = 8;                 // CTAs per cluster
constexpr int kAdThreads = 256, kAdWarps = kAdThreads / 32;
constexpr int kAdChunk = 256;              // bytes of a row of weights, y and out that a CTA takes at a time
constexpr int kAdSteps = kAdChunk / 64;    // steps of 64 bytes (four lanes' 16-byte pieces) per chunk
constexpr int kAdStages = 2;               // chunks of x, and of y, in shared memory
// Row pitches in shared memory: operand fragments (lanes g, q read piece q of row g) are free of bank conflicts at 64 bytes
// modulo 128 (32 for 8-bit rows' 8-byte pieces), accumulator fragments (4 or 8 bytes at column 2 q) at 16.
constexpr int kAdYPitch = kAdChunk + 16;
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
  int32_t* perm;            // [T]            } written by the plan kernel, for more than kAdDirect tokens
  AdapterTile* tiles;       // [max tiles]    }
  int32_t* n_tiles;         // [1]            }
  int32_t* status;          // [2]
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
// A lane's piece (16 bytes of weights' worth of columns) of a row of x in shared memory.
__device__ __forceinline__ uint4 ad_lds_x(const unsigned char* p, int step, int q, float) {
  return *reinterpret_cast<const uint4*>(p + step * 64 + q * 16);
}
__device__ __forceinline__ uint4 ad_lds_x(const unsigned char* p, int step, int q, bf16) {
  return *reinterpret_cast<const uint4*>(p + step * 64 + q * 16);
}
__device__ __forceinline__ uint4 ad_lds_x(const unsigned char* p, int step, int q, __nv_fp8_e4m3) {
  const uint2 v = *reinterpret_cast<const uint2*>(p + step * 32 + q * 8);
  return make_uint4(e4m3x2_to_bf16x2(v.x), e4m3x2_to_bf16x2(v.x >> 16), e4m3x2_to_bf16x2(v.y), e4m3x2_to_bf16x2(v.y >> 16));
}
__device__ __forceinline__ void ad_store_u(float* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }
__device__ __forceinline__ void ad_store_u(bf16* p, float4 v) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
}
// out = y + delta for two neighbouring columns in shared memory.
__device__ __forceinline__ void ad_add2(unsigned char* p, bool have_y, float d0, float d1, float) {
  float2* q = reinterpret_cast<float2*>(p);
  const float2 y = have_y ? *q : make_float2(0.f, 0.f);
  *q = make_float2(y.x + d0, y.y + d1);
}
__device__ __forceinline__ void ad_add2(unsigned char* p, bool have_y, float d0, float d1, bf16) {
  uint32_t* q = reinterpret_cast<uint32_t*>(p);
  const uint32_t y = have_y ? *q : 0u;
  *q = pack_bf16x2(__uint_as_float(y << 16) + d0, __uint_as_float(y & 0xffff0000u) + d1);
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
__device__ __forceinline__ uint32_t map_to_cta(uint32_t addr, int cta) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(cta));
  return r;
}
__device__ __forceinline__ float4 ld_cluster4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void bulk_store_1d(void* dst, const void* src_smem, uint32_t bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(ptx::smem_u32(src_smem)), "r"(bytes)
               : "memory");
}

__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void bulk_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

// ----------------------------------------------------------------------------- shared memory
struct AdapterSmem { int x, y, part, u, list, bars, total; };
// x_pitch: bytes between rows of a chunk of x; slices: parts of a chunk's steps that run side by side; elem: bytes of a value of T.
__host__ __device__ inline int ad_slices(int r) { return r <= 8 ? 8 : r <= 16 ? 4 : r <= 32 ? 2 : 1; }
__host__ __device__ inline int ad_u_pitch(int r, int elem) {
  const int b = (r * elem + 63) & ~63;
  return b % 128 == 0 ? b + 64 : b;
}
__host__ __device__ inline AdapterSmem ad_layout(int tm, int r, int x_pitch, int elem) {
  AdapterSmem m;
  int o = 0;
  m.x = o;    o += kAdStages * tm * x_pitch;
  m.y = o;    o += kAdStages * tm * kAdYPitch;
  m.part = o; o += ad_slices(r) * tm * r * 4;
  m.u = o;    o += tm * ad_u_pitch(r, elem);
  m.list = o; o += tm * 4;
  m.bars = o; o += 2 * kAdStages * 8 + 16;
  m.total = o;
  return m;
}

// The tile of cluster i without a plan: it has one if token i is the first, or the TM-th, ... of its adapter; then its tokens
// are the next TM of that adapter from i on.  By one warp; T <= 64: lane l holds tokens l and l + 32.
__device__ __forceinline__ int ad_direct_tile(const AdapterArgs& a, int i, int tm, int32_t* list, int* adapter) {
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
  if (__popcll(all & below) % tm != 0) return 0;
  const unsigned long long rest = all & ~below;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int t = lane + 32 * h, at = __popcll(rest & ((1ull << t) - 1));
    if ((rest >> t) & 1 && at < tm) list[at] = t;
  }
  return min(tm, __popcll(rest));
}

// X: rows of x (T or e4m3), T: everything else, TM: most tokens of a tile.
template <typename X, typename T, int TM>
__global__ void __cluster_dims__(kAdCtas, 1, 1) __launch_bounds__(kAdThreads, TM == 64 ? 2 : 3) adapters_kernel(const AdapterArgs a) {
  constexpr int kElem = (int)sizeof(T), kCols = kAdChunk / kElem;         // columns of a chunk
  constexpr int kPiece = 16 / kElem;                                      // values of a lane's piece
  constexpr int kXBytes = kCols * (int)sizeof(X);                         // bytes of a chunk of x
  constexpr int kXPitch = kXBytes + (sizeof(X) == 1 ? 32 : 64);
  constexpr int MT = TM / 16;                                             // mma row tiles
  constexpr int NT = kCols / 8 / kAdWarps;                                // column tiles per warp in the second product
  extern __shared__ __align__(128) unsigned char smem[];
  const AdapterSmem lay = ad_layout(TM, a.r, kXPitch, kElem);
  unsigned char* xs = smem + lay.x;
  unsigned char* ys = smem + lay.y;
  float* part = reinterpret_cast<float*>(smem + lay.part);
  unsigned char* us = smem + lay.u;
  int32_t* list = reinterpret_cast<int32_t*>(smem + lay.list);
  uint64_t* bar_x = reinterpret_cast<uint64_t*>(smem + lay.bars);
  uint64_t* bar_y = bar_x + kAdStages;
  volatile int* ctl = reinterpret_cast<volatile int*>(bar_y + kAdStages);  // [0] a wait gave up, [1] rows, [2] adapter
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), g = lane >> 2, q = lane & 3;
  const int cta = blockIdx.x % kAdCtas, cluster = blockIdx.x / kAdCtas, n_clusters = gridDim.x / kAdCtas;
  const int r = a.r, slices = ad_slices(r), rank_tiles = r / 8, u_pitch = ad_u_pitch(r, kElem);
  const int x_chunks = (a.d + kCols - 1) / kCols, y_chunks = (a.n + kCols - 1) / kCols;
  const int my_x = (x_chunks - cta + kAdCtas - 1) / kAdCtas, my_y = (y_chunks - cta + kAdCtas - 1) / kAdCtas;
  if (tid == 0) {
    for (int i = 0; i < kAdStages; ++i) { ptx::mbar_init(&bar_x[i], 1); ptx::mbar_init(&bar_y[i], 1); }
    ctl[0] = 0;
    ptx::fence_barrier_init();
  }
  pdl_wait();
  pdl_trigger();
  const bool direct = a.T <= kAdDirect;
  const int n_tiles = direct ? a.T : *a.n_tiles;
  const X* x = static_cast<const X*>(a.x);
  const T* y = static_cast<const T*>(a.y);
  T* out = static_cast<T*>(a.out);
  int x_seen = 0, y_seen = 0;              // chunks of the tiles in front: the stage and the barrier's parity follow from them
  bool alive = true, owe_wait = false;     // owe_wait: this CTA has told the others that it has read their parts
#pragma unroll 1
  for (int tile = cluster; tile < n_tiles; tile += n_clusters) {
    __syncthreads();                       // the tile in front is done with the list
    if (direct) {
      if (warp == 0) {
        int adapter;
        const int rows = ad_direct_tile(a, tile, TM, list, &adapter);
        if (lane == 0) { ctl[1] = rows; ctl[2] = adapter; }
      }
    } else {
      const AdapterTile td = a.tiles[tile];
      if (tid < td.rows) list[tid] = a.perm[td.first + tid];
      if (tid == 0) { ctl[1] = td.rows; ctl[2] = td.adapter; }
    }
    __syncthreads();
    const int rows = ctl[1], adapter = ctl[2];
    if (rows == 0) continue;               // the same for the whole cluster
    const int mt = (rows + 15) >> 4;
    const bool work = adapter >= 0;
    // chunk i of this CTA into its stage, by warp 0; a lane's rows lane, lane + 32
    auto load_x = [&](int i) {
      const int c0 = (cta + i * kAdCtas) * kCols, bytes = min(kCols, a.d - c0) * (int)sizeof(X), st = (x_seen + i) % kAdStages;
      if (lane == 0) ptx::mbar_expect_tx(&bar_x[st], (uint32_t)(bytes * rows));
      __syncwarp();
      for (int t = lane; t < rows; t += 32)
        ptx::bulk_load_1d(xs + (st * TM + t) * kXPitch, x + (long long)list[t] * a.x_stride + c0, (uint32_t)bytes, &bar_x[st]);
    };
    auto load_y = [&](int i) {
      const int c0 = (cta + i * kAdCtas) * kCols, bytes = min(kCols, a.n - c0) * kElem, st = (y_seen + i) % kAdStages;
      if (lane == 0) ptx::mbar_expect_tx(&bar_y[st], (uint32_t)(bytes * rows));
      __syncwarp();
      for (int t = lane; t < rows; t += 32)
        ptx::bulk_load_1d(ys + (st * TM + t) * kAdYPitch, y + (long long)list[t] * a.y_stride + c0, (uint32_t)bytes, &bar_y[st]);
    };
    if (warp == 0 && alive) {
      if (work)
        for (int i = 0; i < min(my_x, kAdStages); ++i) load_x(i);
      if (y != nullptr) {
        bulk_wait_read();                  // the stores of the tile in front have left the stages of y
        __syncwarp();
        for (int i = 0; i < min(my_y, kAdStages); ++i) load_y(i);
      }
    }
    if (work) {
      // ---- first product: warp = (rank tile, slice of the steps); tokens are mma rows, ranks mma columns
      const T* A = static_cast<const T*>(a.A) + (long long)adapter * r * a.d;
      const int slice = slices > 1 ? warp % slices : 0, rt0 = slices > 1 ? warp / slices : warp;
      float acc[2][MT][4];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][m][e] = 0.f;
#pragma unroll 1
      for (int i = 0; i < my_x; ++i) {
        const int c0 = (cta + i * kAdCtas) * kCols, st = (x_seen + i) % kAdStages;
        uint4 w[2][kAdSteps];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int s = 0; s < kAdSteps; ++s) {
            const int c = c0 + s * 4 * kPiece + q * kPiece, rt = rt0 + h * kAdWarps;
            w[h][s] = make_uint4(0u, 0u, 0u, 0u);
            if (rt < rank_tiles && ((i * kAdSteps + s) & (slices - 1)) == slice && c < a.d)
              w[h][s] = __ldg(reinterpret_cast<const uint4*>(A + (long long)(rt * 8 + g) * a.d + c));
          }
        if (alive) alive = warp_wait(&bar_x[st], (x_seen + i) / kAdStages & 1, ctl, a.status, 41);
        const unsigned char* xb = xs + st * TM * kXPitch;
#pragma unroll
        for (int s = 0; s < kAdSteps; ++s) {
          if (((i * kAdSteps + s) & (slices - 1)) != slice) continue;
          const bool in = c0 + s * 4 * kPiece + q * kPiece < a.d;
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            if (m >= mt) break;
            const uint4 z = make_uint4(0u, 0u, 0u, 0u);
            const uint4 p = in ? ad_lds_x(xb + (m * 16 + g) * kXPitch, s, q, X()) : z;
            const uint4 p8 = in ? ad_lds_x(xb + (m * 16 + g + 8) * kXPitch, s, q, X()) : z;
#pragma unroll
            for (int h = 0; h < 2; ++h)
              if (rt0 + h * kAdWarps < rank_tiles) ad_step(acc[h][m], p, p8, w[h][s], T());
          }
        }
        if (i + kAdStages < my_x) {
          __syncthreads();                 // all warps are done with the stage
          if (warp == 0 && alive) load_x(i + kAdStages);
        }
      }
      x_seen += my_x;
      // parts of u to shared memory: [slice][token][rank]
      if (owe_wait) cluster_wait();        // everybody has read the parts of the tile in front
      owe_wait = false;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int rt = rt0 + h * kAdWarps;
        if (rt >= rank_tiles) continue;
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          if (m >= mt) break;
          float* p = part + ((long long)slice * TM + m * 16 + g) * r + rt * 8 + 2 * q;
          *reinterpret_cast<float2*>(p) = make_float2(acc[h][m][0], acc[h][m][1]);
          *reinterpret_cast<float2*>(p + 8 * r) = make_float2(acc[h][m][2], acc[h][m][3]);
        }
      }
      if (slices > 1) {
        __syncthreads();
        for (int i = tid; i < rows * r; i += kAdThreads) {
          float s = part[i];
          for (int k = 1; k < slices; ++k) s += part[k * TM * r + i];
          part[i] = s;
        }
      }
      // ---- the CTAs' parts are added, each CTA for itself, in the order of the CTAs
      cluster_arrive();
      cluster_wait();
      {
        const float sc = a.scale != nullptr ? a.scale[adapter] : 1.f;
        const uint32_t mine = ptx::smem_u32(part);
        for (int i = tid * 4; i < rows * r; i += kAdThreads * 4) {
          float4 v[kAdCtas];
#pragma unroll
          for (int c = 0; c < kAdCtas; ++c) v[c] = ld_cluster4(map_to_cta(mine + i * 4, c));
          float4 s = v[0];
#pragma unroll
          for (int c = 1; c < kAdCtas; ++c) { s.x += v[c].x; s.y += v[c].y; s.z += v[c].z; s.w += v[c].w; }
          const int t = i / r, j = i - t * r;
          float f = sc;
          if (a.x_scales != nullptr) f *= a.x_scales[list[t]];
          ad_store_u(reinterpret_cast<T*>(us + t * u_pitch) + j, make_float4(s.x * f, s.y * f, s.z * f, s.w * f));
        }
      }
      cluster_arrive();
      owe_wait = true;
      __syncthreads();                     // u is complete
    }
    // ---- second product: a warp owns NT tiles of eight columns of the chunk; u is the left operand, rows of B the right one
    const T* B = static_cast<const T*>(a.B) + (long long)(work ? adapter : 0) * a.n * r;
#pragma unroll 1
    for (int i = 0; i < my_y; ++i) {
      const int c0 = (cta + i * kAdCtas) * kCols, st = (y_seen + i) % kAdStages, cols = min(kCols, a.n - c0);
      unsigned char* yb = ys + st * TM * kAdYPitch;
      float acc[NT][MT][4];
#pragma unroll
      for (int h = 0; h < NT; ++h)
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[h][m][e] = 0.f;
      if (work) {
#pragma unroll 2
        for (int k0 = 0; k0 < r; k0 += 4 * kPiece) {
          const bool in = k0 + q * kPiece < r;
          uint4 w[NT];
#pragma unroll
          for (int h = 0; h < NT; ++h) {
            const int c = (warp * NT + h) * 8 + g;
            w[h] = make_uint4(0u, 0u, 0u, 0u);
            if (in && c < cols) w[h] = __ldg(reinterpret_cast<const uint4*>(B + (long long)(c0 + c) * r + k0 + q * kPiece));
          }
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            if (m >= mt) break;
            const uint4 z = make_uint4(0u, 0u, 0u, 0u);
            const unsigned char* up = us + (m * 16 + g) * u_pitch + (k0 * kElem + q * 16);
            const uint4 p = in ? *reinterpret_cast<const uint4*>(up) : z, p8 = in ? *reinterpret_cast<const uint4*>(up + 8 * u_pitch) : z;
#pragma unroll
            for (int h = 0; h < NT; ++h) ad_step(acc[h][m], p, p8, w[h], T());
          }
        }
      }
      if (y != nullptr) {
        if (alive) alive = warp_wait(&bar_y[st], (y_seen + i) / kAdStages & 1, ctl, a.status, 42);
      } else {
        if (warp == 0) bulk_wait_read();   // the stage's stores have left it
        __syncthreads();
      }
      if (work || y == nullptr) {
#pragma unroll
        for (int h = 0; h < NT; ++h) {
          const int c = (warp * NT + h) * 8;
          if (c >= cols) continue;
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            if (m >= mt) break;
            unsigned char* p = yb + (m * 16 + g) * kAdYPitch + (c + 2 * q) * kElem;
            ad_add2(p, y != nullptr, acc[h][m][0], acc[h][m][1], T());
            ad_add2(p + 8 * kAdYPitch, y != nullptr, acc[h][m][2], acc[h][m][3], T());
          }
        }
      }
      ptx::fence_proxy_async();            // what the threads wrote is to be seen by the bulk stores
      __syncthreads();
      if (warp == 0 && ctl[0] == 0) {
        for (int t = lane; t < rows; t += 32)
          bulk_store_1d(out + (long long)list[t] * a.out_stride + c0, yb + t * kAdYPitch, (uint32_t)(cols * kElem));
        bulk_commit();
        if (y != nullptr && i + kAdStages < my_y) {
          bulk_wait_read();                // (by the lanes that issued the stores)
          __syncwarp();
          load_y(i + kAdStages);
        }
      }
    }
    y_seen += my_y;
  }
  if (warp == 0) bulk_wait_all();
  if (owe_wait) cluster_wait();            // nobody leaves while others read its part
  if (!alive && tid == 0) {
    // a wait gave up: let copies that may still be in flight land before the shared memory is given back
    const uint64_t t0 = ptx::globaltimer_ns();
    while (ptx::globaltimer_ns() - t0 < 2000000ull) __nanosleep(1000);
  }
}

// Most tiles that T tokens on `count` adapters can make.
inline int ad_max_tiles(int T, int count, int tm) { return T / tm + (T < count + 1 ? T : count + 1); }
constexpr int kAdMaxClusters = 1024;
constexpr int kAdMinTile = 32;

template <typename X, typename T, int TM>
inline size_t adapters_smem_bytes(int r) {
  return (size_t)ad_layout(TM, r, kAdChunk / (int)sizeof(T) * (int)sizeof(X) + (sizeof(X) == 1 ? 32 : 64), (int)sizeof(T)).total;
}
template <typename X, typename T, int TM>
inline cudaError_t adapters_launch_tile(const AdapterArgs& a, cudaStream_t st, bool pdl) {
  int tiles = a.T;
  if (a.T > kAdDirect) {
    const cudaError_t e = launch_kernel(adapters_plan_kernel, dim3(1), dim3(kAdPlanThreads), 0, st, pdl, a, TM);
    if (e != cudaSuccess) return e;
    tiles = ad_max_tiles(a.T, a.count, TM);
  }
  const size_t smem = adapters_smem_bytes<X, T, TM>(a.r);
  return launch_kernel(adapters_kernel<X, T, TM>, dim3(kAdCtas * (tiles < kAdMaxClusters ? tiles : kAdMaxClusters)), dim3(kAdThreads),
                       smem, st, pdl, a);
}
template <typename X, typename T>
inline cudaError_t adapters_launch(const AdapterArgs& a, cudaStream_t st, bool pdl) {
  if (sizeof(T) == 2 && a.r >= 48 && a.T > kAdDirect) return adapters_launch_tile<X, T, sizeof(T) == 2 ? 64 : 32>(a, st, pdl);
  return adapters_launch_tile<X, T, 32>(a, st, pdl);
}
// Raises the kernels' limit of dynamic shared memory (once per device and process would do).
inline cudaError_t adapters_set_limits() {
  cudaError_t e = cudaSuccess;
  auto raise = [&](auto kernel, size_t bytes) {
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  };
  raise(adapters_kernel<float, float, 32>, adapters_smem_bytes<float, float, 32>(kAdMaxRank));
  raise(adapters_kernel<bf16, bf16, 32>, adapters_smem_bytes<bf16, bf16, 32>(kAdMaxRank));
  raise(adapters_kernel<bf16, bf16, 64>, adapters_smem_bytes<bf16, bf16, 64>(kAdMaxRank));
  raise(adapters_kernel<__nv_fp8_e4m3, bf16, 32>, adapters_smem_bytes<__nv_fp8_e4m3, bf16, 32>(kAdMaxRank));
  raise(adapters_kernel<__nv_fp8_e4m3, bf16, 64>, adapters_smem_bytes<__nv_fp8_e4m3, bf16, 64>(kAdMaxRank));
  return e;
}

}  // namespace swapmoe
