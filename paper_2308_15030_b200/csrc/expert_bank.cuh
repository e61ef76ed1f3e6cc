// Experts in 8-bit integers behind a router: out[t] = sum_j weights[t, j] * E_slot[t, j](x[t]),  E(x) = W_out act(W_in x).
//
// Pairs (token, choice) are laid out by slot, every slot's rows from a multiple of 32 on, so that the products (int8_gemm.cuh) walk token
// tiles of one slot each.  Where a pair comes to lie inside its slot hangs on the order of atomics; no result does, since every row is
// computed by itself and a token's choices are added in their order.
//   count (more than kBankDirectPairs pairs only): pairs per slot, and every CTA's share of a slot
//   gather: slot offsets, token tiles, rows of x8 with their scales to their places
//   product, activation in fp32 with the rows' largest magnitudes; rows to 8 bits; product; combine.
// The products are bound by the weights' bytes or the tensor cores, the rest by HBM.  Eight experts of 4096 x 14336, 8192 pairs: 690 and 330 us of
// products, hidden rows 86 (6.8 TB/s), combine 25, gather 9 in a short run; whole calls 1160 to 1355 in a graph and 1385 to 1435 back to back, by what the power
// cap leaves of the clock.  64 experts of 2048 x 1024, 244 pairs: 73 us, 64 of them the products'.
#pragma once
#include "int8_gemm.cuh"
#include "quantize_rows.cuh"

namespace swapmoe {

constexpr int kBankMaxSlots = 256;
constexpr int kBankThreads = 256;
constexpr int kBankMaxCtas = 512;               // CTAs of the count and gather kernels
constexpr int kBankDirectPairs = 4096;          // up to here every CTA of the gather kernel counts all pairs itself (us of a call, itself / count kernel: 64
                                                // experts of 1024 x 512, 256 pairs 29.4 / 32.0, 4000 50.3 / 52.1, 6000 62.6 / 58.8; 16 of 4096 x 512, 4000
                                                // pairs 77.3 / 79.4, 8000 126 / 122)

struct BankArgs {
  const int8_t* x8;
  const float* x_scales;
  const int32_t* slots;
  int8_t* rows8;                // [rows, d]
  float* row_scales;
  int32_t *row_pair, *pair_row; // pair of a row (-1: none), row of a pair (-1: none)
  int32_t* largest;             // [rows]
  int32_t *counts, *cta_base;   // [S] zero between calls; [CTAs, S]
  TileDesc* tiles;
  int32_t* n_tiles;             // [0] tiles, [1] most rows of one, [2] rows with the slots' padding
  long long x_stride;
  int P, S, k, d, per_cta;      // pairs, ..., pairs of a CTA
  int cols[2], k_blocks[2];     // weight tiles of a slot, k-blocks of a tile: of the two products
  int pairs;                    // CTA pairs that walk the tiles
};

__device__ __forceinline__ int bank_slot(const BankArgs& a, int p) {
  const int s = a.slots[p];
  return (unsigned)s < (unsigned)a.S ? s : -1;
}

__global__ void __launch_bounds__(kBankThreads) bank_count_kernel(const __grid_constant__ BankArgs a) {
  __shared__ int s_count[kBankMaxSlots];
  for (int s = threadIdx.x; s < a.S; s += kBankThreads) s_count[s] = 0;
  pdl_wait();
  pdl_trigger();
  __syncthreads();
  const int p0 = blockIdx.x * a.per_cta, p1 = min(a.P, p0 + a.per_cta);
  for (int p = p0 + threadIdx.x; p < p1; p += kBankThreads) {
    const int s = bank_slot(a, p);
    if (s >= 0) atomicAdd(&s_count[s], 1);
  }
  __syncthreads();
  for (int s = threadIdx.x; s < a.S; s += kBankThreads)
    a.cta_base[(size_t)blockIdx.x * a.S + s] = s_count[s] ? atomicAdd(&a.counts[s], s_count[s]) : 0;
}

// Most rows of a token tile, by a warp.  Slots of up to 128 rows: one tile each.  Else of 128, 160 ... 256 the one whose rounds of tiles over
// the pairs of CTAs cost least in both products (int8_tile_cost): a round that only a few pairs have work for costs as much as a full one (4096 x
// 14336, eight slots: 38 tiles of 256 are 8.2 rounds of the second product, and take nine).
__device__ __forceinline__ int bank_tile_cap(const BankArgs& a, const int* s_count) {
  const int lane = threadIdx.x & 31;
  int most = 0;
  for (int s = lane; s < a.S; s += 32) most = max(most, s_count[s]);
  most = __reduce_max_sync(0xffffffffu, most);
  if (most <= 128) return most <= 64 ? 64 : 128;
  int best = 256;
  float least = CUDART_INF_F;
  const float inv = 1.f / (float)a.pairs;
  for (int cap = 128; cap <= 256; cap += 32) {
    int n = 0;
    for (int s = lane; s < a.S; s += 32) n += (s_count[s] + cap - 1) / cap;
    const float tiles = (float)__reduce_add_sync(0xffffffffu, n) * inv;
    const float cost = (ceilf(tiles * (float)a.cols[0]) * (float)a.k_blocks[0] + ceilf(tiles * (float)a.cols[1]) * (float)a.k_blocks[1]) * (float)int8_tile_cost(cap);
    if (cost < least) { least = cost; best = cap; }
  }
  return best;
}

// Rows of x8 to their places by the CTA's warps, kRows of them and eight pieces of 16 bytes a lane on their way at once.
template <int kRows>
__device__ __forceinline__ void bank_copy_rows(const BankArgs& a, const int* s_row, int pair0, int n) {
  constexpr int kPieces = 8 / kRows, kWarps = kBankThreads / 32;
  const int lane = threadIdx.x & 31, quads = a.d / 16;
  for (int i = threadIdx.x >> 5; i < n; i += kRows * kWarps)
    for (int c0 = lane; c0 < quads; c0 += 32 * kPieces) {
      uint4 v[kRows][kPieces];
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        const int j = i + r * kWarps;
        const uint4* src = reinterpret_cast<const uint4*>(a.x8 + (size_t)((pair0 + min(j, n - 1)) / a.k) * a.x_stride);
#pragma unroll
        for (int u = 0; u < kPieces; ++u)
          if (j < n && c0 + 32 * u < quads) v[r][u] = src[c0 + 32 * u];
      }
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        const int j = i + r * kWarps, to = j < n ? s_row[j] : -1;
        uint4* dst = reinterpret_cast<uint4*>(a.rows8 + (size_t)max(to, 0) * a.d);
#pragma unroll
        for (int u = 0; u < kPieces; ++u)
          if (to >= 0 && c0 + 32 * u < quads) dst[c0 + 32 * u] = v[r][u];
      }
    }
}

// Slot offsets, by a warp; with `lists` also the list of tiles, and what says that the slots' padding holds no pairs.
__device__ __forceinline__ void bank_offsets(const BankArgs& a, const int* s_count, int* s_off, bool lists) {
  const int lane = threadIdx.x & 31;
  const int cap = lists ? bank_tile_cap(a, s_count) : 256;                   // (of no use without)
  int row0 = 0, tile0 = 0;
  for (int s0 = 0; s0 < a.S; s0 += 32) {
    const int s = s0 + lane, count = s < a.S ? s_count[s] : 0;
    // a slot's rows in as few tiles as the cap allows, by 32 and as even as that can be
    const int padded = (count + 31) & ~31, used = (count + cap - 1) / cap;
    int rows = padded, tiles = used;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, rows, o), v = __shfl_up_sync(0xffffffffu, tiles, o);
      if (lane >= o) { rows += u; tiles += v; }
    }
    const int off = row0 + rows - padded;
    if (s < a.S) s_off[s] = off;
    if (lists) {
      for (int i = 0, at = 0; i < used; ++i) {
        const int units = padded / 32, height = (units / used + (i < units % used ? 1 : 0)) * 32;
        TileDesc td;
        td.phys = td.slot = s; td.row0 = off + at; td.rows = min(height, count - at);
        a.tiles[tile0 + tiles - used + i] = td;
        at += height;
      }
      for (int r = count; r < padded; ++r) a.row_pair[off + r] = -1;
    }
    row0 += __shfl_sync(0xffffffffu, rows, 31);
    tile0 += __shfl_sync(0xffffffffu, tiles, 31);
  }
  if (lists && lane == 0) { a.n_tiles[0] = tile0; a.n_tiles[1] = cap; a.n_tiles[2] = row0; }
}

__device__ __forceinline__ void bank_place(const BankArgs& a, int p, int row, float x_scale) {
  a.row_pair[row] = p;
  a.largest[row] = 0;
  a.row_scales[row] = x_scale;
}

__global__ void __launch_bounds__(kBankThreads) bank_gather_kernel(const __grid_constant__ BankArgs a) {
  __shared__ int s_count[kBankMaxSlots], s_at[kBankMaxSlots], s_off[kBankMaxSlots];
  __shared__ int s_row[kBankThreads];
  const int p0 = blockIdx.x * a.per_cta, p1 = min(a.P, p0 + a.per_cta);
  pdl_wait();
  pdl_trigger();
  for (int s = threadIdx.x; s < a.S; s += kBankThreads) {
    s_count[s] = __ldcg(a.counts + s);
    s_at[s] = a.cta_base[(size_t)blockIdx.x * a.S + s];
  }
  __syncthreads();
  if (threadIdx.x < 32) bank_offsets(a, s_count, s_off, blockIdx.x == 0);
  __syncthreads();
  for (int b = p0; b < p1; b += kBankThreads) {
    const int p = b + threadIdx.x, n = min(kBankThreads, p1 - b);
    int row = -1;
    if (p < p1) {
      const int s = bank_slot(a, p);
      if (s >= 0) {
        row = s_off[s] + atomicAdd(&s_at[s], 1);
        bank_place(a, p, row, a.x_scales[p / a.k]);
      }
      a.pair_row[p] = row;
    }
    s_row[threadIdx.x] = row;
    __syncthreads();
    if (a.d <= 1024) bank_copy_rows<4>(a, s_row, b, n);
    else if (a.d <= 2048) bank_copy_rows<2>(a, s_row, b, n);
    else bank_copy_rows<1>(a, s_row, b, n);
    __syncthreads();
  }
}

// The same for up to kBankDirectPairs pairs, without a count kernel: every CTA counts all pairs.  A warp takes a pair, whose row (its first 4096
// columns) is asked for before the pairs are counted; the last CTA takes none and makes the lists.
constexpr int kBankDirectWarps = kBankThreads / 32;
__global__ void __launch_bounds__(kBankThreads) bank_gather_direct_kernel(const __grid_constant__ BankArgs a) {
  __shared__ int s_count[kBankMaxSlots], s_at[kBankMaxSlots];
  constexpr int kPieces = 8;
  const int lane = threadIdx.x & 31, p0 = blockIdx.x * kBankDirectWarps, p = p0 + (threadIdx.x >> 5), quads = a.d / 16;
  const bool lists = blockIdx.x == gridDim.x - 1, mine = !lists && p < a.P;
  for (int s = threadIdx.x; s < a.S; s += kBankThreads) s_count[s] = s_at[s] = 0;
  pdl_wait();
  pdl_trigger();
  const int slot = mine ? bank_slot(a, p) : -1, token = mine ? p / a.k : 0;
  const float x_scale = mine ? a.x_scales[token] : 0.f;
  const uint4* src = reinterpret_cast<const uint4*>(a.x8 + (size_t)token * a.x_stride);
  uint4 v[kPieces];
#pragma unroll
  for (int u = 0; u < kPieces; ++u)
    if (mine && lane + 32 * u < quads) v[u] = src[lane + 32 * u];
  __syncthreads();
  for (int q = threadIdx.x; q < a.P; q += kBankThreads) {
    const int s = bank_slot(a, q);
    if (s < 0) continue;
    atomicAdd(&s_count[s], 1);
    if (q < p0) atomicAdd(&s_at[s], 1);
  }
  __syncthreads();
  if (lists) {
    if (threadIdx.x < 32) bank_offsets(a, s_count, s_at, true);
    return;
  }
  if (!mine) return;
  int off = 0, row = -1;
  for (int s = lane; s < slot; s += 32) off += (s_count[s] + 31) & ~31;
  off = __reduce_add_sync(0xffffffffu, off);
  if (lane == 0) {
    if (slot >= 0) {
      row = off + atomicAdd(&s_at[slot], 1);
      bank_place(a, p, row, x_scale);
    }
    a.pair_row[p] = row;
  }
  row = __shfl_sync(0xffffffffu, row, 0);
  if (row < 0) return;
  uint4* dst = reinterpret_cast<uint4*>(a.rows8 + (size_t)row * a.d);
#pragma unroll
  for (int u = 0; u < kPieces; ++u)
    if (lane + 32 * u < quads) dst[lane + 32 * u] = v[u];
  for (int c = lane + 32 * kPieces; c < quads; c += 32) dst[c] = src[c];
}

// Hidden values to 8 bits by the rows' largest magnitudes, as quantize_rows does it: a warp per row and 128 kTurns columns, so that the values
// are asked for together with what says whether the row holds a pair; or, where most rows would not (few pairs), per pair.
struct BankQuantizeArgs {
  const float* h;               // [rows, F]
  const int32_t *largest, *row_pair, *pair_row, *n_tiles;
  uint8_t* h8;
  float* h_scales;
  int F, parts;                 // parts of a row
  int n;                        // rows, or pairs
  int by_pair;
};

template <int kTurns>
__global__ void __launch_bounds__(kBankThreads, kTurns == 8 ? 4 : 6) bank_quantize_kernel(const __grid_constant__ BankQuantizeArgs a) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, unit = blockIdx.x * (kBankThreads / 32) + (threadIdx.x >> 5);
  const int index = unit / a.parts, part = unit - index * a.parts;
  if (index >= a.n) return;
  const int row = a.by_pair ? __ldcg(a.pair_row + index) : index;
  if (row < 0) return;
  const int c0 = part * 128 * kTurns + 4 * lane;
  const float* h = a.h + (size_t)row * a.F;
  float4 v[kTurns];
#pragma unroll
  for (int u = 0; u < kTurns; ++u)
    v[u] = c0 + 128 * u < a.F ? __ldcs(reinterpret_cast<const float4*>(h + c0 + 128 * u)) : make_float4(0.f, 0.f, 0.f, 0.f);
  const float most = __int_as_float(__ldcg(a.largest + row));
  if (!a.by_pair) {
    const int rows = __ldcg(a.n_tiles + 2), pair = __ldcg(a.row_pair + row);
    if (row >= rows || pair < 0) return;
  }
  const float divisor = quantize_divisor(most), inverse = __frcp_rn(divisor);
  if (part == 0 && lane == 0) a.h_scales[row] = most == 0.f ? 0.f : divisor;
  uint32_t* out = reinterpret_cast<uint32_t*>(a.h8 + (size_t)row * a.F);
#pragma unroll
  for (int u = 0; u < kTurns; u += 2) {
    float f[8] = {v[u].x, v[u].y, v[u].z, v[u].w, v[u + 1].x, v[u + 1].y, v[u + 1].z, v[u + 1].w};
    uint32_t q[8];
    quotients8(f, divisor, inverse, q);
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (c0 + 128 * (u + i) < a.F) out[(c0 + 128 * (u + i)) / 4] = pack_bytes(q + 4 * i);
  }
}

struct BankCombineArgs {
  const float* y;               // [rows, d]
  const int32_t* pair_row;
  const float* weights;
  int32_t* counts;
  void* out;
  long long out_stride;
  int T, k, d, S, vec;
};

// A CTA per token: four columns a thread and turn, kTurns turns of kRows rows on their way at once.
template <typename T, int kTurns, int kRows>
__global__ void __launch_bounds__(256) bank_combine_kernel(const __grid_constant__ BankCombineArgs a) {
  pdl_wait();
  pdl_trigger();
  const int t = blockIdx.x;
  if (t == 0)
    for (int s = threadIdx.x; s < a.S; s += 256) a.counts[s] = 0;     // for the next call
  const int32_t* rows = a.pair_row + (size_t)t * a.k;
  const float* weights = a.weights + (size_t)t * a.k;
  for (int c0 = 4 * threadIdx.x; c0 < a.d; c0 += 1024 * kTurns) {
    float acc[kTurns][4] = {};
    for (int j0 = 0; j0 < a.k; j0 += kRows) {
      float4 v[kRows][kTurns];
      float w[kRows];
      bool have[kRows];
#pragma unroll
      for (int j = 0; j < kRows; ++j) {
        const int row = j0 + j < a.k ? rows[j0 + j] : -1;
        have[j] = row >= 0;
        w[j] = have[j] ? weights[j0 + j] : 0.f;
        const float* y = a.y + (size_t)max(row, 0) * a.d;
#pragma unroll
        for (int u = 0; u < kTurns; ++u)
          if (have[j] && c0 + 1024 * u < a.d) v[j][u] = __ldcs(reinterpret_cast<const float4*>(y + c0 + 1024 * u));
      }
#pragma unroll
      for (int j = 0; j < kRows; ++j)
        if (have[j])
#pragma unroll
          for (int u = 0; u < kTurns; ++u) {
            acc[u][0] = fmaf(w[j], v[j][u].x, acc[u][0]); acc[u][1] = fmaf(w[j], v[j][u].y, acc[u][1]);
            acc[u][2] = fmaf(w[j], v[j][u].z, acc[u][2]); acc[u][3] = fmaf(w[j], v[j][u].w, acc[u][3]);
          }
    }
    T* out = static_cast<T*>(a.out) + (size_t)t * a.out_stride;
#pragma unroll
    for (int u = 0; u < kTurns; ++u) {
      const int c = c0 + 1024 * u;
      if (c >= a.d) continue;
      if (a.vec) {
        store4(out + c, acc[u]);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) norm_store(out + c + i, acc[u][i]);
      }
    }
  }
}

template <typename T>
inline cudaError_t bank_combine_launch(const BankCombineArgs& a, cudaStream_t st, bool pdl) {
  const dim3 grid(a.T), block(256);
  if (a.d <= 1024) return launch_kernel(bank_combine_kernel<T, 1, 4>, grid, block, 0, st, pdl, a);
  if (a.d <= 2048) return launch_kernel(bank_combine_kernel<T, 2, 4>, grid, block, 0, st, pdl, a);
  return launch_kernel(bank_combine_kernel<T, 4, 2>, grid, block, 0, st, pdl, a);
}

}  // namespace swapmoe
