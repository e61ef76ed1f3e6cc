// Experts in 8-bit integers behind a router: out[t] = sum_j weights[t, j] * E_slot[t, j](x[t]),  E(x) = W_out act(W_in x).
//
// Pairs (token, choice) are laid out by slot, every slot's rows from a multiple of 32 on, so that the products (int8_gemm.cuh) walk token
// tiles of one slot each.  Where a pair comes to lie inside its slot hangs on the order of atomics; no result does, since every row is
// computed by itself and a token's choices are added in their order.
//   count (more than kBankDirectPairs pairs only): pairs per slot, and every CTA's share of a slot
//   gather: slot offsets, token tiles, rows of x8 with their scales to their places
//   product, activation in fp32; rows to 8 bits (quantize_rows.cuh); product; combine.
#pragma once
#include "int8_gemm.cuh"
#include "quantize_rows.cuh"

namespace swapmoe {

constexpr int kBankMaxSlots = 256;
constexpr int kBankThreads = 256;
constexpr int kBankMaxCtas = 512;               // CTAs of the count and gather kernels
constexpr int kBankDirectPairs = 4096;          // up to here every CTA of the gather kernel counts all pairs itself

struct BankArgs {
  const int8_t* x8;
  const float* x_scales;
  const int32_t* slots;
  const float* weights;
  int8_t* rows8;                // [rows, d]
  float* row_scales;
  int32_t *row_pair, *pair_row; // pair of a row (-1: none), row of a pair (-1: none)
  int32_t *counts, *cta_base;   // [S] zero between calls; [CTAs, S]
  TileDesc* tiles;
  int32_t* n_tiles;             // [0] tiles, [1] most rows of one, [2] rows with the slots' padding
  long long x_stride;
  int P, S, k, d, per_cta;      // pairs, pairs of a CTA
  int direct;
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

// Token tiles of one slot: equal heights, multiples of 32, of at most `cap` rows.
__device__ __forceinline__ int bank_tile_rows(int count, int cap) {
  const int n = (count + cap - 1) / cap;
  return n ? ((count + n - 1) / n + 31) & ~31 : 32;
}

__global__ void __launch_bounds__(kBankThreads) bank_gather_kernel(const __grid_constant__ BankArgs a) {
  __shared__ int s_count[kBankMaxSlots], s_at[kBankMaxSlots], s_off[kBankMaxSlots];
  __shared__ int s_row[kBankThreads];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int p0 = blockIdx.x * a.per_cta, p1 = min(a.P, p0 + a.per_cta);
  if (a.direct)
    for (int s = threadIdx.x; s < a.S; s += kBankThreads) s_count[s] = s_at[s] = 0;
  pdl_wait();
  pdl_trigger();
  __syncthreads();
  if (a.direct) {
    for (int p = threadIdx.x; p < a.P; p += kBankThreads) {
      const int s = bank_slot(a, p);
      if (s < 0) continue;
      atomicAdd(&s_count[s], 1);
      if (p < p0) atomicAdd(&s_at[s], 1);
    }
  } else {
    for (int s = threadIdx.x; s < a.S; s += kBankThreads) {
      s_count[s] = __ldcg(a.counts + s);
      s_at[s] = a.cta_base[(size_t)blockIdx.x * a.S + s];
    }
  }
  __syncthreads();
  if (warp == 0) {
    // slot offsets, and by the first CTA the list of tiles
    int most = 0;
    for (int s = lane; s < a.S; s += 32) most = max(most, s_count[s]);
    most = __reduce_max_sync(0xffffffffu, most);
    const int cap = most > 128 ? 256 : most > 64 ? 128 : 64;
    int row0 = 0, tile0 = 0;
    for (int s0 = 0; s0 < a.S; s0 += 32) {
      const int s = s0 + lane, count = s < a.S ? s_count[s] : 0;
      const int padded = (count + 31) & ~31, n = (count + cap - 1) / cap, height = bank_tile_rows(count, cap);
      const int used = (count + height - 1) / height;         // (heights are rounded up: the last tile may have become empty)
      int rows = padded, tiles = used;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, rows, o), v = __shfl_up_sync(0xffffffffu, tiles, o);
        if (lane >= o) { rows += u; tiles += v; }
      }
      (void)n;
      const int off = row0 + rows - padded;
      if (s < a.S) s_off[s] = off;
      if (blockIdx.x == 0) {
        for (int i = 0; i < used; ++i) {
          TileDesc td;
          td.phys = td.slot = s; td.row0 = off + i * height; td.rows = min(height, count - i * height);
          a.tiles[tile0 + tiles - used + i] = td;
        }
        for (int r = count; r < padded; ++r) a.row_pair[off + r] = -1;
      }
      row0 += __shfl_sync(0xffffffffu, rows, 31);
      tile0 += __shfl_sync(0xffffffffu, tiles, 31);
    }
    if (blockIdx.x == 0 && lane == 0) { a.n_tiles[0] = tile0; a.n_tiles[1] = cap; a.n_tiles[2] = row0; }
  }
  __syncthreads();
  for (int b = p0; b < p1; b += kBankThreads) {
    const int p = b + threadIdx.x, n = min(kBankThreads, p1 - b);
    int row = -1;
    if (p < p1) {
      const int s = bank_slot(a, p);
      if (s >= 0) {
        row = s_off[s] + atomicAdd(&s_at[s], 1);
        a.row_pair[row] = p;
        a.row_scales[row] = a.x_scales[p / a.k];
      }
      a.pair_row[p] = row;
    }
    s_row[threadIdx.x] = row;
    __syncthreads();
    for (int i = warp; i < n; i += kBankThreads / 32) {
      const int to = s_row[i];
      if (to < 0) continue;
      const uint4* src = reinterpret_cast<const uint4*>(a.x8 + (size_t)((b + i) / a.k) * a.x_stride);
      uint4* dst = reinterpret_cast<uint4*>(a.rows8 + (size_t)to * a.d);
      for (int c = lane; c < a.d / 16; c += 32) dst[c] = src[c];
    }
    __syncthreads();
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

template <typename T>
__global__ void __launch_bounds__(256) bank_combine_kernel(const __grid_constant__ BankCombineArgs a) {
  pdl_wait();
  pdl_trigger();
  if (blockIdx.x == 0 && blockIdx.y == 0)
    for (int s = threadIdx.x; s < a.S; s += 256) a.counts[s] = 0;     // for the next call
  const int t = blockIdx.x, c = (blockIdx.y * 256 + threadIdx.x) * 4;
  if (c >= a.d) return;
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
  for (int j = 0; j < a.k; ++j) {
    const int row = a.pair_row[t * a.k + j];
    if (row < 0) continue;
    const float w = a.weights[t * a.k + j];
    float v[4];
    load4(a.y + (size_t)row * a.d + c, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] = fmaf(w, v[i], acc[i]);
  }
  T* out = static_cast<T*>(a.out) + (size_t)t * a.out_stride + c;
  if (a.vec) {
    store4(out, acc);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) norm_store(out + i, acc[i]);
  }
}

}  // namespace swapmoe
