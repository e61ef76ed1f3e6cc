// Products of 8-bit integers for few tokens, where the weights' bytes are all there is to move.
//
// Warp-level mma (m16n8k32, int32 sums) on operands that go from global memory straight to registers: a lane's 16 bytes of a weight row are
// the operands of two mma, which contract the columns in an order of their own, the same for weights and tokens.  Sixteen weight rows belong to a
// CTA, whose eight warps split the contraction in turns of 64 columns, so that a row's loads follow one another through memory and the whole matrix
// is on its way at once; their sums meet in shared memory.  Against a ring of TMA stages with tensor memory behind it a call has no barriers to
// set up, no tensor memory to take and no ring to fill.
//
// With experts (up to 64 pairs of token and choice) the same in two launches, whose CTAs serve whole tokens of up to 16 pairs each: the first takes
// the rows of W_in of every slot that its tokens ask for (SwiGLU: both products of sixteen hidden units), applies the activation and leaves h in fp32
// with the largest magnitude of every 16 values; the second takes rows of W_out, fetched before the first has finished, and its tokens' h to 8 bits
// in shared memory, and adds a token's choices in their order.
// 1 to 8 tokens, 1024 x 1024 2.4 us; experts of 1024 x 512, 3 tokens of two choices 7.9 us, 32 pairs 14.7 (five launches 24).
#pragma once
#include "quantize_rows.cuh"

namespace swapmoe {

constexpr int kStreamThreads = 256;
constexpr int kStreamWarps = kStreamThreads / 32;
constexpr int kStreamTurn = kStreamWarps * 64;                // columns that a CTA's warps take in one turn
constexpr int kStreamPairs = 64;                              // pairs of a call
constexpr int kStreamMaxPairs = 16;                           // pairs of a CTA's tokens

__device__ __forceinline__ void mma_int8(int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The first `left` of 16 bytes (aligned), zeros behind them; weights are read once and not kept in L1.
template <bool kOnce>
__device__ __forceinline__ uint4 load_bytes16(const int8_t* p, int left) {
  uint4 v = make_uint4(0u, 0u, 0u, 0u);
  if (left >= 16) {
    if (kOnce) asm volatile("ld.global.nc.L1::no_allocate.L2::256B.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    else v = *reinterpret_cast<const uint4*>(p);
  } else if (left > 0) {
    uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 15; ++i)
      if (i < left) w[i >> 2] |= (uint32_t)(uint8_t)p[i] << (8 * (i & 3));
    v = make_uint4(w[0], w[1], w[2], w[3]);
  }
  return v;
}

// A warp's share of rows x tokens: kM tiles of sixteen weight rows, kN tiles of eight tokens, kBatch turns of weights in registers.
// Lane l holds rows l / 4 and l / 4 + 8 of a tile and token l / 4 of the eight, columns 16 (l % 4) ... + 15 of the turn's 64.
template <int kM, int kN, int kBatch>
struct StreamTile {
  int acc[kM][kN][4];
  uint4 w[kBatch][kM][2];

  // rows[m][h]: this lane's two weight rows of a tile (nullptr: none), from column c0 on, `turn` columns from one of the warp's turns to the next
  __device__ __forceinline__ void fetch(const int8_t* const (&rows)[kM][2], int c0, int turn, int K) {
#pragma unroll
    for (int b = 0; b < kBatch; ++b)
#pragma unroll
      for (int m = 0; m < kM; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int c = c0 + b * turn;
          w[b][m][h] = load_bytes16<true>(rows[m][h] + c, rows[m][h] != nullptr ? K - c : 0);
        }
  }
  // The warp's share of the contraction, from column c0 on.  tokens(n, c): 16 columns of this lane's token of tile n from column c on.
  // fetched: the first batch is in registers already.  used: tiles of tokens that hold some (mma's rate for 8-bit integers is low).
  template <typename Tokens>
  __device__ __forceinline__ void run(const int8_t* const (&rows)[kM][2], Tokens tokens, int used, int c0, int turn, int K, bool fetched) {
#pragma unroll
    for (int m = 0; m < kM; ++m)
#pragma unroll
      for (int n = 0; n < kN; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[m][n][i] = 0;
    const int own = 16 * (threadIdx.x & 3);
    for (; c0 - own < K; c0 += kBatch * turn) {
      if (!fetched) fetch(rows, c0, turn, K);
      fetched = false;
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        const int c = c0 + b * turn;
        if (c - own < K) {                                   // the same for the warp
#pragma unroll
          for (int n = 0; n < kN; ++n) {
            if (kN > 1 && n >= used) break;
            const uint4 x = tokens(n, c);
#pragma unroll
            for (int m = 0; m < kM; ++m) {
              mma_int8(acc[m][n], w[b][m][0].x, w[b][m][1].x, w[b][m][0].y, w[b][m][1].y, x.x, x.y);
              mma_int8(acc[m][n], w[b][m][0].z, w[b][m][1].z, w[b][m][0].w, w[b][m][1].w, x.z, x.w);
            }
          }
        }
      }
    }
  }
  // sums of the warps: part[warp][m][token][row]
  __device__ __forceinline__ void put(int* part) const {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int m = 0; m < kM; ++m)
#pragma unroll
      for (int n = 0; n < kN; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          part[((warp * kM + m) * kN * 8 + n * 8 + 2 * (lane & 3) + (i & 1)) * 16 + (lane >> 2) + 8 * (i >> 1)] = acc[m][n][i];
  }
  // of `warps` warps from warp w0 on
  static __device__ __forceinline__ int sum(const int* part, int m, int token, int row, int w0, int warps) {
    int v = 0;
#pragma unroll 4
    for (int w = w0; w < w0 + warps; ++w) v += part[((w * kM + m) * kN * 8 + token) * 16 + row];
    return v;
  }
};
// The first column of a lane where all warps of the CTA share a contraction.
__device__ __forceinline__ int stream_column() { return (threadIdx.x >> 5) * 64 + 16 * (threadIdx.x & 3); }

// ------------------------------------------------------------------ a whole matrix
struct I8StreamArgs {
  const int8_t *x, *w;
  const float *x_scales, *w_scales, *bias;
  void* out;
  long long x_stride, w_stride, out_stride;
  int T, K, N;                  // T: up to kStreamTokens
};
constexpr int kStreamTokens = 8;

template <typename T>
__global__ void __launch_bounds__(kStreamThreads) int8_stream_kernel(const __grid_constant__ I8StreamArgs a) {
  typedef StreamTile<1, 1, 4> Tile;
  __shared__ int s_part[kStreamWarps * 8 * 16];
  const int lane = threadIdx.x & 31, n0 = blockIdx.x * 16;
  const int8_t* rows[1][2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int n = n0 + (lane >> 2) + 8 * h;
    rows[0][h] = n < a.N ? a.w + (size_t)n * a.w_stride : nullptr;
  }
  const int t = lane >> 2;
  const int8_t* x = t < a.T ? a.x + (size_t)t * a.x_stride : nullptr;
  Tile tile;
  pdl_wait();
  pdl_trigger();
  tile.run(rows, [&](int, int c) { return load_bytes16<false>(x + c, x != nullptr ? a.K - c : 0); }, 1, stream_column(), kStreamTurn, a.K, false);
  tile.put(s_part);
  __syncthreads();
  const int i = threadIdx.x, token = i >> 4, r = i & 15, n = n0 + r;
  if (token >= a.T || n >= a.N) return;
  const float f = (float)Tile::sum(s_part, 0, token, r, 0, kStreamWarps) * a.w_scales[n], bias = a.bias != nullptr ? a.bias[n] : 0.f;
  norm_store(static_cast<T*>(a.out) + (size_t)token * a.out_stride + n, fmaf(f, a.x_scales[token], bias));
}

// ------------------------------------------------------------------ experts
struct BankStreamArgs {
  const int8_t *x8, *w_in, *w_out;
  const float *x_scales, *in_scales, *out_scales, *weights;
  const int32_t* slots;
  float *h, *largest;           // [P, F], [P, F / 16]
  void* out;
  long long x_stride, out_stride;
  int P, S, k, d, F, T;
  int in_tokens, out_tokens;    // tokens of a CTA of the two kernels
};

// The share of `tokens` tokens that belongs to this CTA (blockIdx.z).
template <typename T>
__device__ __forceinline__ BankStreamArgs bank_share(const BankStreamArgs& whole, int tokens) {
  BankStreamArgs a = whole;
  const int t0 = (int)blockIdx.z * tokens;
  a.T = min(tokens, a.T - t0); a.P = a.T * a.k;
  a.x8 += (size_t)t0 * a.x_stride; a.x_scales += t0; a.slots += t0 * a.k; a.weights += t0 * a.k;
  a.h += (size_t)t0 * a.k * a.F; a.largest += (size_t)t0 * a.k * (a.F / 16);
  a.out = static_cast<T*>(a.out) + (size_t)t0 * a.out_stride;
  return a;
}

// The pairs by the slots they ask for: slots in the order of their first pair.
struct BankLists {
  int n;                               // slots
  int slot[kStreamMaxPairs], start[kStreamMaxPairs + 1], pair[kStreamMaxPairs];
};
__device__ __forceinline__ void bank_lists(const BankStreamArgs& a, BankLists* l) {       // by one warp
  const int lane = threadIdx.x & 31;
  const int given = lane < a.P ? __ldcg(a.slots + lane) : -1;
  const bool ok = (unsigned)given < (unsigned)a.S;
  const unsigned same = __match_any_sync(0xffffffffu, ok ? given : -1);
  const bool leads = ok && (same & ((1u << lane) - 1u)) == 0;
  const unsigned leaders = __ballot_sync(0xffffffffu, leads);
  const int u = __popc(leaders & ((1u << lane) - 1u));
  // pairs of the slots in front
  int start = leads ? __popc(same) : 0;
  const int own = start;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, start, o);
    if (lane >= o) start += v;
  }
  if (lane == 31) l->start[__popc(leaders)] = start;
  start -= own;
  if (leads) { l->slot[u] = given; l->start[u] = start; }
  const int first = __shfl_sync(0xffffffffu, start, __ffs(same) - 1);
  if (ok) l->pair[first + __popc(same & ((1u << lane) - 1u))] = lane;
  if (lane == 0) l->n = __popc(leaders);
}

// h of sixteen hidden units of one slot for the pairs that the CTA's tokens have there.
template <bool kSwiglu, int kN>
__global__ void __launch_bounds__(kStreamThreads) bank_stream_in_kernel(const __grid_constant__ BankStreamArgs whole) {
  const BankStreamArgs a = bank_share<char>(whole, whole.in_tokens);
  constexpr int kM = kSwiglu ? 2 : 1;
  typedef StreamTile<kM, kN, 4 / kM> Tile;
  __shared__ int s_part[kStreamWarps * kM * kN * 8 * 16];
  __shared__ BankLists s_lists;
  const int lane = threadIdx.x & 31, f0 = blockIdx.x * 16;
  pdl_wait();
  pdl_trigger();
  if (threadIdx.x < 32) bank_lists(a, &s_lists);
  __syncthreads();
  if ((int)blockIdx.y >= s_lists.n) return;
  const int slot = s_lists.slot[blockIdx.y], start = s_lists.start[blockIdx.y], count = s_lists.start[blockIdx.y + 1] - start;
  Tile tile;
  const int8_t* rows[kM][2];
#pragma unroll
  for (int m = 0; m < kM; ++m)
#pragma unroll
    for (int h = 0; h < 2; ++h) rows[m][h] = a.w_in + (((size_t)slot * kM + m) * a.F + f0 + (lane >> 2) + 8 * h) * a.d;
  tile.fetch(rows, stream_column(), kStreamTurn, a.d);
  const int8_t* x[kN];
#pragma unroll
  for (int n = 0; n < kN; ++n) {
    const int i = n * 8 + (lane >> 2);
    x[n] = i < count ? a.x8 + (size_t)(s_lists.pair[start + i] / a.k) * a.x_stride : nullptr;
  }
  const int r = threadIdx.x & 15;
  const float* ws = a.in_scales + (size_t)slot * kM * a.F + f0 + r;
  const float w0 = ws[0], w1 = kSwiglu ? ws[a.F] : 0.f;
  tile.run(rows, [&](int n, int c) { return load_bytes16<false>(x[n] + c, x[n] != nullptr ? a.d - c : 0); }, (count + 7) / 8,
           stream_column(), kStreamTurn, a.d, true);
  tile.put(s_part);
  __syncthreads();
  for (int i0 = 0; i0 < count * 16; i0 += kStreamThreads) {
    const int t = (i0 + (int)threadIdx.x) >> 4;
    const bool mine = t < count;
    const int p = mine ? s_lists.pair[start + t] : 0;
    float h = 0.f;
    if (mine) {
      const float xs = a.x_scales[p / a.k];
      h = (float)Tile::sum(s_part, 0, t, r, 0, kStreamWarps) * w0 * xs;
      if constexpr (kSwiglu) h = silu(h) * ((float)Tile::sum(s_part, 1, t, r, 0, kStreamWarps) * w1 * xs);
      else h = h < 0.f ? 0.f : h;
      a.h[(size_t)p * a.F + f0 + r] = h;
    }
    float most = max_magnitude(0.f, h, 0.f);
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) most = max_magnitude(most, __shfl_xor_sync(0xffffffffu, most, o), 0.f);
    if (mine && r == 0) a.largest[(size_t)p * (a.F / 16) + blockIdx.x] = most;
  }
}

// Sixteen values of a row of h to 8 bits.
__device__ __forceinline__ uint4 quantize16(const float* h, float divisor, float inverse) {
  uint32_t b[4];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float v[8];
    uint32_t q[8];
    const float4 lo = __ldcg(reinterpret_cast<const float4*>(h + 8 * i)), hi = __ldcg(reinterpret_cast<const float4*>(h + 8 * i + 4));
    v[0] = lo.x; v[1] = lo.y; v[2] = lo.z; v[3] = lo.w; v[4] = hi.x; v[5] = hi.y; v[6] = hi.z; v[7] = hi.w;
    quotients8(v, divisor, inverse, q);
    b[2 * i] = pack_bytes(q); b[2 * i + 1] = pack_bytes(q + 4);
  }
  return make_uint4(b[0], b[1], b[2], b[3]);
}

// Sixteen channels of the result for the CTA's tokens.  The CTA's warps share the slots out among them: as many slots side by side as there are (up to
// all warps), the warps of a slot take turns of its columns.
constexpr int kBankOutThreads = 512;
constexpr int kBankOutWarps = kBankOutThreads / 32;
// Two rows that a warp reads side by side start half of the banks apart.
__host__ __device__ constexpr int bank_row_bytes(int F) { return (F + 127) / 128 * 128 + 64; }
constexpr int kBankOutRowBytes = 64 * 1024;                  // most shared memory for them
static_assert(kStreamMaxPairs * 16 <= kBankOutThreads && kStreamMaxPairs <= 32, "a thread per pair and channel, a lane per pair");

template <typename T, int kN>
__global__ void __launch_bounds__(kBankOutThreads) bank_stream_out_kernel(const __grid_constant__ BankStreamArgs whole) {
  const BankStreamArgs a = bank_share<T>(whole, whole.out_tokens);
  typedef StreamTile<1, kN, 4> Tile;
  __shared__ int s_part[kBankOutWarps * kN * 8 * 16];
  __shared__ float s_y[kStreamMaxPairs * 16];
  __shared__ float s_scale[kStreamMaxPairs], s_inverse[kStreamMaxPairs], s_divisor[kStreamMaxPairs], s_weight[kStreamMaxPairs];
  __shared__ BankLists s_lists;
  extern __shared__ __align__(16) int8_t s_rows[];           // the pairs' rows in 8 bits, bank_row_bytes apart
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n0 = (int)blockIdx.x * 16, r = threadIdx.x & 15;
  // slots and weights are older than the kernel in front: the first are fetched while it runs
  if (warp == 0) bank_lists(a, &s_lists);
  if (warp == 1 && lane < a.P) s_weight[lane] = (unsigned)__ldcg(a.slots + lane) < (unsigned)a.S ? __ldcg(a.weights + lane) : 0.f;
  if (threadIdx.x < kStreamMaxPairs * 16) s_y[threadIdx.x] = 0.f;
  __syncthreads();
  const int n_slots = s_lists.n, n_pairs = s_lists.start[n_slots];
  int side = 1;                                              // slots side by side
  while (side < n_slots && side < kBankOutWarps) side *= 2;
  const int warps = kBankOutWarps / side, turn = warps * 64, mine = warp / warps, c0 = (warp - mine * warps) * 64 + 16 * (lane & 3);
  Tile tile;
  const int8_t* rows[1][2];
  auto fetch = [&](int u) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      rows[0][h] = u < n_slots ? a.w_out + ((size_t)s_lists.slot[u] * a.d + n0 + (lane >> 2) + 8 * h) * a.F : nullptr;
    tile.fetch(rows, c0, turn, a.F);
  };
  fetch(mine);
  // this thread's pair and channel at the end
  const int own = threadIdx.x >> 4;
  int own_slot = 0;
  for (int u = 1; u < n_slots; ++u) own_slot += s_lists.start[u] <= own ? 1 : 0;
  const float out_scale = own < n_pairs ? a.out_scales[(size_t)s_lists.slot[own_slot] * a.d + n0 + r] : 0.f;
  pdl_wait();
  pdl_trigger();
  // scales of the rows of h, a pair per warp
  for (int i = warp; i < n_pairs; i += kBankOutWarps) {
    const int p = s_lists.pair[i];
    float most = 0.f;
    for (int g = lane; g < a.F / 16; g += 32) most = max_magnitude(most, __ldcg(a.largest + (size_t)p * (a.F / 16) + g), 0.f);
    most = warp_largest(most);
    if (lane == 0) {
      const float q = quantize_divisor(most);
      s_divisor[i] = q; s_inverse[i] = __frcp_rn(q); s_scale[i] = most == 0.f ? 0.f : q;
    }
  }
  __syncthreads();
  const int row_bytes = bank_row_bytes(a.F);
  for (int i = threadIdx.x; i < n_pairs * (a.F / 16); i += kBankOutThreads) {
    const int p = i / (a.F / 16), c = (i - p * (a.F / 16)) * 16;
    *reinterpret_cast<uint4*>(s_rows + p * row_bytes + c) = quantize16(a.h + (size_t)s_lists.pair[p] * a.F + c, s_divisor[p], s_inverse[p]);
  }
  __syncthreads();
  for (int u0 = 0; u0 < n_slots; u0 += side) {
    const int u = u0 + mine;
    if (u0 > 0) fetch(u);
    const int start = u < n_slots ? s_lists.start[u] : 0, count = u < n_slots ? s_lists.start[u + 1] - start : 0;
    tile.run(rows, [&](int n, int c) {
      const int i = n * 8 + (lane >> 2);
      return i < count && c < a.F ? *reinterpret_cast<const uint4*>(s_rows + (start + i) * row_bytes + c) : make_uint4(0u, 0u, 0u, 0u);
    }, (count + 7) / 8, c0, turn, count > 0 ? a.F : 0, true);
    tile.put(s_part);
    __syncthreads();
    if (own < n_pairs && own_slot >= u0 && own_slot < u0 + side)
      s_y[s_lists.pair[own] * 16 + r] =
          (float)Tile::sum(s_part, 0, own - s_lists.start[own_slot], r, (own_slot - u0) * warps, warps) * out_scale * s_scale[own];
    __syncthreads();
  }
  for (int i = threadIdx.x; i < a.T * 16; i += kBankOutThreads) {
    const int t = i >> 4;
    float acc = 0.f;
    for (int j = 0; j < a.k; ++j) acc = fmaf(s_weight[t * a.k + j], s_y[(t * a.k + j) * 16 + r], acc);
    norm_store(static_cast<T*>(a.out) + (size_t)t * a.out_stride + n0 + r, acc);
  }
}

}  // namespace swapmoe
