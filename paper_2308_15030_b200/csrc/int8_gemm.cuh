// Products of 8-bit integers on CTA pairs, with a scale for each token and each channel:
//   C[t, n] = x_scales[t] * w_scales[n] * sum_k x8[t, k] * w8[n, k] (+ bias[n]).
// The sums are exact (int32; |sum| <= 2^14 K, K < 2^17); an epilogue turns them to fp32, scales them and rounds the result once.
//
// Bound by the tensor cores for many tokens and by the weights' bytes for few.  As in the grouped GEMM of bf16 layers (gemm_tc_pair.cuh)
// two SMs share a tile of 256 WEIGHT rows x up to 256 TOKENS through tcgen05 `cta_group::2`, here of kind::i8: a k-block is 128
// columns, the same 128 bytes a row that 64 bf16 values take, for the same tensor clocks and twice the products.  Weights are the MMA's
// rows, so tokens, whose number is ragged, are its columns, in steps of 32.  Roles in each CTA (640 threads): warp 0 = TMA
// producer, warp 1 = MMA issuer (even CTA only), warp 2 = TMEM allocation, warps 4-19 = epilogue of the CTA's own 128 weight rows, which
// overlaps the next tile's MMAs through two accumulators.  Sixteen warps, sixteen tokens at a time: what an epilogue does is a chain of
// instructions that wait for one another, and with short contractions it sets the pace: a round of 256 tokens takes 1.5 us at 512 columns without an
// epilogue and 3.2 with it, 2.6 and 4.0 at 1024, 10.7 and 11.5 at 4096.  No load uses cluster multicast.  Every mbarrier wait is
// bounded; the cluster barriers behind them and the allocation of tensor memory (a CTA has its SM to itself) are not.
// 8192 tokens, 4096 -> 14336: 288 to 302 us in a short graph, 3.2 to 3.3 POP/s (twice the rate of a bf16 library product: 3.3); calls back to back 336 to 345
// under the power cap, 2.8 POP/s (twice the library's there: 2.8).  61 tokens 13.6 us, 4.3 TB/s of weights.
#pragma once
#include "launch.cuh"
#include "pair_common.cuh"
#include "quantize_rows.cuh"

namespace swapmoe {

constexpr int kI8BK = 128;                                    // columns of a k-block: one 128-byte swizzle row
constexpr int kI8MaxK = (1 << 17) - 1;                        // 2^14 (2^17 - 1) < 2^31
enum { kI8Bf16 = 0, kI8F32 = 1, kI8Relu = 2, kI8Swiglu = 3 };

// A bounded wait of these kernels that gave up: flag and code of the wait, read by the host.
static __device__ int32_t g_int8_status[2];

struct I8GemmArgs {
  void* C;                  // [rows, ldc]
  const TileDesc* tiles;    // token tiles of the slots (nullptr: one matrix of T rows, tiles of `height` rows)
  const int32_t* n_tiles;   // [0] their number, [1] what they hold at most
  const float *x_scales, *w_scales, *bias;
  long long ldc;
  int32_t n_cols;           // columns of C
  int32_t n_col_tiles;      // weight tiles per slot (256 rows; SwiGLU 128 of either matrix)
  int32_t k_blocks;
  int32_t w_rows;           // weight rows per slot
  int32_t row_group;        // token tiles per scheduling group (see decode_tile)
  int32_t T, height;        // height: multiple of 32, up to 256
  int32_t direct;           // rows of C that the TMA unit cannot store: elements leave one by one (2: bf16 ones two by two)
  // 1: the kernel in front holds no tensor memory and has waited for all before it: pairs get ready while it runs.  2: and the list of
  // tiles and the weights are older than it: the first boxes of weights are requested too.
  int32_t early;
  int32_t* largest;         // [rows] largest magnitude of a row of hidden values, as its bits (ReLU, SwiGLU: zero before)
};

// (sum * w_scale) of two tokens to results: times the tokens' scales plus the bias in one rounding, as all forms of the product do it.
__device__ __forceinline__ void scaled2(float& a, float& b, float x0, float x1, float bias) {
  float u = bias, v = bias;
  fma2(u, v, a, b, x0, x1);
  a = u; b = v;
}

// What a k-block of a tile costs by the tile's tokens: its bytes, 256 weight rows and the tokens (4096 x 14336: a round of 128 tokens 10.5 us, of 256
// 13.4; eight slots of about 1000 rows, both products: tiles of up to 256 rows 1050 us, of about 128 1390).
__host__ __device__ constexpr int int8_tile_cost(int tokens) { return 256 + tokens; }

// Instruction descriptor: int8 x int8 -> int32, both operands K-major, M x N tile.
__host__ __device__ constexpr uint32_t make_idesc_int8(int M, int N) {
  return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

namespace ptx {
// All of this thread's stores but the last one have read their shared memory.
__device__ __forceinline__ void tma_store_wait_read_but_one() { asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory"); }
__device__ __forceinline__ void umma_int8_pair(uint32_t tmem_d, uint64_t desc_a, uint64_t desc_b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n}\n" ::"r"(tmem_d),
      "l"(desc_a), "l"(desc_b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Sixteen lanes x sixteen columns of tensor memory as the fragments of 8 x 8 matrices: v[4 j + 2 i + e] is lane l / 4 + 8 i, column 8 j + 2 (l % 4) + e.
__device__ __forceinline__ void tmem_ld_fragments(uint32_t taddr, uint32_t* v) {
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
               : "r"(taddr)
               : "memory");
}
// Loads out of tensor memory have arrived in v: what uses it stays behind this.
__device__ __forceinline__ void tmem_ld_wait_for(uint32_t (&v)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]), "+r"(v[10]),
                 "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15])
               :
               : "memory");
}
// Four 8 x 8 matrices of 16-bit values, transposed; lane 8 m + r has the place of row r of matrix m.
__device__ __forceinline__ void store_matrices_transposed(uint32_t at, uint32_t m0, uint32_t m1, uint32_t m2, uint32_t m3) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(m0), "r"(m1), "r"(m2), "r"(m3) : "memory");
}
}  // namespace ptx

constexpr int kI8EpiWarps = 16;
constexpr int kI8EpiParts = kI8EpiWarps / 4;                  // warps that share a quarter of tensor memory
constexpr int kI8Chunk = 16;                                  // tokens an epilogue warp takes at once
constexpr int kI8Threads = 128 + 32 * kI8EpiWarps;
// staging of an epilogue warp: two boxes of 16 tokens x 32 columns (SwiGLU 16), so that one is filled while the other leaves
__host__ __device__ constexpr int int8_box_bytes(int epi) { return epi == kI8F32 || epi == kI8Relu ? 2048 : 1024; }
// the ring takes what that leaves: stages of 256 / 128 / 64 tokens 6 / 8 / 9, where boxes are of 2 KB 5 / 6 / 8
__host__ __device__ constexpr int int8_ring_bytes(int epi) { return (int8_box_bytes(epi) == 2048 ? 5 : 6) * (kPairABytes + kPairBBytes); }
__host__ __device__ constexpr int int8_stages(int epi, int max_tokens) {
  return int8_box_bytes(epi) == 2048 ? (max_tokens > 128 ? 5 : max_tokens > 64 ? 6 : 8) : max_tokens > 128 ? 6 : max_tokens > 64 ? 8 : 9;
}
// ... and the scales of a warp's tokens
__host__ __device__ constexpr int int8_smem_bytes(int epi) { return int8_ring_bytes(epi) + 2048 + kI8EpiWarps * (2 * int8_box_bytes(epi) + 4 * kI8Chunk); }
static_assert(int8_smem_bytes(kI8F32) <= 227 * 1024 && int8_smem_bytes(kI8Bf16) <= 227 * 1024, "what a CTA may have");
static_assert(!fits_beside_cluster(int8_smem_bytes(kI8F32)) && !fits_beside_cluster(int8_smem_bytes(kI8Bf16)), "tensor memory is not shared with clusters");
static_assert(int8_stages(kI8F32, 64) * (kPairABytes + 32 * kI8BK) <= int8_ring_bytes(kI8F32) && int8_stages(kI8Bf16, 64) <= kPairMaxStages, "stages fit");

template <int EPI>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kI8Threads, 1)
int8_gemm_pair_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX128,
                      const __grid_constant__ CUtensorMap tmX64, const __grid_constant__ CUtensorMap tmX32,
                      const __grid_constant__ CUtensorMap tmX16, const __grid_constant__ CUtensorMap tmC,
                      const __grid_constant__ I8GemmArgs a) {
  constexpr bool kSwiglu = EPI == kI8Swiglu;
  constexpr uint32_t kTmemCols = 2 * kPairTokens;             // two accumulator sets

  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  unsigned char* sW = smem;                                   // [stages][128][128] int8
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + int8_ring_bytes(EPI));
  uint64_t* full = bars;                    // [stages]  used in the even CTA
  uint64_t* empty = bars + kPairMaxStages;  // [stages]  one in each CTA (the commit reaches both)
  uint64_t* acc_full = bars + 2 * kPairMaxStages;  // [2]  one in each CTA
  uint64_t* acc_empty = acc_full + 2;       // [2]       used in the even CTA
  uint64_t* tmem_ready = acc_empty + 2;     // used in the even CTA: the odd one has allocated its half
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(tmem_ready + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int32_t* const status = g_int8_status;

  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;   // warp-uniform
  const uint32_t rank = ptx::cluster_ctarank();               // 0: issues the MMAs
  const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;

  if (threadIdx.x == 0) {
    ptx::mbar_init(tmem_ready, 1);
    for (int s = 0; s < kPairMaxStages; ++s) { ptx::mbar_init(&full[s], 1); ptx::mbar_init(&empty[s], 1); }
    for (int b = 0; b < 2; ++b) { ptx::mbar_init(&acc_full[b], 1); ptx::mbar_init(&acc_empty[b], 2 * kI8EpiWarps); }
    *abort_flag = 0;
    ptx::fence_barrier_init();
    ptx::prefetch_tmap(&tmW);
    ptx::prefetch_tmap(&tmX128);
  }
  // Operands and the list of tiles come from the kernels in front; tensor memory is taken only when those have let go of theirs, and
  // the next kernel's CTAs are let in only when these have got it.
  if (a.early == 0) pdl_wait();
  ptx::cluster_start_sync();                                  // both CTAs run and their barriers are initialised
  uint32_t tmem_base = 0;
  if (warp != 0 && warp != 3) {
    if (warp == 2) {
      ptx::tmem_alloc_pair(tmem_slot, kTmemCols);             // issued in both CTAs: one allocation for the pair
      ptx::tmem_relinquish_pair();
      if (rank == 1 && lane == 0) ptx::mbar_arrive_release_cluster(ptx::map_to_cta(ptx::smem_u32(tmem_ready), 0u));
    }
    ptx::tc_fence_before();
    asm volatile("bar.sync 1, %0;" ::"n"(kI8Threads - 64) : "memory");
    ptx::tc_fence_after();
    tmem_base = *tmem_slot;
    if (a.early != 0) pdl_wait();
    pdl_trigger();
  } else if (a.early == 1 || warp == 3) {
    if (a.early != 0) pdl_wait();
  }                                                           // (the producer of early weights waits behind them)

  // tokens of a tile in the MMA's columns; each CTA stages half of them
  const bool listed = a.tiles != nullptr;
  const int n_row_tiles = listed ? __ldcg(a.n_tiles) : (a.T + a.height - 1) / a.height;
  const int max_tokens = listed ? __ldcg(a.n_tiles + 1) : a.height > 128 ? 256 : a.height > 64 ? 128 : 64;
  auto tile_cols = [&](const TileDesc& td) { return listed ? (td.rows + kPairTokenStep - 1) & ~(kPairTokenStep - 1) : a.height; };
  auto tile_at = [&](int rt) {
    TileDesc td;
    if (listed) {                                              // (the list holds one entry at least)
      const int4 raw = __ldcg(reinterpret_cast<const int4*>(a.tiles + rt));
      td.phys = raw.x; td.row0 = raw.y; td.rows = raw.z; td.slot = raw.w;
    } else {
      td.phys = td.slot = 0; td.row0 = rt * a.height; td.rows = min(a.height, a.T - td.row0);
    }
    return td;
  };
  const int total = n_row_tiles * a.n_col_tiles;
  auto at_step = [&](int t) {                                  // the tile of step t (behind the last step: any)
    int rt = 0, ct_unused = 0;
    if (t < total) decode_tile(t, n_row_tiles, a.n_col_tiles, a.row_group, &rt, &ct_unused);
    return tile_at(rt);
  };
  const int n_stages = int8_stages(EPI, max_tokens), x_bytes = max_tokens / 2 * kI8BK;
  unsigned char* sX = smem + n_stages * kPairABytes;          // [stages][max_tokens / 2][128] int8

  if (warp == 0) {
    // ------------------------------------------------------------------ TMA producer (both CTAs)
    const uint32_t full0 = ptx::map_to_cta(ptx::smem_u32(full), 0u);
    auto load_w = [&](int stage, int kb, int phys, int ct) {
      const uint32_t bar = full0 + 8u * (uint32_t)stage;
      if (kSwiglu)
        ptx::tma_load_5d_pair(sW + stage * kPairABytes, &tmW, bar, kb * kI8BK, 0, 0, ct * 8 + (int)rank * 4, phys);
      else
        ptx::tma_load_2d_pair(sW + stage * kPairABytes, &tmW, bar, kb * kI8BK, phys * a.w_rows + ct * 2 * kTcBM + (int)rank * kTcBM);
    };
    int pre = 0;                                              // k-blocks of the first tile whose weights are on their way
    if (a.early == 2) {
      if (pair < total) {
        int rt, ct;
        decode_tile(pair, n_row_tiles, a.n_col_tiles, a.row_group, &rt, &ct);
        const TileDesc td = tile_at(rt);
        pre = min(a.k_blocks, n_stages);
        for (int kb = 0; kb < pre; ++kb) {
          if (ptx::elect_one()) {
            if (rank == 0) ptx::mbar_expect_tx(&full[kb], (uint32_t)(2 * kPairABytes + tile_cols(td) * kI8BK));
            load_w(kb, kb, td.phys, ct);
          }
          __syncwarp();
        }
      }
      pdl_wait();
    }
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int t = pair; t < total && ok; t += n_pairs) {
      int rt, ct;
      decode_tile(t, n_row_tiles, a.n_col_tiles, a.row_group, &rt, &ct);
      const TileDesc td = tile_at(rt);
      const int cols = tile_cols(td), half = cols / 2;         // half: a multiple of 16, at most 128
      const int xrow = td.row0 + (int)rank * half;
      const uint32_t bytes = (uint32_t)(2 * kPairABytes + cols * kI8BK);
      for (int kb = 0; kb < a.k_blocks; ++kb) {
        const bool early = t == pair && kb < pre;              // armed and weights requested above
        if (!early) {
          ok = warp_wait<true>(&empty[stage], phase ^ 1u, abort_flag, status, 31);
          if (!ok) break;
        }
        if (ptx::elect_one()) {
          if (rank == 0 && !early) ptx::mbar_expect_tx(&full[stage], bytes);
          const uint32_t bar = full0 + 8u * (uint32_t)stage;
          unsigned char* dst = sX + stage * x_bytes;
          if (!early) load_w(stage, kb, td.phys, ct);
          if (half == 128) {
            ptx::tma_load_2d_pair(dst, &tmX128, bar, kb * kI8BK, xrow);
          } else {                                             // boxes of 64, 32 and 16 rows
            if (half & 64) ptx::tma_load_2d_pair(dst, &tmX64, bar, kb * kI8BK, xrow);
            if (half & 32) ptx::tma_load_2d_pair(dst + (half & 64) * 128, &tmX32, bar, kb * kI8BK, xrow + (half & 64));
            if (half & 16) ptx::tma_load_2d_pair(dst + (half & 96) * 128, &tmX16, bar, kb * kI8BK, xrow + (half & 96));
          }
        }
        __syncwarp();
        if (++stage == n_stages) { stage = 0; phase ^= 1u; }
      }
    }
    if (!ok) {
      // Give copies that are still in flight time to land before shared memory is released.
      const uint64_t t0 = ptx::globaltimer_ns();
      while (ptx::globaltimer_ns() - t0 < 2000000ull) __nanosleep(1000);
    }
  } else if (warp == 1) {
    if (rank == 0) {
      // ------------------------------------------------------------------ MMA issuer (even CTA, for the pair)
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 0;
      bool ok = warp_wait<true>(tmem_ready, 0u, abort_flag, status, 35);
      ptx::tc_fence_after();
      TileDesc ahead = at_step(pair);                          // (a tile's descriptor comes while the one before it is multiplied)
      for (int t = pair; t < total && ok; t += n_pairs) {
        const uint32_t idesc = make_idesc_int8(2 * kTcBM, tile_cols(ahead));
        ahead = at_step(t + n_pairs);
        ok = warp_wait<true>(&acc_empty[acc], acc_phase ^ 1u, abort_flag, status, 32);
        if (!ok) break;
        ptx::tc_fence_after();
        const uint32_t tmem_d = tmem_base + (uint32_t)(acc * kPairTokens);
        for (int kb = 0; kb < a.k_blocks; ++kb) {
          ok = warp_wait<true>(&full[stage], phase, abort_flag, status, 33);
          if (!ok) break;
          ptx::tc_fence_after();
          const uint64_t dw = make_kmajor_sw128_desc(ptx::smem_u32(sW + stage * kPairABytes));
          const uint64_t dx = make_kmajor_sw128_desc(ptx::smem_u32(sX + stage * x_bytes));
          if (ptx::elect_one()) {
#pragma unroll
            for (int k = 0; k < 4; ++k)                        // 32 columns each
              ptx::umma_int8_pair(tmem_d, dw + (uint64_t)(2 * k), dx + (uint64_t)(2 * k), idesc, (kb > 0 || k > 0) ? 1u : 0u);
            ptx::umma_commit_pair(&empty[stage]);   // frees the stage in both CTAs once these MMAs have read it
            if (kb + 1 == a.k_blocks) ptx::umma_commit_pair(&acc_full[acc]);    // accumulator complete, in both CTAs
          }
          __syncwarp();
          if (++stage == n_stages) { stage = 0; phase ^= 1u; }
        }
        if (!ok) break;
        if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
      }
    }
  } else if (warp >= 4) {
    // -------------------------------------------------------------------- epilogue (own 128 weight rows)
    const int q = warp & 3;                    // TMEM lane quarter this warp may read
    const int part = (warp - 4) >> 2;          // the warps of a quarter take turns with the chunks of tokens
    // bf16 and SwiGLU: a lane holds rows l / 4 + 8 i + 16 h of the warp's 32 (SwiGLU: unit l / 4 + 8 i of matrix h) and tokens
    // 8 j + 2 (l % 4) + e of a chunk's 16, v[8 h + 4 j + 2 i + e]; else lane l holds row l and all sixteen.
    constexpr bool kFragments = EPI == kI8Bf16 || kSwiglu;
    constexpr int kRows = kFragments ? 4 : 1;  // weight rows of a lane
    const int row8 = lane >> 2, two = 2 * (lane & 3), hi = lane >> 4;
    constexpr int kBox = int8_box_bytes(EPI);
    unsigned char* const stg0 = smem + int8_ring_bytes(EPI) + 1024 + (warp - 4) * 2 * kBox;
    float* s_scale = reinterpret_cast<float*>(smem + int8_ring_bytes(EPI) + 1024 + 2 * kI8EpiWarps * kBox) + (warp - 4) * kI8Chunk;
    int box = 0;                               // which of the two is filled next
    const uint32_t acc_empty0 = ptx::map_to_cta(ptx::smem_u32(acc_empty), 0u);
    int acc = 0;
    uint32_t acc_phase = 0;
    bool ok = true;
    // What a tile needs from memory comes while the tiles before it are worked on: its descriptor two steps ahead, its scales one.
    struct Scales { float w[kRows], bias[EPI == kI8Bf16 ? 4 : 1], token; };
    auto first_col = [&](int t) {                              // of this warp's output columns (32; SwiGLU 16)
      int rt = 0, ct = 0;
      if (t < total) decode_tile(t, n_row_tiles, a.n_col_tiles, a.row_group, &rt, &ct);
      return kSwiglu ? (ct * 8 + (int)rank * 4 + q) * 16 : ct * 2 * kTcBM + (int)rank * kTcBM + q * 32;
    };
    auto token_scale = [&](const TileDesc& td, int c) {
      const int token = kI8Chunk * c + (lane & (kI8Chunk - 1));
      return token < td.rows ? a.x_scales[td.row0 + token] : 0.f;
    };
    auto scales_of = [&](int t, const TileDesc& td) {
      Scales s = {};
      const int col0 = first_col(t);
      if (t >= total) return s;
      s.token = token_scale(td, part);
#pragma unroll
      for (int r = 0; r < kRows; ++r) {                        // r = 2 h + i
        const int col = kSwiglu ? col0 + 8 * (r & 1) + row8 : kFragments ? col0 + 8 * r + row8 : col0 + lane;
        if (col >= a.n_cols) continue;
        s.w[r] = kSwiglu ? a.w_scales[((size_t)td.phys * 2 + (r >> 1)) * a.n_cols + col] : a.w_scales[(size_t)td.phys * a.w_rows + col];
        if (!kSwiglu && a.bias != nullptr) s.bias[r] = a.bias[col];
      }
      return s;
    };
    TileDesc td_next = at_step(pair), td_after = at_step(pair + n_pairs);
    Scales s_next = scales_of(pair, td_next);
    for (int t = pair; t < total && ok; t += n_pairs) {
      const TileDesc td = td_next;
      const Scales scales = s_next;
      float next = scales.token;                             // scales of the tokens, a chunk ahead
      td_next = td_after;
      td_after = at_step(t + 2 * n_pairs);
      s_next = scales_of(t + n_pairs, td_next);
      const int col0 = first_col(t), col = col0 + lane;
      const bool col_ok = col0 < a.n_cols;
      const int last = (td.rows - 1) / kI8Chunk;             // the tile's last chunk
      const int my_last = part <= last ? last - (last - part) % kI8EpiParts : -1;              // this warp's last one (-1: none)
      ok = warp_wait<true>(&acc_full[acc], acc_phase, abort_flag, status, 34);
      if (!ok) break;
      ptx::tc_fence_after();
      const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(acc * kPairTokens);
      auto release = [&]() {
        // last read of this accumulator: one arrival per warp on the even CTA's barrier, all warps' hand it back to the MMA issuer
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive_cluster(acc_empty0 + 8u * (uint32_t)acc);
      };
      uint32_t v[kI8Chunk];
      auto load = [&](int first) {                             // (a load of the whole warp)
        if (kFragments) {
          ptx::tmem_ld_fragments(taddr + (uint32_t)first, v);
          ptx::tmem_ld_fragments(taddr + (16u << 16) + (uint32_t)first, v + 8);
        } else {
          ptx::tmem_ld16(taddr + (uint32_t)first, v);
        }
      };
      __syncwarp();
      if (my_last < 0) release();
      else load(kI8Chunk * part);
#pragma unroll 1
      for (int c = part; c <= last; c += kI8EpiParts) {
        const int t0 = kI8Chunk * c, left = td.rows - t0;    // valid tokens of this chunk (may exceed its size)
        __syncwarp();                                        // the scales of the chunk before have been read
        if (lane < kI8Chunk) s_scale[lane] = next;
        next = token_scale(td, c + kI8EpiParts);
        ptx::tmem_ld_wait_for(v);
        float f[kI8Chunk];
#pragma unroll
        for (int j = 0; j < kI8Chunk; ++j) f[j] = (float)(int)v[j];
        __syncwarp();
        // the next chunk comes out of tensor memory while this one is worked on
        if (c == my_last) release();
        else load(t0 + kI8Chunk * kI8EpiParts);
        if (!col_ok) continue;
        if (kFragments) {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float2 x = *reinterpret_cast<const float2*>(s_scale + 8 * j + two);
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
              float &f0 = f[8 * (r >> 1) + 4 * j + 2 * (r & 1)], &f1 = f[8 * (r >> 1) + 4 * j + 2 * (r & 1) + 1];
              mul2(f0, f1, scales.w[r], scales.w[r]);
              if (EPI == kI8Bf16) scaled2(f0, f1, x.x, x.y, scales.bias[EPI == kI8Bf16 ? r : 0]);
              else mul2(f0, f1, x.x, x.y);
            }
          }
        } else {
#pragma unroll
          for (int j = 0; j < kI8Chunk; j += 4) {
            const float4 x = *reinterpret_cast<const float4*>(s_scale + j);
            mul2(f[j], f[j + 1], scales.w[0], scales.w[0]);
            mul2(f[j + 2], f[j + 3], scales.w[0], scales.w[0]);
            scaled2(f[j], f[j + 1], x.x, x.y, scales.bias[0]);
            scaled2(f[j + 2], f[j + 3], x.z, x.w, scales.bias[0]);
          }
          if (EPI == kI8Relu)
#pragma unroll
            for (int j = 0; j < kI8Chunk; ++j) f[j] = f[j] < 0.f ? 0.f : f[j];               // NaN stays NaN
        }
        if (kSwiglu)
#pragma unroll
          for (int i = 0; i < 8; ++i)
            f[i] = silu(f[i]) * f[8 + i];
        if (EPI == kI8F32 && a.direct) {
#pragma unroll
          for (int j = 0; j < kI8Chunk; ++j)
            if (j < left && col < a.n_cols) static_cast<float*>(a.C)[(size_t)(td.row0 + t0 + j) * a.ldc + col] = f[j];
          continue;
        }
        // Boxes of 16 tokens leave through the TMA unit.  Rows of a listed tile up to the next multiple of 16 are stored with the valid
        // ones: they lie in the slot's own segment, and nobody reads a row that no pair occupies.
        unsigned char* const stg = stg0 + box * kBox;
        box ^= 1;
        if (lane == 0) ptx::tma_store_wait_read_but_one();     // the box before the last one has left
        __syncwarp();
        if (kSwiglu) {
          // [16 tokens][16 units] with the 64-byte swizzle; lanes of units 4 ... 7 begin with their odd token, whose row lies in the other banks
          const int swap = hi;
#pragma unroll
          for (int u = 0; u < 8; ++u) {
            const int j = u >> 2, i = (u >> 1) & 1, e = (u & 1) ^ swap, token = 8 * j + two + e;
            const float odd_value = f[4 * j + 2 * i + 1], even_value = f[4 * j + 2 * i];
            reinterpret_cast<float*>(stg)[token * 16 + 4 * ((2 * i + (row8 >> 2)) ^ (two >> 1)) + (row8 & 3)] = e ? odd_value : even_value;
          }
        } else if (EPI == kI8Bf16) {
          // [16 tokens][32 columns] with the 64-byte swizzle, eight tokens a store; this lane has the place of token l % 8, columns 8 (l / 8) ... + 7
          const uint32_t at = ptx::smem_u32(stg) + (uint32_t)((lane & 7) * 64 + 16 * ((lane >> 3) ^ ((lane >> 1) & 3)));
#pragma unroll
          for (int j = 0; j < 2; ++j)
            ptx::store_matrices_transposed(at + 512u * j, pack_bf16x2(f[4 * j], f[4 * j + 1]), pack_bf16x2(f[4 * j + 2], f[4 * j + 3]),
                                           pack_bf16x2(f[8 + 4 * j], f[8 + 4 * j + 1]), pack_bf16x2(f[8 + 4 * j + 2], f[8 + 4 * j + 3]));
          if (a.direct) {                                      // (the box is a way between the lanes)
            __syncwarp();
            if (a.direct == 2) {
              const int pair = lane & 15;
#pragma unroll
              for (int j = hi; j < kI8Chunk; j += 2)
                if (j < left && col0 + 2 * pair < a.n_cols)
                  *reinterpret_cast<uint32_t*>(static_cast<bf16*>(a.C) + (size_t)(td.row0 + t0 + j) * a.ldc + col0 + 2 * pair) =
                      reinterpret_cast<const uint32_t*>(stg)[j * 16 + 4 * ((pair >> 2) ^ ((j >> 1) & 3)) + (pair & 3)];
            } else {
#pragma unroll
              for (int j = 0; j < kI8Chunk; ++j)
                if (j < left && col < a.n_cols)
                  static_cast<bf16*>(a.C)[(size_t)(td.row0 + t0 + j) * a.ldc + col] =
                      reinterpret_cast<const bf16*>(stg)[j * 32 + 8 * ((lane >> 3) ^ ((j >> 1) & 3)) + (lane & 7)];
            }
            continue;
          }
        } else {
          float* w = reinterpret_cast<float*>(stg) + lane;     // [16 tokens][32 columns]
#pragma unroll
          for (int j = 0; j < kI8Chunk; ++j) w[32 * j] = f[j];
        }
        ptx::fence_proxy_async();                              // the staged box is read by the TMA unit
        __syncwarp();
        if (lane == 0) ptx::tma_store_2d(&tmC, stg, col0, td.row0 + t0);
        if (EPI == kI8Relu || kSwiglu) {
          // two lanes take a token over the box's columns
          constexpr int kQuads = kSwiglu ? 2 : 4;
          const float4* row = reinterpret_cast<const float4*>(stg) + lane * kQuads;
          float most = 0.f;
#pragma unroll
          for (int i = 0; i < kQuads; ++i) {
            const float4 u = row[i];
            most = max_magnitude(max_magnitude(most, u.x, u.y), u.z, u.w);
          }
          most = max_magnitude(most, __shfl_xor_sync(0xffffffffu, most, 1), 0.f);
          if ((lane & 1) == 0 && lane / 2 < left) atomicMax(a.largest + td.row0 + t0 + lane / 2, __float_as_int(most) & 0x7fffffff);
        }
      }
      if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
    }
    if (!a.direct && lane == 0) ptx::tma_store_wait_all();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::cluster_sync_all();       // neither CTA's shared memory, barriers or TMEM go away while the peer may touch them
  if (warp == 2) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc_pair(tmem_base, kTmemCols);
  }
}

// ----------------------------------------------------------------------------- host side
typedef void (*I8GemmKernel)(const CUtensorMap, const CUtensorMap, const CUtensorMap, const CUtensorMap, const CUtensorMap,
                             const CUtensorMap, const I8GemmArgs);

inline I8GemmKernel int8_gemm_kernel(int epi) {
  return epi == kI8Bf16 ? int8_gemm_pair_kernel<kI8Bf16> : epi == kI8F32 ? int8_gemm_pair_kernel<kI8F32>
         : epi == kI8Relu ? int8_gemm_pair_kernel<kI8Relu> : int8_gemm_pair_kernel<kI8Swiglu>;
}

// How a staged box of results lies in shared memory (rows of 64 bytes: swizzled, for the stores that transpose).
inline CUtensorMapSwizzle int8_out_swizzle(int epi) { return int8_box_bytes(epi) == 1024 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_NONE; }

// View of a row-major matrix [rows, cols] with a box of box_cols x box_rows elements (type: unsigned bytes, bf16 or fp32).
inline bool int8_encode_2d(PFN_encodeTiled enc, CUtensorMap* m, const void* base, CUtensorMapDataType type, uint64_t elem, uint64_t rows,
                           uint64_t cols, uint64_t stride, uint32_t box_cols, uint32_t box_rows, CUtensorMapSwizzle swizzle) {
  const cuuint64_t dims[2] = {cols, rows};
  const cuuint64_t strides[1] = {stride * elem};
  const cuuint32_t box[2] = {box_cols, box_rows};
  const cuuint32_t estr[2] = {1, 1};
  return enc(m, type, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
inline bool int8_encode_operand(PFN_encodeTiled enc, CUtensorMap* m, const void* base, uint64_t rows, uint64_t cols, uint64_t stride,
                                uint32_t box_rows) {
  return int8_encode_2d(enc, m, base, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, rows, cols, stride, kI8BK, box_rows, CU_TENSOR_MAP_SWIZZLE_128B);
}

// Once per device and process: shared memory limits of the kernels; 0 or the number of CTA pairs that run at once.
inline int int8_gemm_init(int sm_count) {
  for (int epi = 0; epi < 4; ++epi)
    if (cudaFuncSetAttribute(int8_gemm_kernel(epi), cudaFuncAttributeMaxDynamicSharedMemorySize, int8_smem_bytes(epi)) != cudaSuccess) {
      cudaGetLastError();
      return 0;
    }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2 * (sm_count / 2)); cfg.blockDim = dim3(kI8Threads); cfg.dynamicSmemBytes = int8_smem_bytes(kI8F32);
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  int n = 0;
  if (cudaOccupancyMaxActiveClusters(&n, int8_gemm_pair_kernel<kI8F32>, &cfg) != cudaSuccess) {
    cudaGetLastError();
    return 0;
  }
  return n < sm_count / 2 ? n : sm_count / 2;
}

// Rows of a token tile for T rows and n_col_tiles weight tiles on n_pairs pairs of CTAs: the height whose rounds of tiles cost least.
inline int int8_tile_height(int T, int n_col_tiles, int n_pairs) {
  int best = 256;
  long long least = -1;
  for (int h = 256; h >= 32; h -= 32) {
    const long long tiles = (long long)((T + h - 1) / h) * n_col_tiles;
    const long long cost = (tiles + n_pairs - 1) / n_pairs * int8_tile_cost(h);
    if (least < 0 || cost < least) { least = cost; best = h; }
  }
  return best;
}

}  // namespace swapmoe
