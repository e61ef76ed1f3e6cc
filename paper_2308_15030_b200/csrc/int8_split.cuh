// Products of 8-bit integers on few tiles, for up to 128 tokens and more on narrow matrices: a cluster shares the contraction of a tile.
//
// n / 128 tiles for each group of up to 128 tokens are too few for the SMs that the bytes should come through: an SM takes in 87 GB/s at most, which is
// what bounds a CTA.  Each CTA of a cluster takes a share of the k-blocks of 128 weight rows x all tokens of the group (tcgen05 kind::i8, operands by
// TMA), and the shares are added as integers, so that neither the split nor its order changes a bit: every CTA collects the tokens of its rank from
// the others' shared memory, scales them and stores them.
// Roles (320 threads): warp 0 = TMA producer, warp 1 = TMEM allocation and MMA issuer, warps 2-9 = sums out of
// tensor memory, and what is done with them.  No load uses cluster multicast.  Every mbarrier wait is bounded; the cluster barriers behind them
// are not, nor is the allocation of tensor memory (three CTAs an SM take 384 of its 512 columns; kernels beside them wait for no cluster with theirs).
// 1 token, 4096 x 4096: 4.4 us where the weights lie in L2, 5.8 from memory; 256 tokens, 4096 -> 1024 6.1 us (CTA pairs 10.5).
#pragma once
#include "int8_gemm.cuh"

namespace swapmoe {

constexpr int kSplitThreads = 320;
constexpr int kSplitMaxTokens = 128;
constexpr int kSplitMaxStages = 12;
constexpr int kSplitABytes = kTcBM * kI8BK;
constexpr int kSplitRoom = 108 * 1024;                        // bytes of the ring: two CTAs an SM
constexpr int kSplitMaxSmem = 1024 + kSplitRoom;

struct I8SplitArgs {
  void* out;
  const float *x_scales, *w_scales, *bias;
  long long ldc;
  int32_t T, N, k_blocks, share;       // share: k-blocks of a CTA
  int32_t cols, n_stages;              // tokens of a cluster, a multiple of 16 and of 4 x its CTAs; stages of the ring
};

namespace ptx {
__device__ __forceinline__ void umma_int8(uint32_t tmem_d, uint64_t desc_a, uint64_t desc_b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n}\n" ::"r"(tmem_d),
      "l"(desc_a), "l"(desc_b), "r"(idesc), "r"(accumulate)
      : "memory");
}
}  // namespace ptx

// bytes behind the ring's start: the ring, or (when it has been read) the shares of `cols` tokens
__host__ __device__ inline int int8_split_area(int cols, int n_stages) {
  const int ring = n_stages * (kSplitABytes + cols * kI8BK), sums = cols * kTcBM * 4;
  return ring > sums ? ring : sums;
}

template <typename Out>
__global__ void __launch_bounds__(kSplitThreads) int8_split_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX,
                                                                   const __grid_constant__ I8SplitArgs a) {
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  __shared__ uint64_t full[kSplitMaxStages], empty[kSplitMaxStages], done;
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_word;
  __shared__ __align__(16) float s_x_scale[kSplitMaxTokens];
  volatile int* abort_flag = &abort_word;
  int32_t* const status = g_int8_status;
  uint32_t rank, size;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(size));
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int n0 = (int)(blockIdx.x / size) * kTcBM, first = (int)blockIdx.y * a.cols, T = a.T - first;       // first token, tokens from there on
  const int q = warp & 3, part = (warp - 2) >> 2, n = n0 + q * 32 + lane;   // warps 2-9: the quarter of tensor memory that the warp may read, and its weight row
  float w_scale = 0.f, bias = 0.f;
  const int kb0 = (int)rank * a.share, kb1 = min(a.k_blocks, kb0 + a.share), blocks = max(0, kb1 - kb0);
  unsigned char* sW = smem;                                   // [stages][128][128]
  unsigned char* sX = smem + a.n_stages * kSplitABytes;       // [stages][cols][128]
  const int x_bytes = a.cols * kI8BK;
  if (threadIdx.x == 0) {
    for (int s = 0; s < a.n_stages; ++s) { ptx::mbar_init(&full[s], 1); ptx::mbar_init(&empty[s], 1); }
    ptx::mbar_init(&done, 1);
    abort_word = 0;
    ptx::fence_barrier_init();
    ptx::prefetch_tmap(&tmW);
    ptx::prefetch_tmap(&tmX);
  }
  __syncthreads();
  const uint32_t tmem_cols = a.cols <= 32 ? 32u : a.cols <= 64 ? 64u : 128u;
  uint32_t tmem_base = 0;
  pdl_wait();
  if (warp == 0) {
    // ------------------------------------------------------------------ TMA producer
    bool ok = true;
    int stage = 0;
    uint32_t phase = 0;
    for (int i = 0; i < blocks; ++i) {
      ok = warp_wait(&empty[stage], phase ^ 1u, abort_flag, status, 41);
      if (!ok) break;
      if (ptx::elect_one()) {
        ptx::mbar_expect_tx(&full[stage], (uint32_t)(kSplitABytes + x_bytes));
        ptx::tma_load_2d(sW + stage * kSplitABytes, &tmW, &full[stage], (kb0 + i) * kI8BK, n0);
        ptx::tma_load_2d(sX + stage * x_bytes, &tmX, &full[stage], (kb0 + i) * kI8BK, first);
      }
      __syncwarp();
      if (++stage == a.n_stages) { stage = 0; phase ^= 1u; }
    }
    if (!ok) {
      // Give copies that are still in flight time to land before shared memory is used for something else.
      const uint64_t t0 = ptx::globaltimer_ns();
      while (ptx::globaltimer_ns() - t0 < 2000000ull) __nanosleep(1000);
    }
  } else {
    if (warp == 1) {
      ptx::tmem_alloc(&tmem_slot, tmem_cols);
      ptx::tmem_relinquish();
    }
    ptx::tc_fence_before();
    asm volatile("bar.sync 1, %0;" ::"n"(kSplitThreads - 32) : "memory");
    ptx::tc_fence_after();
    tmem_base = *reinterpret_cast<volatile uint32_t*>(&tmem_slot);
    pdl_trigger();
    if (warp == 1) {
      // ---------------------------------------------------------------- MMA issuer
      const uint32_t idesc = make_idesc_int8(kTcBM, a.cols);
      int stage = 0;
      uint32_t phase = 0;
      for (int i = 0; i < blocks; ++i) {
        if (!warp_wait(&full[stage], phase, abort_flag, status, 42)) break;
        ptx::tc_fence_after();
        const uint64_t dw = make_kmajor_sw128_desc(ptx::smem_u32(sW + stage * kSplitABytes));
        const uint64_t dx = make_kmajor_sw128_desc(ptx::smem_u32(sX + stage * x_bytes));
        if (ptx::elect_one()) {
#pragma unroll
          for (int k = 0; k < 4; ++k)
            ptx::umma_int8(tmem_base, dw + (uint64_t)(2 * k), dx + (uint64_t)(2 * k), idesc, (i > 0 || k > 0) ? 1u : 0u);
          ptx::umma_commit(&empty[stage]);
          if (i + 1 == blocks) ptx::umma_commit(&done);
        }
        __syncwarp();
        if (++stage == a.n_stages) { stage = 0; phase ^= 1u; }
      }
    } else {
      // ---------------------------------------------------------------- scales meanwhile, then the sums
      if (n < a.N) {
        w_scale = a.w_scales[n];
        if (a.bias != nullptr) bias = a.bias[n];
      }
      const int t = q * 32 + lane;
      if (part == 0) s_x_scale[t] = t < T ? a.x_scales[first + t] : 0.f;
      if (blocks > 0) {
        warp_wait(&done, 0u, abort_flag, status, 43);
        ptx::tc_fence_after();
      }
    }
  }
  // The rings of all CTAs have been read: their memory takes the shares, four tokens of a weight row at a time.  (A CTA whose wait gave up goes
  // on with what it has: the status says so.)
  __syncwarp();
  if (size > 1) ptx::cluster_sync_all();
  else __syncthreads();
  const int mine = a.cols / (int)size;                        // tokens that a CTA collects
  int4* s_sums = reinterpret_cast<int4*>(smem);               // [size][mine / 4][128]
  if (warp >= 2) {
    const uint32_t to0 = ptx::smem_u32(s_sums) + 16u * (uint32_t)((int)rank * (mine / 4) * kTcBM + q * 32 + lane);
    // CTA that collects these tokens, and their place there (mine / 4 may be anything: divided once)
    int owner = part * 4 / (mine / 4), at = part * 4 - owner * (mine / 4);
#pragma unroll 1
    for (int c0 = 16 * part; c0 < a.cols; c0 += 32) {
      uint32_t v[16];
      if (blocks > 0) {
        ptx::tmem_ld16(tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)c0, v);
        ptx::tmem_ld_wait();
      } else {
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] = 0u;
      }
#pragma unroll
      for (int j = 0; j < 16; j += 4) {
        const uint32_t to = to0 + 16u * (uint32_t)(at * kTcBM);
        asm volatile("st.shared::cluster.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(ptx::map_to_cta(to, (uint32_t)owner)), "r"(v[j]), "r"(v[j + 1]),
                     "r"(v[j + 2]), "r"(v[j + 3])
                     : "memory");
        if (++at == mine / 4) { at = 0; ++owner; }
      }
      for (at += 4; at >= mine / 4; at -= mine / 4) ++owner;  // the other warps' sixteen
    }
  }
  ptx::tc_fence_before();
  if (size > 1) ptx::cluster_sync_all();
  else __syncthreads();
  if (warp == 1) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem_base, tmem_cols);
  }
  if (warp < 2 || n >= a.N) return;
  const int t0 = (int)rank * mine;
#pragma unroll 2
  for (int i = part; i < mine / 4 && t0 + 4 * i < T; i += 2) {
    int4 v = s_sums[i * kTcBM + q * 32 + lane];
    for (int o = 1; o < (int)size; ++o) {
      const int4 u = s_sums[(o * (mine / 4) + i) * kTcBM + q * 32 + lane];
      v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
    }
    const float4 xs = *reinterpret_cast<const float4*>(s_x_scale + t0 + 4 * i);
    const float f[4] = {fmaf((float)v.x * w_scale, xs.x, bias), fmaf((float)v.y * w_scale, xs.y, bias), fmaf((float)v.z * w_scale, xs.z, bias),
                        fmaf((float)v.w * w_scale, xs.w, bias)};
    Out* out = static_cast<Out*>(a.out) + (size_t)(first + t0 + 4 * i) * a.ldc + n;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (t0 + 4 * i + j < T) {
        if constexpr (sizeof(Out) == 2) out[j * a.ldc] = __float2bfloat16_rn(f[j]);
        else out[j * a.ldc] = f[j];
      }
  }
}

}  // namespace swapmoe
