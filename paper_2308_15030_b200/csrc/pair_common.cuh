// What the GEMMs on CTA pairs share: the geometry of their stages, PTX wrappers for clusters of two and tcgen05 `cta_group::2`.
#pragma once
#include "tc_common.cuh"

namespace swapmoe {

constexpr int kPairTokens = 256;                              // most tokens of a tile
constexpr int kPairMinTokens = 64;                            // ... and the least that pick_tile_height allows it
constexpr int kPairTokenStep = 32;                            // their number is a multiple of this
constexpr int kPairThreads = 384;
constexpr int kPairABytes = kTcBM * kTcBK * 2;                // 16 KB: the CTA's weight rows of a k-block
constexpr int kPairBBytes = kPairTokens / 2 * kTcBK * 2;      // at most 16 KB: its tokens
constexpr int kPairStageArea = 6 * (kPairABytes + kPairBBytes);   // 6 stages of 256 tokens, 8 of 128, 9 of 64
constexpr int kPairMaxStages = 9;
__device__ __forceinline__ int pair_stages(int max_tokens) { return max_tokens > 128 ? 6 : max_tokens > 64 ? 8 : 9; }

// Shared memory that a CTA takes at least if it waits for its cluster with tensor memory in hand: none of a GEMM on CTA pairs, which takes all
// columns of two SMs, then fits its SM beside it.  (One SM's columns would be the cluster's, the other's the pair's, and either wait for the
// rest.)
constexpr int kClusterMinSmem = 28 * 1024;
constexpr bool fits_beside_cluster(int pair_smem) { return pair_smem + kClusterMinSmem + 2 * 1024 <= 228 * 1024; }       // (the system keeps 1 KB of each)

namespace ptx {

__device__ __forceinline__ uint32_t cluster_ctarank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
// Address of the same shared-memory location in CTA `rank` of the cluster (shared::cluster window).
__device__ __forceinline__ uint32_t map_to_cta(uint32_t smem_addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// tcgen05.alloc.cta_group::2 takes columns in both SMs, so neither CTA may issue it before the other one has started: without
// this a pair was seen waiting for ever in its allocation (8192 tokens, top-4 of 256 experts, where CTAs of the
// permutation in front still occupy a part of the SMs when the pairs come up).
__device__ __forceinline__ void cluster_start_sync() {
  __syncthreads();
  cluster_sync_all();
}
// Tile load whose completion bytes are credited to a barrier that may live in the peer CTA.
__device__ __forceinline__ void tma_load_2d_pair(void* dst, const CUtensorMap* map, uint32_t bar_cluster_addr, int c0,
                                                 int c1) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
      ::"r"(smem_u32(dst)), "l"(map), "r"(bar_cluster_addr), "r"(c0), "r"(c1)
      : "memory");
}
// The same for a box of five dimensions.
__device__ __forceinline__ void tma_load_5d_pair(void* dst, const CUtensorMap* map, uint32_t bar_cluster_addr, int c0,
                                                 int c1, int c2, int c3, int c4) {
  asm volatile(
      "cp.async.bulk.tensor.5d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];"
      ::"r"(smem_u32(dst)), "l"(map), "r"(bar_cluster_addr), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4)
      : "memory");
}
// Arrival on a barrier that may live in the peer CTA, releasing what this thread has done before.
__device__ __forceinline__ void mbar_arrive_release_cluster(uint32_t bar_cluster_addr) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar_cluster_addr) : "memory");
}
// A box of shared memory to global memory; columns and rows outside the matrix are left out.
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* map, const void* src, int c0, int c1) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];\ncp.async.bulk.commit_group;" ::"l"(map),
               "r"(smem_u32(src)), "r"(c0), "r"(c1)
               : "memory");
}
// This thread's stores have read their shared memory.
__device__ __forceinline__ void tma_store_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void tma_store_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
// Arrival on a barrier that the peer CTA's threads wait on (mbar_try_wait_cluster).  Relaxed at cluster scope: with the tcgen05
// fences on either side it orders this warp's tcgen05 accesses (the accumulator has been read, tcgen05.wait::ld has
// returned) before the waiter's, and nothing else is handed over: nobody in this kernel reads the stores of the epilogue.  With
// .release every epilogue warp waited here until its tile's global stores had been performed, behind the operand loads in
// flight (24044 rows, d_model 1024, d_ff 512, y in fp32: GEMM-2 alone 49 -> 42 us; 8192 rows 768 x 3072: GEMM-1 49.5 -> 46.0).
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar_cluster_addr) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar_cluster_addr) : "memory");
}
__device__ __forceinline__ void tmem_alloc_pair(uint32_t* dst_smem, uint32_t ncols) {
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(dst_smem)),
               "r"(ncols)
               : "memory");
}
__device__ __forceinline__ void tmem_relinquish_pair() {
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_dealloc_pair(uint32_t taddr, uint32_t ncols) {
  asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols) : "memory");
}
// Arrives on the barrier at this shared-memory offset in both CTAs of the pair once the MMAs issued so far are done.
__device__ __forceinline__ void umma_commit_pair(uint64_t* bar) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
          smem_u32(bar)),
      "h"((unsigned short)3)
      : "memory");
}

}  // namespace ptx

}  // namespace swapmoe
