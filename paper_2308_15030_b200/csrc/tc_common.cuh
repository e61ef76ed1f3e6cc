// What the tensor-core kernels share: operand descriptors, the order of tiles, the driver's tensor-map encoder.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include "common.cuh"
#include "ptx.cuh"

namespace swapmoe {

constexpr int kTcBM = 128;   // rows per tile (TMEM lanes)
constexpr int kTcBK = 64;    // bf16 elements per k-block = one 128-byte swizzle row
constexpr int kTcUmmaK = 16;

// Shared-memory operand descriptor: K-major tile whose rows are 128 bytes, written by
// TMA with 128-byte swizzle; 8-row groups are 1024 bytes apart.
__device__ __forceinline__ uint64_t make_kmajor_sw128_desc(uint32_t smem_addr) {
  uint64_t d = 0;
  d |= (uint64_t)((smem_addr & 0x3FFFFu) >> 4);  // start address
  d |= (uint64_t)(1024u >> 4) << 32;             // stride between 8-row groups
  d |= (uint64_t)1 << 46;                        // descriptor version of this architecture
  d |= (uint64_t)2 << 61;                        // 128-byte swizzle
  return d;
}
// Work item t -> (row tile, column tile).  Row tiles vary fastest inside a group of `group` row
// tiles, column tiles next, groups last: the row tiles of a slot (which share weights) run side
// by side, and for large problems the activations of one group stay in L2 while its column
// tiles are walked (group >= n_row_tiles: one group).
__device__ __forceinline__ void decode_tile(int t, int n_row_tiles, int n_col_tiles, int group, int* rt, int* ct) {
  group = min(group, n_row_tiles);
  const int per_group = group * n_col_tiles;
  const int g = t / per_group;
  const int r0 = g * group;
  const int rows_here = min(group, n_row_tiles - r0);
  const int u = t - g * per_group;
  *ct = u / rows_here;
  *rt = r0 + (u - *ct * rows_here);
}

typedef CUresult (*PFN_encodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                    const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                    CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                    CUtensorMapFloatOOBfill);

// The driver's tensor-map encoder (nullptr when it cannot be had).
inline PFN_encodeTiled tc_get_encoder() {
  void* fn = nullptr;
  cudaDriverEntryPointQueryResult qres;
  if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &qres) != cudaSuccess ||
      qres != cudaDriverEntryPointSuccess) {
    cudaGetLastError();
    return nullptr;
  }
  return reinterpret_cast<PFN_encodeTiled>(fn);
}

}  // namespace swapmoe
