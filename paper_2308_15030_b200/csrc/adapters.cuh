// Low-rank adapters of many requests beside a projection that all of them share:
//   out[t] = y[t] + scale_a * B_a (A_a x[t]),  a = ids[t]  (no adapter: out[t] = y[t]),
// A_a [rank, d_in], B_a [d_out, rank], y the shared projection's row.
#pragma once
#include <cuda_fp8.h>

#include "common.cuh"
#include "launch.cuh"

namespace swapmoe {

constexpr int kAdMaxRank = 128, kAdMaxCount = 4096, kAdMaxWidth = 1 << 20;

struct AdapterArgs {
  const void* x;            // [T, d] rows of T or e4m3
  const float* x_scales;    // [T] with e4m3 rows
  const int32_t* ids;       // [T]
  const void* y;            // [T, n] or nullptr (zeros)
  void* out;                // [T, n]
  const void *A, *B;        // [count, r, d], [count, n, r]
  const float* scale;       // [count] or nullptr (ones)
  float* u;                 // [T, r]
  long long x_stride, y_stride, out_stride;
  int T, d, n, r, count;
};

__device__ __forceinline__ float ad_value(float v) { return v; }
__device__ __forceinline__ float ad_value(bf16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float ad_value(__nv_fp8_e4m3 v) { return (float)v; }
__device__ __forceinline__ void ad_store(float* p, float v) { *p = v; }
__device__ __forceinline__ void ad_store(bf16* p, float v) { *p = __float2bfloat16_rn(v); }

// u[t, j] = scale * A_a[j] . x[t]: a warp per (t, j).
template <typename X, typename T>
__global__ void adapters_shrink_kernel(const AdapterArgs a) {
  pdl_wait();
  pdl_trigger();
  const long long w = (long long)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (w >= (long long)a.T * a.r) return;
  const long long t = w / a.r;
  const int j = (int)(w - t * a.r), id = a.ids[t];
  if (id < 0 || id >= a.count) return;
  const X* x = static_cast<const X*>(a.x) + t * a.x_stride;
  const T* A = static_cast<const T*>(a.A) + ((long long)id * a.r + j) * a.d;
  float s = 0.f;
  for (int c = lane; c < a.d; c += 32) s = fmaf(ad_value(x[c]), ad_value(A[c]), s);
  s = warp_sum(s);
  if (a.x_scales != nullptr) s *= a.x_scales[t];
  if (a.scale != nullptr) s *= a.scale[id];
  if (lane == 0) a.u[t * a.r + j] = s;
}

template <typename T>
__global__ void adapters_expand_kernel(const AdapterArgs a) {
  pdl_wait();
  pdl_trigger();
  const long long t = blockIdx.x;
  const int c = blockIdx.y * blockDim.x + threadIdx.x, id = a.ids[t];
  if (c >= a.n) return;
  float v = a.y != nullptr ? ad_value(static_cast<const T*>(a.y)[t * a.y_stride + c]) : 0.f;
  if (id >= 0 && id < a.count) {
    const T* B = static_cast<const T*>(a.B) + ((long long)id * a.n + c) * a.r;
    float s = 0.f;
    for (int j = 0; j < a.r; ++j) s = fmaf(a.u[t * a.r + j], ad_value(B[j]), s);
    v += s;
  }
  ad_store(static_cast<T*>(a.out) + t * a.out_stride + c, v);
}

template <typename X, typename T>
inline cudaError_t adapters_launch(const AdapterArgs& a, cudaStream_t st, bool pdl) {
  const long long warps = (long long)a.T * a.r;
  cudaError_t e = launch_kernel(adapters_shrink_kernel<X, T>, dim3((unsigned)((warps + 7) / 8)), dim3(256), 0, st, pdl, a);
  if (e != cudaSuccess) return e;
  return launch_kernel(adapters_expand_kernel<T>, dim3((unsigned)a.T, (unsigned)((a.n + 255) / 256)), dim3(256), 0, st, pdl, a);
}

}  // namespace swapmoe
