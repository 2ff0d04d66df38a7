// The learned bias of relative positions: the table of buckets spread over the distances, and the gradient of its entries.
#include <cuda_bf16.h>

#include "internal.h"

namespace ea {
namespace {

template <typename T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// One thread per (head, distance): the largest bucket that starts at or before the distance, found by bisection (empty
// buckets share their start with the next one, which is then the larger).  H x bias_len numbers, a launch's latency.
template <typename T>
__global__ void __launch_bounds__(256) bias_expand_kernel(const BiasParams p) {
  const int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (at >= static_cast<int64_t>(p.H) * p.bias_len) return;
  const int h = static_cast<int>(at / p.bias_len), d = static_cast<int>(at - static_cast<int64_t>(h) * p.bias_len);
  int lo = 0, hi = p.buckets;                                // starts[lo] <= d < starts[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (__ldg(p.starts + mid) <= d) lo = mid; else hi = mid;
  }
  p.bias[at] = to_f<T>(static_cast<const T*>(p.table)[static_cast<int64_t>(h) * p.buckets + lo]) * 1.4426950408889634f;
}

// Gradient of one table entry: the sums of dS that the backward pass left for its bucket, added in a fixed order (thread t
// takes parts t, t + 128, ...; then a tree), in 64 bits, so that the result does not depend on the order of arrival.
template <typename T>
__global__ void __launch_bounds__(128) bias_reduce_kernel(const TrainParams p) {
  const int h = blockIdx.x, u = blockIdx.y, t = threadIdx.x;
  const float* part = p.bias_part + static_cast<int64_t>(h) * p.bias_parts * p.buckets + u;
  double sum = 0;
  for (int i = t; i < p.bias_parts; i += 128) sum += part[static_cast<int64_t>(i) * p.buckets];
  __shared__ double warps[4];
#pragma unroll
  for (int d = 16; d >= 1; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  if ((t & 31) == 0) warps[t >> 5] = sum;
  __syncthreads();
  if (t == 0)
    static_cast<T*>(p.dtable)[static_cast<int64_t>(h) * p.buckets + u] =
        from_f<T>(static_cast<float>((warps[0] + warps[1]) + (warps[2] + warps[3])));
}

}  // namespace

cudaError_t launch_bias_expand(const BiasParams& p, int dtype, cudaStream_t s, uint64_t* launches) {
  const unsigned grid = static_cast<unsigned>((static_cast<int64_t>(p.H) * p.bias_len + 255) / 256);
  if (dtype == 0) bias_expand_kernel<__nv_bfloat16><<<grid, 256, 0, s>>>(p);
  else bias_expand_kernel<float><<<grid, 256, 0, s>>>(p);
  ++*launches;
  return cudaGetLastError();
}

cudaError_t launch_bias_reduce(const TrainParams& p, int dtype, cudaStream_t s, uint64_t* launches) {
  const dim3 grid(p.H, p.buckets);
  if (dtype == 0) bias_reduce_kernel<__nv_bfloat16><<<grid, 128, 0, s>>>(p);
  else bias_reduce_kernel<float><<<grid, 128, 0, s>>>(p);
  ++*launches;
  return cudaGetLastError();
}

}  // namespace ea
