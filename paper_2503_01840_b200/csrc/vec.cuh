// Eight elements of a row at a time, as 32-bit floats; sums over a block.
#pragma once
#include "common.cuh"

namespace spec {

__device__ __forceinline__ float load_as_f32(const void *p, int dtype, long long i) {      // dtype: 0 fp32, 1 bf16
  return dtype == 0 ? ((const float *)p)[i] : __bfloat162float(((const bf16 *)p)[i]);
}
__device__ __forceinline__ void store_from_f32(void *p, int dtype, long long i, float v) {
  if (dtype == 0) ((float *)p)[i] = v;
  else ((bf16 *)p)[i] = __float2bfloat16_rn(v);
}

// Sum and maximum over a block of whole warps, the same for every thread; `room`: 32 floats of shared memory, free again after the next barrier.
__device__ __forceinline__ float block_sum(float v, float *room) {
#pragma unroll
  for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) room[threadIdx.x >> 5] = v;
  __syncthreads();
  const int warps = blockDim.x >> 5;
  v = (threadIdx.x & 31) < warps ? room[threadIdx.x & 31] : 0.0f;
#pragma unroll
  for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}
__device__ __forceinline__ uint32_t block_max(uint32_t v, float *room) {
  v = __reduce_max_sync(0xffffffffu, v);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) room[threadIdx.x >> 5] = __uint_as_float(v);
  __syncthreads();
  v = (threadIdx.x & 31) < (blockDim.x >> 5) ? __float_as_uint(room[threadIdx.x & 31]) : 0u;
  return __reduce_max_sync(0xffffffffu, v);
}

}  // namespace spec
