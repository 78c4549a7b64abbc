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

// eight neighbours, 16-byte aligned
__device__ __forceinline__ void unpack2(uint32_t u, float &a, float &b) { a = __uint_as_float(u << 16), b = __uint_as_float(u & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *(const uint32_t *)&v;
}
__device__ __forceinline__ void load8(const float *p, float (&y)[8]) {
  const float4 a = ((const float4 *)p)[0], b = ((const float4 *)p)[1];
  y[0] = a.x, y[1] = a.y, y[2] = a.z, y[3] = a.w, y[4] = b.x, y[5] = b.y, y[6] = b.z, y[7] = b.w;
}
__device__ __forceinline__ void load8(const bf16 *p, float (&y)[8]) {
  const uint4 u = *(const uint4 *)p;
  unpack2(u.x, y[0], y[1]), unpack2(u.y, y[2], y[3]), unpack2(u.z, y[4], y[5]), unpack2(u.w, y[6], y[7]);
}
__device__ __forceinline__ void store8(float *p, const float (&y)[8]) {
  ((float4 *)p)[0] = make_float4(y[0], y[1], y[2], y[3]);
  ((float4 *)p)[1] = make_float4(y[4], y[5], y[6], y[7]);
}
__device__ __forceinline__ void store8(bf16 *p, const float (&y)[8]) {
  *(uint4 *)p = make_uint4(pack2(y[0], y[1]), pack2(y[2], y[3]), pack2(y[4], y[5]), pack2(y[6], y[7]));
}
// Two 32-bit numbers, whose sums and products take one instruction
typedef unsigned long long Pair;
__device__ __forceinline__ Pair pair(float a, float b) {
  Pair p;
  asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "f"(a), "f"(b));
  return p;
}
__device__ __forceinline__ void unpair(Pair p, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p)); }
__device__ __forceinline__ Pair add(Pair a, Pair b) {
  Pair p;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(p) : "l"(a), "l"(b));
  return p;
}
__device__ __forceinline__ Pair mul(Pair a, Pair b) {
  Pair p;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(p) : "l"(a), "l"(b));
  return p;
}
__device__ __forceinline__ Pair fma(Pair a, Pair b, Pair c) {
  Pair p;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(p) : "l"(a), "l"(b), "l"(c));
  return p;
}

// Eight neighbours as they lie in memory
template <typename T> struct Raw8;
template <> struct Raw8<float> {
  float4 a, b;
  __device__ __forceinline__ void take(const float *p) { a = ((const float4 *)p)[0], b = ((const float4 *)p)[1]; }
  __device__ __forceinline__ void floats(float (&y)[8]) const { y[0] = a.x, y[1] = a.y, y[2] = a.z, y[3] = a.w, y[4] = b.x, y[5] = b.y, y[6] = b.z, y[7] = b.w; }
};
template <> struct Raw8<bf16> {
  uint4 u;
  __device__ __forceinline__ void take(const bf16 *p) { u = *(const uint4 *)p; }
  __device__ __forceinline__ void floats(float (&y)[8]) const { unpack2(u.x, y[0], y[1]), unpack2(u.y, y[2], y[3]), unpack2(u.z, y[4], y[5]), unpack2(u.w, y[6], y[7]); }
};
// Copies to shared memory that run on while the thread does; those of a thread complete by groups, in order.
__device__ __forceinline__ uint32_t smem_of(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy16(void *to, const void *from) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_of(to)), "l"(from) : "memory"); }
template <typename T> __device__ __forceinline__ void copy8(T *to, const T *from) {      // eight elements
  copy16(to, from);
  if (sizeof(T) == 4) copy16(to + 4, from + 4);
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_but() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }      // all groups but the last N are there

// rows whose pieces of 16 bytes are aligned, elements of e bytes
inline bool pieces_aligned(const void *p, long long row_stride, size_t e) { return ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)(row_stride * (long long)e)) & 15) == 0; }

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
