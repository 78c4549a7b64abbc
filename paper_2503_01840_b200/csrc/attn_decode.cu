// Single-token attention: which body takes a call, and how many query heads a warp takes together.
#include <algorithm>

#include "attn_decode_kernel.cuh"

namespace spec {

constexpr size_t DA_COUNT_BYTES = 2048;
static_assert(DA_MAX_CTAS * sizeof(unsigned) <= DA_COUNT_BYTES, "a counter per CTA");
size_t decode_attn_workspace_bytes() { return DA_COUNT_BYTES + (size_t)DA_MAX_CTAS * 2 * DA_PART_FLOATS * sizeof(float); }

cudaError_t launch_decode_attn(const DecodeAttn &a, int dtype, int fmt, cudaStream_t s) {
  DaArgs p{};
  p.a = a;
  p.page_shift = (a.cache.page_size & (a.cache.page_size - 1)) == 0 ? __builtin_ctz(a.cache.page_size) : -1;
  const int group = a.H / a.cache.G, hd = a.cache.hd;
  p.q_f32 = dtype == KV_F32;
  const bool mma = fmt != KV_F32 && (hd == 64 || hd == 128 || hd == 256);
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return e;
  const int ctas = std::min(sms, DA_MAX_CTAS);
  // query heads a warp takes together: what the body holds, fewer where a large batch's table leaves no room for their partial states
  auto fits = [&](int heads) {      // the larger of what the bodies take
    int hp = 1;
    while (hp < heads) hp *= 2;
    const int warps = hd <= 128 ? 16 : 8, own = mma ? 0 : hp * hd + 64;
    return da_smem_bytes(a.batch, warps, own, heads, hd) <= DA_SMEM;
  };
  int most = mma ? (p.q_f32 ? 8 : 16) / (hd < 256 ? 1 : 2) : 8;
  while (most > 1 && !fits(std::min(most, group))) most /= 2;
  p.chunks = (group + most - 1) / most;
  p.heads = (group + p.chunks - 1) / p.chunks;
  p.group = group;
  p.vheads = a.cache.G * p.chunks;
  p.segs = a.batch * p.vheads;
  p.count = (unsigned *)a.workspace;
  p.part = (float *)((char *)a.workspace + DA_COUNT_BYTES);
  return mma ? launch_decode_mma(p, fmt, ctas, s) : launch_decode_fma(p, fmt, ctas, s);
}

}  // namespace spec
