// Single-token attention: which body takes a call, and how many query heads a warp takes together.
#include <algorithm>

#include "attn_decode_kernel.cuh"

namespace spec {

constexpr size_t DA_COUNT_BYTES = 2048;
static_assert(DA_MAX_CTAS * sizeof(unsigned) <= DA_COUNT_BYTES, "a counter per CTA");
size_t decode_attn_workspace_bytes() { return DA_COUNT_BYTES + (size_t)DA_MAX_CTAS * 2 * DA_PART_FLOATS * sizeof(float); }

// A body is the same for all calls of a format, head size, number of heads that a warp takes together and, for heads of 128 in 8 bits, of segments.  Tensor cores:
// up to 16 columns of query heads (fp32 queries take two each), 8 where a head's O is 256 wide.
// NG groups of 16 positions a tile: a warp waits for a tile's keys and for its values once each, so with long runs a tile of 4 KB of 8-bit keys
// or values is better read by 8 warps; 16 warps with half of it lose less where runs are short and every (sequence, KV head) begins with a wait
// of its own.  us with 16 / 8 warps, 8 KV heads of 128 in e4m3 or int8: one sequence of 613 positions 12.0 / 10.7, 4 of 1000 to 8000 19.3 / 17.2, 32 of
// 100 to 400 13.1 / 11.7, 16 of 8192 56.2 / 55.9, 64 of 256 to 2048 42.5 / 48.3; 40 KV heads, 64 of 10 to 100 26.6 / 30.1: up to two of them a CTA 8 warps.
DecodePlan decode_attn_plan(int q_f32, int fmt, int batch, int H, int G, int hd, int ctas, long long positions) {
  const bool mma = fmt != KV_F32 && (hd == 64 || hd == 128 || hd == 256);
  const int group = H / G, bytes = kv_is_8bit(fmt) ? 1 : 2;
  DecodePlan p{};
  // As many heads as the body holds, so that a cache is walked once.  Half of them where there are few (sequence, KV head)s: more than seven CTAs then share one, and the join of their
  // states, by one CTA, takes longer than a second walk.  us with 16 / 8 heads together, 16 query heads a KV head of 128 in e4m3, sequences x KV heads: 1 x 2 of 16384 positions
  // 63.2 / 27.1, 4 x 2 of 8192 30.4 / 20.0, 16 x 1 of 8192 30.0 / 23.2, 24 x 1 of 4096 25.4 / 20.9 and of 32768 58.6 / 78.8, 16 x 2 of 4096 27.0 / 23.5 and of 32768 70.6 / 101,
  // 16 x 8 of 4096 39.9 / 58.3 (bf16 cache 60.3 / 94.4).
  // Half of them too where segments cannot stay whole and the table is so narrow that a CTA's share is read in the time that a join takes: 16 x 2 of 4096 in a table of as many have 226 KB a CTA in
  // e4m3, 64 query heads 31.5 / 29.8 us; 452 KB in bf16 36.8 / 43.1.  (In a wider table the lengths decide, on the device.)
  // And fewer where a large batch's table leaves no room for their queries and partial states (plain FMAs, heads of 240 and 256).
  const long long segs = (long long)batch * G;
  const bool few = segs * 7 < ctas || (segs * 2 < ctas && segs * (double)positions * hd * 2 * bytes < (double)DA_SPARE_BYTES * ctas);
  for (int most = mma ? (q_f32 ? 8 : 16) / (hd < 256 && !few ? 1 : 2) : 8;; most /= 2) {
    p.chunks = (group + most - 1) / most;
    p.heads = (group + p.chunks - 1) / p.chunks;
    int own = 0;
    if (mma) {
      p.columns = hd < 256 && p.heads > (q_f32 ? 4 : 8) ? 16 : 8;
      p.groups = hd * bytes <= 128 ? 2 : 1;
      if (hd * bytes == 128 && bytes == 1 && p.columns == 8 && (long long)batch * G * p.chunks > 2 * ctas) p.groups = 1;
      p.warps = da_mma_warps(hd, bytes, p.columns, p.groups);
    } else {
      for (p.columns = 1; p.columns < p.heads;) p.columns *= 2;
      p.warps = da_fma_warps(hd, p.columns);
      own = p.columns * hd + 64;
    }
    if (most == 1 || da_smem_bytes(batch, p.warps, own, p.heads, hd) <= DA_SMEM) return p;
  }
}

cudaError_t launch_decode_attn(const DecodeAttn &a, int dtype, int fmt, cudaStream_t s) {
  DaArgs p{};
  p.a = a;
  p.page_shift = (a.cache.page_size & (a.cache.page_size - 1)) == 0 ? __builtin_ctz(a.cache.page_size) : -1;
  p.q_f32 = dtype == KV_F32;
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return e;
  const int ctas = std::min(sms, DA_MAX_CTAS);
  const DecodePlan plan = decode_attn_plan(p.q_f32, fmt, a.batch, a.H, a.cache.G, a.cache.hd, ctas, (long long)a.cache.pages_per_seq * a.cache.page_size);
  p.group = a.H / a.cache.G;
  auto deal_of = [&](int heads) {
    const int chunks = (p.group + heads - 1) / heads;
    return DaDeal{heads, chunks, a.cache.G * chunks, a.batch * a.cache.G * chunks, 0};
  };
  p.deal = deal_of(plan.heads);
  p.halves = deal_of((plan.heads + 1) / 2);
  p.halve_below = DA_HALVE_BELOW;
  p.count = (unsigned *)a.workspace;
  p.part = (float *)((char *)a.workspace + DA_COUNT_BYTES);
  return plan.groups ? launch_decode_mma(p, fmt, plan, ctas, s) : launch_decode_fma(p, fmt, ctas, s);
}

}  // namespace spec
