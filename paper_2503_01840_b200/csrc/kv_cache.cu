// Rotary positions, writing keys and values into the paged cache (rotated and quantised on the way), reading positions of it back.
//
// Rotation: the pair (a, b) of a head's dimensions at position p becomes m (a cos t - b sin t, b cos t + a sin t), t = p f; its
// gradient is the transposed matrix, -t for t.  Quantisation, for each token and head: scale = max(amax / top, 2^-120) over the
// rotated 32-bit values, code = round(x / scale).  A row with an infinity or a NaN gets a scale that is infinite or NaN and
// reads back as NaN throughout.
#include "kv_cache.cuh"

namespace spec {

constexpr int ROPE_THREADS = 256, ROPE_MAX_HD = 256;

// ---------------------------------------------------------------- any head size up to 256, any strides
// A block per token, a warp per head: a lane holds dimensions lane, lane + 32, ...
template <typename T, int FMT>
__global__ void __launch_bounds__(ROPE_THREADS) rope_append_any_kernel(RopeAppend a) {
  pdl_wait();
  pdl_trigger();
  typedef typename KvElem<FMT>::type E;
  __shared__ float2 cs[ROPE_MAX_HD / 2];
  const int t = blockIdx.x, lane = threadIdx.x & 31, half = a.rope.half, hd = a.hd;
  if (half) {
    const int pos = a.pos[t];
    for (int i = threadIdx.x; i < half; i += ROPE_THREADS) cs[i] = rope_angle(a.rope, pos, i);
  }
  __shared__ long long row0;
  if (threadIdx.x == 0) row0 = a.k.p ? kv_row(a.cache, a.seq[t], a.kvpos[t], a.status, t) : -1;
  __syncthreads();
  const int G = a.k.p ? a.cache.G : 0;
  for (int i = threadIdx.x >> 5; i < a.H + 2 * G; i += ROPE_THREADS / 32) {
    const int kind = i < a.H ? 0 : i < a.H + G ? 1 : 2, h = kind == 0 ? i : kind == 1 ? i - a.H : i - a.H - G;
    if (kind && row0 < 0) continue;
    const HeadView &src = kind == 0 ? a.q : kind == 1 ? a.k : a.v;
    const T *x = (const T *)src.p + t * src.ts + h * src.hs;
    float y[ROPE_MAX_HD / 32];
    uint32_t top = 0;                                    // bits of the largest magnitude: NaN counts as the largest of all
#pragma unroll
    for (int j = 0; j < ROPE_MAX_HD / 32; j++) {
      const int d = lane + j * 32;
      if (d >= hd) continue;
      const float v = to_f32(x[d]);
      y[j] = v;
      if (kind < 2 && d < 2 * half) {
        const bool second = a.rope.interleaved ? d & 1 : d >= half;
        const float2 c = cs[a.rope.interleaved ? d >> 1 : second ? d - half : d];
        const float w = to_f32(x[a.rope.interleaved ? d ^ 1 : second ? d - half : d + half]);
        y[j] = second ? fmaf(v, c.x, w * c.y) : fmaf(v, c.x, -(w * c.y));
      }
      top = max(top, __float_as_uint(y[j]) & 0x7fffffffu);
    }
    __syncwarp();                                        // the output may be the input
    if (kind == 0) {
      T *o = (T *)a.q_out + t * a.qo_ts + h * a.qo_hs;
#pragma unroll
      for (int j = 0; j < ROPE_MAX_HD / 32; j++)
        if (lane + j * 32 < hd) o[lane + j * 32] = from_f32<T>(y[j]);
      continue;
    }
    const long long row = row0 + (long long)h * a.cache.page_size;
    E *o = (E *)(kind == 1 ? a.cache.k : a.cache.v) + row * hd;
    if constexpr (kv_is_8bit(FMT)) {
      const float amax = __uint_as_float(__reduce_max_sync(0xffffffffu, top)) * (1.0f / kv_top<FMT>());
      const float scale = amax < KV_SCALE_FLOOR ? KV_SCALE_FLOOR : amax, inv = 1.0f / scale;
#pragma unroll
      for (int j = 0; j < ROPE_MAX_HD / 32; j++)
        if (lane + j * 32 < hd) o[lane + j * 32] = kv_encode<FMT>(y[j] * inv);
      if (lane == 0) (kind == 1 ? a.cache.ks : a.cache.vs)[row] = scale;
    } else {
#pragma unroll
      for (int j = 0; j < ROPE_MAX_HD / 32; j++)
        if (lane + j * 32 < hd) o[lane + j * 32] = from_f32<E>(y[j]);
    }
  }
}

template <typename T, int FMT> static cudaError_t rope_append(const RopeAppend &a, cudaStream_t s) {
  return launch_k(rope_append_any_kernel<T, FMT>, dim3(a.tokens), dim3(ROPE_THREADS), 0, s, a);
}

cudaError_t launch_rope_append(const RopeAppend &a, int dtype, int fmt, cudaStream_t s) {
  if (dtype == KV_F32) return fmt == KV_E4M3 ? rope_append<float, KV_E4M3>(a, s) : fmt == KV_INT8 ? rope_append<float, KV_INT8>(a, s) : rope_append<float, KV_F32>(a, s);
  return fmt == KV_E4M3 ? rope_append<bf16, KV_E4M3>(a, s) : fmt == KV_INT8 ? rope_append<bf16, KV_INT8>(a, s) : rope_append<bf16, KV_BF16>(a, s);
}

// ---------------------------------------------------------------- reading back
// A block per row: row r of the output is position kvpos[r] of sequence seq[r], zeros where there is none.
template <int FMT, typename T>
__global__ void __launch_bounds__(256) kv_read_any_kernel(KvRead a) {
  pdl_wait();
  pdl_trigger();
  typedef typename KvElem<FMT>::type E;
  const int r = blockIdx.x, hd = a.cache.hd, n = a.cache.G * hd;
  __shared__ long long row0;
  if (threadIdx.x == 0) row0 = kv_row(a.cache, a.seq[r], a.kvpos[r], a.status, r);
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * n; i += 256) {
    const int kv = i >= n, e = i - kv * n, h = e / hd;
    float x = 0.0f;
    if (row0 >= 0) {
      const long long row = row0 + (long long)h * a.cache.page_size;
      x = kv_decode<FMT>(((const E *)(kv ? a.cache.v : a.cache.k))[row * hd + (e - h * hd)]);
      if constexpr (kv_is_8bit(FMT)) x *= (kv ? a.cache.vs : a.cache.ks)[row];
    }
    ((T *)(kv ? a.v_out : a.k_out))[(size_t)r * n + e] = from_f32<T>(x);
  }
}

template <int FMT> static cudaError_t kv_read(const KvRead &a, int out_dtype, cudaStream_t s) {
  if (out_dtype == KV_F32) return launch_k(kv_read_any_kernel<FMT, float>, dim3(a.rows), dim3(256), 0, s, a);
  return launch_k(kv_read_any_kernel<FMT, bf16>, dim3(a.rows), dim3(256), 0, s, a);
}

cudaError_t launch_kv_read(const KvRead &a, int fmt, int out_dtype, cudaStream_t s) {
  return fmt == KV_F32 ? kv_read<KV_F32>(a, out_dtype, s) : fmt == KV_BF16 ? kv_read<KV_BF16>(a, out_dtype, s)
       : fmt == KV_E4M3 ? kv_read<KV_E4M3>(a, out_dtype, s) : kv_read<KV_INT8>(a, out_dtype, s);
}

}  // namespace spec
