// Rotary positions and the paged key-value cache of bf16, fp32, e4m3 or int8 that the operators of kv_cache.cu write and read and
// attn_decode.cu attends to.
#pragma once
#include <cuda_fp8.h>

#include "common.cuh"

namespace spec {

enum { KV_F32 = 0, KV_BF16 = 1, KV_E4M3 = 2, KV_INT8 = 3 };
template <int FMT> struct KvElem;
template <> struct KvElem<KV_F32> { typedef float type; };
template <> struct KvElem<KV_BF16> { typedef bf16 type; };
template <> struct KvElem<KV_E4M3> { typedef uint8_t type; };
template <> struct KvElem<KV_INT8> { typedef int8_t type; };
constexpr bool kv_is_8bit(int fmt) { return fmt == KV_E4M3 || fmt == KV_INT8; }

// A scale is max(amax / top, 2^-120): its reciprocal is then finite for every row of finite numbers, one of zeros too.
constexpr float KV_SCALE_FLOOR = 7.52316384526264e-37f;
template <int FMT> constexpr float kv_top() { return FMT == KV_E4M3 ? 448.0f : 127.0f; }

// pools [num_pages][G][page_size][hd], scales [num_pages][G][page_size] (8-bit formats), table [n_seq][pages_per_seq]
struct KvCache {
  void *k, *v;
  float *ks, *vs;
  const int32_t *table;
  int n_seq, pages_per_seq, page_size, num_pages, G, hd;
};

struct Rope {
  const double *inv_freq;      // radians per position of each pair
  int half, interleaved;       // pairs; 0: dimension i with i + half, 1: 2 i with 2 i + 1
  float mscale, sign;          // factor on cosine and sine; -1 on the sine for the transposed rotation
};

// heads of one tensor: element (t, h, d) at p[t * ts + h * hs + d]
struct HeadView {
  const void *p;
  long long ts, hs;
};

// queries (or any heads that only turn): H heads of q into q_out; keys and values: cache.G heads each, if k is given
struct RopeAppend {
  HeadView q, k, v;
  void *q_out;
  long long qo_ts, qo_hs;
  int H, hd, tokens;
  const int32_t *seq, *pos, *kvpos;
  Rope rope;
  KvCache cache;
  int32_t *status;
};
cudaError_t launch_rope_append(const RopeAppend &a, int dtype, int fmt, cudaStream_t s);

struct KvRead {
  KvCache cache;
  const int32_t *seq, *kvpos;
  int rows;
  void *k_out, *v_out;
  int32_t *status;
};
cudaError_t launch_kv_read(const KvRead &a, int fmt, int out_dtype, cudaStream_t s);

// Row (of hd elements) of a cache position's first head, -1 where there is none; the heads follow page_size rows apart.
__device__ __forceinline__ long long kv_row(const KvCache &c, int seq, int pos, int32_t *status, int row) {
  if (seq < 0) return -1;
  const int at = pos / c.page_size;
  if (seq >= c.n_seq || pos < 0 || at >= c.pages_per_seq) {
    set_status(status, ST_BOUNDS, 60, row, seq >= c.n_seq ? seq : pos);
    return -1;
  }
  const int page = c.table[(size_t)seq * c.pages_per_seq + at];
  if (page < 0 || page >= c.num_pages) {
    set_status(status, ST_BOUNDS, 61, row, page);
    return -1;
  }
  return (long long)page * c.G * c.page_size + (pos - at * c.page_size);
}

// Cosine and sine of position * frequency.  The angle is formed in 64 bits and brought to less than half a turn there: at position
// 10^5 a 32-bit product would be off by thousandths of a radian.  What is left is exact enough for the 32-bit functions.
__device__ __forceinline__ float2 rope_angle(const Rope &r, int pos, int pair) {
  const double turns = (double)pos * r.inv_freq[pair] * 0.15915494309189533576888376337251;      // 1 / (2 pi)
  float s, c;
  sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
  return make_float2(c * r.mscale, s * (r.mscale * r.sign));
}

template <int FMT> __device__ __forceinline__ float kv_decode(typename KvElem<FMT>::type x) {
  if constexpr (FMT == KV_E4M3) return __half2float(__half(__nv_cvt_fp8_to_halfraw(x, __NV_E4M3)));
  else return (float)x;
}
// x / scale rounded to nearest even; numbers past the format's largest (the product's own rounding) become the largest
template <int FMT> __device__ __forceinline__ typename KvElem<FMT>::type kv_encode(float y) {
  if constexpr (FMT == KV_E4M3) return __nv_cvt_float_to_fp8(y, __NV_SATFINITE, __NV_E4M3);
  else return (int8_t)max(-127, min(127, __float2int_rn(y)));
}

}  // namespace spec
