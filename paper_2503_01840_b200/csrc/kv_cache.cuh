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
// Tokens and heads of a block, of `heads` heads a token, `step` of which it rotates at a time
struct RopePlan { int per_block, heads; };
RopePlan rope_plan(int tokens, int heads, int step);
cudaError_t launch_rope_append(const RopeAppend &a, int dtype, int fmt, cudaStream_t s);

struct KvRead {
  KvCache cache;
  const int32_t *seq, *kvpos;
  int rows;
  void *k_out, *v_out;
  int32_t *status;
};
cudaError_t launch_kv_read(const KvRead &a, int fmt, int out_dtype, cudaStream_t s);

// Row (of hd elements; a pool has fewer than 2^31) of a cache position's first head, -1 where there is none; the heads follow page_size
// rows apart.
__device__ __forceinline__ int kv_row(const KvCache &c, int seq, int pos, int32_t *status, int row) {
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
  return page * c.G * c.page_size + (pos - at * c.page_size);
}

// Cosine and sine of position * frequency.  The angle is formed in 64 bits and brought to less than half a turn there: at position
// 10^5 a 32-bit product would be off by thousandths of a radian.  What is left is exact enough for the 32-bit functions.
__device__ __forceinline__ float2 rope_angle(const Rope &r, int pos, int pair) {
  const double turns = (double)pos * r.inv_freq[pair] * 0.15915494309189533576888376337251;      // 1 / (2 pi)
  float s, c;
  sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
  return make_float2(c * r.mscale, s * (r.mscale * r.sign));
}

// Conversions by pairs and quadruples: one to a type or from it at a time runs at a quarter of the rate or less, and is then what
// bounds a kernel that should be bound by its bytes.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *(const uint32_t *)&v;
}
// four elements; int8 by bits: 0x4b000000 | u is 2^23 + u
template <int FMT> struct Four;
template <> struct Four<KV_F32> { typedef uint4 raw; };
template <> struct Four<KV_BF16> { typedef uint2 raw; };
template <> struct Four<KV_E4M3> { typedef uint32_t raw; };
template <> struct Four<KV_INT8> { typedef uint32_t raw; };
__device__ __forceinline__ float4 kv_decode4(uint4 u) { return make_float4(__uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z), __uint_as_float(u.w)); }
__device__ __forceinline__ float4 kv_decode4(uint2 u) {
  return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16), __uint_as_float(u.y & 0xffff0000u));
}
// e4m3 by pairs to f16, which holds them all; straight from the halves of a word (through the type's struct the compiler takes pairs apart)
__device__ __forceinline__ void e4m3_to_f16(uint32_t u, uint32_t &lo, uint32_t &hi) {
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=r"(lo), "=r"(hi) : "r"(u));
}
template <int FMT> __device__ __forceinline__ float4 kv_decode4(uint32_t u) {
  if constexpr (FMT == KV_E4M3) {
    uint32_t a, b;
    e4m3_to_f16(u, a, b);
    const float2 x = __half22float2(*(const __half2 *)&a), y = __half22float2(*(const __half2 *)&b);
    return make_float4(x.x, x.y, y.x, y.y);
  } else {
    u ^= 0x80808080u;
    const float off = 8388736.0f;
    return make_float4(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7440)) - off, __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7441)) - off,
                       __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7442)) - off, __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7443)) - off);
  }
}
template <int FMT> __device__ __forceinline__ float4 kv_decode_four(typename Four<FMT>::raw u) {
  if constexpr (kv_is_8bit(FMT)) return kv_decode4<FMT>(u);
  else return kv_decode4(u);
}
// four numbers over their scale as codes, rounded to nearest even; what the product's own rounding puts past the largest becomes the
// largest.  int8: after y + 1.5 2^23 the integer stands in the low bits.
template <int FMT> __device__ __forceinline__ uint32_t kv_encode4(float a, float b, float c, float d) {
  if constexpr (FMT == KV_E4M3) {
    return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3) |
           (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3) << 16;
  } else {
    auto bits = [](float y) { return __float_as_uint(fminf(fmaxf(y, -127.0f), 127.0f) + 12582912.0f); };
    return __byte_perm(__byte_perm(bits(a), bits(b), 0x0040), __byte_perm(bits(c), bits(d), 0x0040), 0x5410);
  }
}
// The scale of a head whose largest magnitude has these bits.  An infinity or a NaN among its numbers makes it a NaN: whatever the codes are,
// the row then reads back as NaN.
template <int FMT> __device__ __forceinline__ float kv_scale(uint32_t top_bits) {
  const float amax = __uint_as_float(top_bits) * (1.0f / (FMT == KV_E4M3 ? 448.0f : 127.0f));
  return fmaf(amax, 0.0f, amax < KV_SCALE_FLOOR ? KV_SCALE_FLOOR : amax);
}

}  // namespace spec
