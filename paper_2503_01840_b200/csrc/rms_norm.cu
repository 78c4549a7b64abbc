// Root-mean-square norm: s = x + r, y = s u w with u = 1 / sqrt(mean s^2 + eps); its gradient ds = u (g w - h mean(g w h)), dw = sum over rows of g h, h = s u.
// The norm is taken of the sum in 32 bits, before it is rounded to the residual stream's type.
#include "rms_norm.cuh"

#include <algorithm>

#include "vec.cuh"

namespace spec {

using std::max;
using std::min;

template <int FMT> __device__ __forceinline__ void store_code(void *y, long long i, float v) { ((uint8_t *)y)[i] = (uint8_t)kv_encode4<FMT>(v, 0.0f, 0.0f, 0.0f); }

// ---------------------------------------------------------------- any width, stride and alignment: a block a row, which it reads again for each step
__global__ void __launch_bounds__(256) rms_norm_any_kernel(RmsNorm a) {
  pdl_wait();
  pdl_trigger();
  __shared__ float room[32];
  const long long row = blockIdx.x;
  const int tid = threadIdx.x;
  auto at = [&](int c) {
    const float x = load_as_f32(a.x, a.x_type, row * a.x_rs + c);
    return a.res ? x + load_as_f32(a.res, a.r_type, row * a.r_rs + c) : x;
  };
  float ss = 0.0f;
  for (int c = tid; c < a.dim; c += 256) {
    const float s = at(c);
    ss = fmaf(s, s, ss);
  }
  const float u = rsqrtf(block_sum(ss, room) / a.dim + a.eps);
  auto normed = [&](int c) { return at(c) * u * load_as_f32(a.gain, a.g_type, c); };
  if (a.y_type == KV_F32 || a.y_type == KV_BF16) {
    for (int c = tid; c < a.dim; c += 256) {
      const float s = at(c);
      store_from_f32(a.y, a.y_type, row * a.y_rs + c, s * u * load_as_f32(a.gain, a.g_type, c));
      if (a.res) store_from_f32(a.sum, a.r_type, row * a.s_rs + c, s);
    }
    return;
  }
  // scales: a warp for each group, or all of them for the row
  const int lane = tid & 31, groups = (a.dim + a.group - 1) / a.group;
  const bool whole = groups == 1;
  for (int i = whole ? 0 : tid >> 5; i < groups; i += 8) {
    const int c0 = i * a.group, c1 = min(a.dim, c0 + a.group), first = whole ? tid : lane, step = whole ? 256 : 32;
    uint32_t top = 0;
    for (int c = c0 + first; c < c1; c += step) top = max(top, __float_as_uint(normed(c)) & 0x7fffffffu);
    top = whole ? block_max(top, room) : __reduce_max_sync(0xffffffffu, top);
    const float scale = a.y_type == KV_E4M3 ? kv_scale<KV_E4M3>(top) : kv_scale<KV_INT8>(top), inv = 1.0f / scale;
    for (int c = c0 + first; c < c1; c += step) {
      const float v = normed(c) * inv;
      if (a.y_type == KV_E4M3) store_code<KV_E4M3>(a.y, row * a.y_rs + c, v);
      else store_code<KV_INT8>(a.y, row * a.y_rs + c, v);
      if (a.res) store_from_f32(a.sum, a.r_type, row * a.s_rs + c, at(c));
    }
    if (first == 0) a.scale[row * groups + i] = scale;
  }
}

// ---------------------------------------------------------------- rows of whole eights
// Widths of whole eights up to 16384, aligned to 16 bytes.  A thread has N times eight neighbours in every row that its block takes in turn; rows come through a ring of STAGES in shared
// memory, in which a thread's part is its own, so that the next rows are under way while one is summed, without a register for them and with one barrier a row.
// Up to 256 columns a warp has a row, and nothing to wait for.  In 8 bits a scale's group is part of a warp's 256 columns, or the row.
// Bytes bound it: 16384 rows of 4096 in bf16 with the residual 97 us (5.5 TB/s, 85 % of a copy's rate), 8192 rows of 8192 without 46 us (5.8 TB/s); to e4m3 84 us (5.6 TB/s) with the scales'
// and codes' instructions close to them.  A block a row with the row in registers 106 / 82 / 125 us; half as many blocks an SM 98 / 61 / 107; two or four stages 98 / 47 / 87 and 98 / 49 / 90; at 4096 columns
// eight neighbours a thread 101 / - / 87, 32 of them 95 / 46 / 88.
constexpr int STAGES = 3;

template <int FMT> __device__ __forceinline__ uint2 codes_of(float (&y)[8], float inv) {
#pragma unroll
  for (int k = 0; k < 8; k += 2) unpair(mul(pair(y[k], y[k + 1]), pair(inv, inv)), y[k], y[k + 1]);
  return make_uint2(kv_encode4<FMT>(y[0], y[1], y[2], y[3]), kv_encode4<FMT>(y[4], y[5], y[6], y[7]));
}
// of a warp's lanes, and of a block's warps through `room`
__device__ __forceinline__ float sum_of(float v, float *room, bool block) {
#pragma unroll
  for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  if (!block) return v;
  const int lane = threadIdx.x & 31;
  if (lane == 0) room[threadIdx.x >> 5] = v;
  __syncthreads();
  v = (lane & 15) < (blockDim.x >> 5) ? room[lane & 15] : 0.0f;      // both halves of the warp alike
#pragma unroll
  for (int d = 8; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}

// What follows the sum: v is the residual sum, w the gain; thread t of `of_row` threads of the row
template <int N> __device__ __forceinline__ void norm_out(const RmsNorm &a, long long row, int t, int of_row, float (&v)[N][8], const float (&w)[N][8], float u, float *room, bool block) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int i = 0; i < N; i++)
#pragma unroll
    for (int k = 0; k < 8; k += 2) unpair(mul(mul(pair(v[i][k], v[i][k + 1]), pair(u, u)), pair(w[i][k], w[i][k + 1])), v[i][k], v[i][k + 1]);
  if (a.y_type == KV_F32 || a.y_type == KV_BF16) {
#pragma unroll
    for (int i = 0; i < N; i++) {
      const int c = (i * of_row + t) * 8;
      if (c >= a.dim) continue;
      if (a.y_type == KV_F32) store8((float *)a.y + row * a.y_rs + c, v[i]);
      else store8((bf16 *)a.y + row * a.y_rs + c, v[i]);
    }
    return;
  }
  const bool whole = a.group >= a.dim;
  const int shift = whole ? 0 : 31 - __clz(a.group), groups = whole ? 1 : (a.dim + a.group - 1) >> shift, lanes = a.group >> 3;      // lanes of a group: 4 to 32
  uint32_t top[N];                                       // bits of the largest magnitude: NaN counts as the largest of all
#pragma unroll
  for (int i = 0; i < N; i++) {
    float m = 0.0f;
#pragma unroll
    for (int k = 0; k < 8; k++) asm("max.NaN.xorsign.abs.f32 %0, %0, %1;" : "+f"(m) : "f"(v[i][k]));      // up to a sign
    top[i] = __float_as_uint(m) & 0x7fffffffu;
  }
  if (whole) {
#pragma unroll
    for (int i = 1; i < N; i++) top[0] = max(top[0], top[i]);
    top[0] = __reduce_max_sync(0xffffffffu, top[0]);
    if (block) {
      if (lane == 0) room[16 + (threadIdx.x >> 5)] = __uint_as_float(top[0]);
      __syncthreads();
      top[0] = __reduce_max_sync(0xffffffffu, lane < (blockDim.x >> 5) ? __float_as_uint(room[16 + (lane & 15)]) : 0u);
    }
#pragma unroll
    for (int i = 1; i < N; i++) top[i] = top[0];
  } else {
#pragma unroll
    for (int i = 0; i < N; i++)
      for (int d = 1; d < lanes; d <<= 1) top[i] = max(top[i], __shfl_xor_sync(0xffffffffu, top[i], d));
  }
#pragma unroll
  for (int i = 0; i < N; i++) {
    const int c = (i * of_row + t) * 8;
    if (c >= a.dim) continue;
    const float scale = a.y_type == KV_E4M3 ? kv_scale<KV_E4M3>(top[i]) : kv_scale<KV_INT8>(top[i]), inv = 1.0f / scale;
    *(uint2 *)((uint8_t *)a.y + row * a.y_rs + c) = a.y_type == KV_E4M3 ? codes_of<KV_E4M3>(v[i], inv) : codes_of<KV_INT8>(v[i], inv);
    if (whole ? i == 0 && t == 0 : (t & (lanes - 1)) == 0) a.scale[row * groups + (whole ? 0 : c >> shift)] = scale;
  }
}
template <int N> __device__ __forceinline__ void gain_of(const RmsNorm &a, int t, int of_row, float (&w)[N][8]) {
#pragma unroll
  for (int i = 0; i < N; i++) {
    const int c = (i * of_row + t) * 8;
#pragma unroll
    for (int k = 0; k < 8; k++) w[i][k] = 0.0f;
    if (c >= a.dim) continue;
    if (a.g_type == KV_F32) load8((const float *)a.gain + c, w[i]);
    else load8((const bf16 *)a.gain + c, w[i]);
  }
}
template <int N> __device__ __forceinline__ float square_of(const float (&v)[N][8]) {
  Pair ss = pair(0.0f, 0.0f);
#pragma unroll
  for (int i = 0; i < N; i++)
#pragma unroll
    for (int k = 0; k < 8; k += 2) {
      const Pair p = pair(v[i][k], v[i][k + 1]);
      ss = fma(p, p, ss);
    }
  float even, odd;
  unpair(ss, even, odd);
  return even + odd;
}

template <typename TX, typename TR>
__global__ void __launch_bounds__(128) rms_norm_warp_kernel(const __grid_constant__ RmsNorm a) {
  pdl_wait();
  pdl_trigger();
  const int t = threadIdx.x & 31, c = t * 8;
  const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (row >= a.rows) return;
  float v[1][8] = {}, w[1][8];
  if (c < a.dim) {
    Raw8<TX> x;
    Raw8<TR> r;
    x.take((const TX *)a.x + row * a.x_rs + c);
    if (a.res) r.take((const TR *)a.res + row * a.r_rs + c);
    x.floats(v[0]);
    if (a.res) {
      float y[8];
      r.floats(y);
#pragma unroll
      for (int k = 0; k < 8; k++) v[0][k] += y[k];
      store8((TR *)a.sum + row * a.s_rs + c, v[0]);
    }
  }
  gain_of<1>(a, t, 32, w);
  norm_out<1>(a, row, t, 32, v, w, rsqrtf(sum_of(square_of<1>(v), nullptr, false) / a.dim + a.eps), nullptr, false);
}

template <typename TX, typename TR, int N>
__global__ void __launch_bounds__(512) rms_norm_kernel(const __grid_constant__ RmsNorm a) {
  pdl_wait();
  pdl_trigger();
  extern __shared__ __align__(16) char ring[];
  __shared__ float room[2][32];
  const int t = threadIdx.x, of_row = blockDim.x;
  TX *const xs = (TX *)ring;                             // [stages][dim]
  TR *const rs = (TR *)(ring + (size_t)STAGES * a.dim * sizeof(TX));
  auto ask = [&](long long row, int stage) {
    if (row < a.rows)
#pragma unroll
      for (int i = 0; i < N; i++) {
        const int c = (i * of_row + t) * 8;
        if (c >= a.dim) continue;
        copy8(xs + stage * a.dim + c, (const TX *)a.x + row * a.x_rs + c);
        if (a.res) copy8(rs + stage * a.dim + c, (const TR *)a.res + row * a.r_rs + c);
      }
    copies_commit();
  };
  long long row = blockIdx.x;
#pragma unroll
  for (int k = 0; k < STAGES; k++) ask(row + (long long)k * gridDim.x, k);
  float w[N][8];
  gain_of<N>(a, t, of_row, w);
  const float over_dim = 1.0f / a.dim;
  for (int stage = 0, turn = 0; row < a.rows; row += gridDim.x, turn ^= 1) {
    copies_but<STAGES - 1>();
    float v[N][8];
#pragma unroll
    for (int i = 0; i < N; i++) {
      const int c = (i * of_row + t) * 8;
#pragma unroll
      for (int k = 0; k < 8; k++) v[i][k] = 0.0f;
      if (c >= a.dim) continue;
      load8(xs + stage * a.dim + c, v[i]);
      if (!a.res) continue;
      float y[8];
      load8(rs + stage * a.dim + c, y);
#pragma unroll
      for (int k = 0; k < 8; k++) v[i][k] += y[k];
      store8((TR *)a.sum + row * a.s_rs + c, v[i]);
    }
    const float u = rsqrtf(fmaf(sum_of(square_of<N>(v), room[turn], true), over_dim, a.eps));
    ask(row + (long long)STAGES * gridDim.x, stage);
    norm_out<N>(a, row, t, of_row, v, w, u, room[turn], true);
    stage = stage == STAGES - 1 ? 0 : stage + 1;
  }
}

static size_t bytes_of(int type) { return type == KV_F32 ? 4 : type == KV_BF16 ? 2 : 1; }
static bool rows_aligned(const void *p, long long row_stride, int type, int rows, size_t to = 16) {
  return ((reinterpret_cast<uintptr_t>(p) | (rows > 1 ? (uintptr_t)(row_stride * (long long)bytes_of(type)) : 0)) & (to - 1)) == 0;
}

template <typename TX, typename TR, int N> static cudaError_t rms_norm_by_ring(const RmsNorm &a, cudaStream_t s) {
  static SmemLimit limit;
  const int threads = (a.dim + 256 * N - 1) / (256 * N) * 32;
  const size_t smem = (size_t)STAGES * a.dim * (sizeof(TX) + (a.res ? sizeof(TR) : 0));
  if (smem > 46 << 10 && !limit.ensure(rms_norm_kernel<TX, TR, N>, (int)smem)) return cudaErrorInvalidValue;
  const int per_sm = max(1, min(min((int)((227 << 10) / (smem + 1280)), 16), (N == 1 ? 1536 : N == 2 ? 1024 : 512) / threads));      // as many threads as registers allow
  return launch_k(rms_norm_kernel<TX, TR, N>, dim3(min(a.rows, 148 * per_sm)), dim3(threads), smem, s, a);
}
template <typename TX, typename TR> static cudaError_t rms_norm_in_eights(const RmsNorm &a, cudaStream_t s) {
  if (a.dim <= 256) return launch_k(rms_norm_warp_kernel<TX, TR>, dim3((a.rows + 3) / 4), dim3(128), 0, s, a);
  if (a.dim <= 1024) return rms_norm_by_ring<TX, TR, 1>(a, s);
  if (a.dim <= 8192) return rms_norm_by_ring<TX, TR, 2>(a, s);
  return rms_norm_by_ring<TX, TR, 4>(a, s);
}

cudaError_t launch_rms_norm(const RmsNorm &a, cudaStream_t s) {
  const bool eight = kv_is_8bit(a.y_type);
  const size_t stage = (size_t)a.dim * (bytes_of(a.x_type) + (a.res ? bytes_of(a.r_type) : 0));
  const bool pieces = a.dim % 8 == 0 && a.dim <= 16384 && STAGES * stage <= 220 << 10 && rows_aligned(a.x, a.x_rs, a.x_type, a.rows) && rows_aligned(a.gain, 0, a.g_type, 1) &&
                      (!a.res || (rows_aligned(a.res, a.r_rs, a.r_type, a.rows) && rows_aligned(a.sum, a.s_rs, a.r_type, a.rows))) &&
                      rows_aligned(a.y, a.y_rs, a.y_type, a.rows, eight ? 8 : 16) &&
                      (!eight || a.group >= a.dim || a.group == 32 || a.group == 64 || a.group == 128 || a.group == 256);
  if (!pieces) return launch_k(rms_norm_any_kernel, dim3(a.rows), dim3(256), 0, s, a);
  const bool r = a.res && a.r_type == KV_BF16;
  if (a.x_type == KV_F32) return r ? rms_norm_in_eights<float, bf16>(a, s) : rms_norm_in_eights<float, float>(a, s);
  return r || !a.res ? rms_norm_in_eights<bf16, bf16>(a, s) : rms_norm_in_eights<bf16, float>(a, s);
}

// ---------------------------------------------------------------- gradient
// Blocks take rows in turn and keep their own sums for the gain's gradient, which the next launch adds up in the blocks' order.
struct GradPlan {
  int n, threads, stages, blocks;      // eights of a thread, threads of a block, rows of the ring
};
// row: bytes of a row of all inputs, of which as many are under way as there is shared memory for (2 to 4 in a block)
static GradPlan grad_plan(int rows, int dim, size_t row) {
  const int n = dim <= 1024 ? 1 : 2, threads = min(512, (dim + 256 * n - 1) / (256 * n) * 32);
  const int per_sm = (int)max<size_t>(1, min<size_t>(max(1, min(16, (n == 1 ? 1024 : 512) / threads)), (220 << 10) / (2 * row + 1280)));
  return {n, threads, (int)max<size_t>(2, min<size_t>(4, ((220 << 10) / per_sm - 1280) / row)), min(rows, 148 * per_sm)};
}
__global__ void __launch_bounds__(256) rms_norm_grad_any_kernel(RmsNormGrad a) {
  pdl_wait();
  pdl_trigger();
  __shared__ float room[32];
  float *const part = a.part + (long long)blockIdx.x * a.dim;
  for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
    float ss = 0.0f, dot = 0.0f;
    for (int c = threadIdx.x; c < a.dim; c += 256) {
      const float x = load_as_f32(a.x, a.x_type, row * a.x_rs + c), gw = load_as_f32(a.g, a.g_type, row * a.g_rs + c) * load_as_f32(a.gain, a.w_type, c);
      ss = fmaf(x, x, ss), dot = fmaf(gw, x, dot);
    }
    const float u = rsqrtf(block_sum(ss, room) / a.dim + a.eps), along = block_sum(dot, room) / a.dim * u * u;
    for (int c = threadIdx.x; c < a.dim; c += 256) {
      const float x = load_as_f32(a.x, a.x_type, row * a.x_rs + c), g = load_as_f32(a.g, a.g_type, row * a.g_rs + c);
      float d = u * fmaf(-x, along, g * load_as_f32(a.gain, a.w_type, c));
      if (a.carried) d += load_as_f32(a.carried, a.c_type, row * a.c_rs + c);
      store_from_f32(a.dx, a.d_type, row * a.d_rs + c, d);
      part[c] = row == blockIdx.x ? g * (x * u) : fmaf(g, x * u, part[c]);
    }
  }
}

// The gradient's rows come through a ring as the norm's do.  Bytes bound it: 8192 rows of 4096 in bf16 with what is carried 43 us (6.2 TB/s, 95 % of a copy's rate) and 6 us for the second
// launch, 52 us in all; with a row in registers and the next one's loads 92 us, with eight neighbours a thread 59.
template <typename TG, typename TX, typename TD, int N>
__global__ void __launch_bounds__(512) rms_norm_grad_kernel(const __grid_constant__ RmsNormGrad a, int stages) {
  pdl_wait();
  pdl_trigger();
  extern __shared__ __align__(16) char ring[];
  __shared__ float2 room[2][16];
  const int t = threadIdx.x, of_row = blockDim.x, lane = t & 31, warp = t >> 5, warps = of_row >> 5;
  TG *const gs = (TG *)ring;                             // [stages][dim]
  TX *const xs = (TX *)(ring + (size_t)stages * a.dim * sizeof(TG));
  TD *const cs = (TD *)(ring + (size_t)stages * a.dim * (sizeof(TG) + sizeof(TX)));
  auto ask = [&](long long row, int stage) {
    if (row < a.rows)
#pragma unroll
      for (int i = 0; i < N; i++) {
        const int c = (i * of_row + t) * 8;
        if (c >= a.dim) continue;
        copy8(gs + stage * a.dim + c, (const TG *)a.g + row * a.g_rs + c);
        copy8(xs + stage * a.dim + c, (const TX *)a.x + row * a.x_rs + c);
        if (a.carried) copy8(cs + stage * a.dim + c, (const TD *)a.carried + row * a.c_rs + c);
      }
    copies_commit();
  };
  long long row = blockIdx.x;
  for (int k = 0; k < stages; k++) ask(row + (long long)k * gridDim.x, k);
  float w[N][8], sum[N][8] = {};
  const float over_dim = 1.0f / a.dim;
#pragma unroll
  for (int i = 0; i < N; i++) {
    const int c = (i * of_row + t) * 8;
#pragma unroll
    for (int k = 0; k < 8; k++) w[i][k] = 0.0f;
    if (c >= a.dim) continue;
    if (a.w_type == KV_F32) load8((const float *)a.gain + c, w[i]);
    else load8((const bf16 *)a.gain + c, w[i]);
  }
  for (int stage = 0, turn = 0; row < a.rows; row += gridDim.x, turn ^= 1) {
    if (stages == 2) copies_but<1>();
    else if (stages == 3) copies_but<2>();
    else copies_but<3>();
    Raw8<TG> g[N];
    Raw8<TX> x[N];
    float ss = 0.0f, dot = 0.0f;
#pragma unroll
    for (int i = 0; i < N; i++) {
      const int c = (i * of_row + t) * 8;
      if (c >= a.dim) continue;
      g[i].take(gs + stage * a.dim + c);
      x[i].take(xs + stage * a.dim + c);
      float gr[8], xr[8];
      g[i].floats(gr);
      x[i].floats(xr);
#pragma unroll
      for (int k = 0; k < 8; k++) ss = fmaf(xr[k], xr[k], ss), dot = fmaf(gr[k] * w[i][k], xr[k], dot);
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d), dot += __shfl_xor_sync(0xffffffffu, dot, d);
    if (lane == 0) room[turn][warp] = make_float2(ss, dot);
    __syncthreads();
    const float2 some = (lane & 15) < warps ? room[turn][lane & 15] : make_float2(0.0f, 0.0f);      // both halves of the warp alike
    ss = some.x, dot = some.y;
#pragma unroll
    for (int d = 8; d; d >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d), dot += __shfl_xor_sync(0xffffffffu, dot, d);
    const float u = rsqrtf(fmaf(ss, over_dim, a.eps)), along = dot * over_dim * u * u;
#pragma unroll
    for (int i = 0; i < N; i++) {
      const int c = (i * of_row + t) * 8;
      if (c >= a.dim) continue;
      float gr[8], xr[8], d[8] = {};
      g[i].floats(gr);
      x[i].floats(xr);
      if (a.carried) load8(cs + stage * a.dim + c, d);
#pragma unroll
      for (int k = 0; k < 8; k++) {
        sum[i][k] = fmaf(gr[k], xr[k] * u, sum[i][k]);
        d[k] = fmaf(u, fmaf(-xr[k], along, gr[k] * w[i][k]), d[k]);
      }
      store8((TD *)a.dx + row * a.d_rs + c, d);
    }
    ask(row + (long long)stages * gridDim.x, stage);
    stage = stage == stages - 1 ? 0 : stage + 1;
  }
#pragma unroll
  for (int i = 0; i < N; i++) {
    const int c = (i * of_row + t) * 8;
    if (c < a.dim) store8(a.part + (long long)blockIdx.x * a.dim + c, sum[i]);
  }
}

// 32 columns a block; its warps add up runs of the blocks' sums, and each of them then one column's 32
__global__ void __launch_bounds__(1024) rms_norm_gain_kernel(RmsNormGrad a, int blocks) {
  pdl_wait();
  pdl_trigger();
  __shared__ float some[32][33];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = blockIdx.x * 32 + lane, per = (blocks + 31) / 32;
  float sum = 0.0f;
  if (c < a.dim)
#pragma unroll 8
    for (int b = w * per; b < min(blocks, (w + 1) * per); b++) sum += a.part[(long long)b * a.dim + c];
  some[w][lane] = sum;
  __syncthreads();
  sum = some[lane][w];
#pragma unroll
  for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  if (lane == 0 && blockIdx.x * 32 + w < a.dim) store_from_f32(a.dgain, a.w_type, blockIdx.x * 32 + w, sum);
}

size_t rms_norm_grad_scratch_bytes(int rows, int dim) { return (size_t)grad_plan(rows, dim, 4 * (size_t)dim).blocks * dim * sizeof(float); }      // with one input of 32 bits: as many blocks as any has

template <typename TG, typename TX, typename TD, int N> static cudaError_t rms_norm_grad_by_ring(const RmsNormGrad &a, const GradPlan &p, size_t row, cudaStream_t s) {
  static SmemLimit limit;
  const size_t smem = p.stages * row;
  if (smem > 46 << 10 && !limit.ensure(rms_norm_grad_kernel<TG, TX, TD, N>, (int)smem)) return cudaErrorInvalidValue;
  return launch_k(rms_norm_grad_kernel<TG, TX, TD, N>, dim3(p.blocks), dim3(p.threads), smem, s, a, p.stages);
}
template <typename TG, typename TX> static cudaError_t rms_norm_grad_in_eights(const RmsNormGrad &a, const GradPlan &p, size_t row, cudaStream_t s) {
  if (a.d_type == KV_F32) return p.n == 1 ? rms_norm_grad_by_ring<TG, TX, float, 1>(a, p, row, s) : rms_norm_grad_by_ring<TG, TX, float, 2>(a, p, row, s);
  return p.n == 1 ? rms_norm_grad_by_ring<TG, TX, bf16, 1>(a, p, row, s) : rms_norm_grad_by_ring<TG, TX, bf16, 2>(a, p, row, s);
}

cudaError_t launch_rms_norm_grad(const RmsNormGrad &a, cudaStream_t s) {
  const size_t row = (size_t)a.dim * (bytes_of(a.g_type) + bytes_of(a.x_type) + (a.carried ? bytes_of(a.d_type) : 0));
  GradPlan p = grad_plan(a.rows, a.dim, row);
  if (a.rows) {
    // what is carried has the output's type, as it has where both are of the residual stream
    const bool pieces = a.dim % 8 == 0 && a.dim <= 8192 && 2 * row <= 220 << 10 && rows_aligned(a.g, a.g_rs, a.g_type, a.rows) && rows_aligned(a.x, a.x_rs, a.x_type, a.rows) &&
                        rows_aligned(a.gain, 0, a.w_type, 1) && rows_aligned(a.dx, a.d_rs, a.d_type, a.rows) &&
                        (!a.carried || (a.c_type == a.d_type && rows_aligned(a.carried, a.c_rs, a.c_type, a.rows)));
    cudaError_t e;
    if (!pieces) e = launch_k(rms_norm_grad_any_kernel, dim3(p.blocks), dim3(256), 0, s, a);
    else if (a.g_type == KV_F32) e = a.x_type == KV_F32 ? rms_norm_grad_in_eights<float, float>(a, p, row, s) : rms_norm_grad_in_eights<float, bf16>(a, p, row, s);
    else e = a.x_type == KV_F32 ? rms_norm_grad_in_eights<bf16, float>(a, p, row, s) : rms_norm_grad_in_eights<bf16, bf16>(a, p, row, s);
    if (e) return e;
  }
  return launch_k(rms_norm_gain_kernel, dim3((a.dim + 31) / 32), dim3(1024), 0, s, a, a.rows ? p.blocks : 0);
}

}  // namespace spec
