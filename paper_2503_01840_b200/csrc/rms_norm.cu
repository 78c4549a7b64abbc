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

// ---------------------------------------------------------------- rows held in registers
// Widths of whole eights up to 16384, aligned to 16 bytes: every thread has N times eight neighbours, of which the row has its threads or, up to 1024 columns, a warp.  Each
// input is read once and all of it is asked for before the first sum.  In 8 bits a scale's group is part of a warp's 256 columns, or the row.
template <int FMT> __device__ __forceinline__ uint2 codes_of(const float (&y)[8], float inv) {
  return make_uint2(kv_encode4<FMT>(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv), kv_encode4<FMT>(y[4] * inv, y[5] * inv, y[6] * inv, y[7] * inv));
}

template <typename TX, typename TR, int N, bool WARP>
__global__ void __launch_bounds__(512) rms_norm_kernel(const __grid_constant__ RmsNorm a) {
  pdl_wait();
  pdl_trigger();
  __shared__ float room[2][16];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, of_row = WARP ? 32 : blockDim.x, t = WARP ? lane : threadIdx.x;
  const long long row = WARP ? (long long)blockIdx.x * (blockDim.x >> 5) + warp : blockIdx.x;
  if (WARP && row >= a.rows) return;
  const TX *const x = (const TX *)a.x + row * a.x_rs;
  float v[N][8], w[N][8];
#pragma unroll
  for (int i = 0; i < N; i++) {
    const int c = (i * of_row + t) * 8;
    if (c < a.dim) {
      load8(x + c, v[i]);
      if (a.g_type == KV_F32) load8((const float *)a.gain + c, w[i]);
      else load8((const bf16 *)a.gain + c, w[i]);
    } else {
#pragma unroll
      for (int k = 0; k < 8; k++) v[i][k] = w[i][k] = 0.0f;
    }
  }
  if (a.res) {
    float r[N][8];
#pragma unroll
    for (int i = 0; i < N; i++) {
      const int c = (i * of_row + t) * 8;
      if (c < a.dim) load8((const TR *)a.res + row * a.r_rs + c, r[i]);
    }
#pragma unroll
    for (int i = 0; i < N; i++) {
      const int c = (i * of_row + t) * 8;
      if (c >= a.dim) continue;
#pragma unroll
      for (int k = 0; k < 8; k++) v[i][k] += r[i][k];
      store8((TR *)a.sum + row * a.s_rs + c, v[i]);
    }
  }
  float ss = 0.0f;
#pragma unroll
  for (int i = 0; i < N; i++)
#pragma unroll
    for (int k = 0; k < 8; k++) ss = fmaf(v[i][k], v[i][k], ss);
#pragma unroll
  for (int d = 16; d; d >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d);
  if (!WARP) {
    if (lane == 0) room[0][warp] = ss;
    __syncthreads();
    ss = lane < (blockDim.x >> 5) ? room[0][lane & 15] : 0.0f;
#pragma unroll
    for (int d = 8; d; d >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d);
    ss = __shfl_sync(0xffffffffu, ss, 0);
  }
  const float u = rsqrtf(ss / a.dim + a.eps);
#pragma unroll
  for (int i = 0; i < N; i++)
#pragma unroll
    for (int k = 0; k < 8; k++) v[i][k] = v[i][k] * u * w[i][k];
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
  const int groups = whole ? 1 : (a.dim + a.group - 1) / a.group, lanes = a.group >> 3;      // lanes: of a group, 4 to 32
  uint32_t top[N];                                       // bits of the largest magnitude: NaN counts as the largest of all
#pragma unroll
  for (int i = 0; i < N; i++) {
    top[i] = 0;
#pragma unroll
    for (int k = 0; k < 8; k++) top[i] = max(top[i], __float_as_uint(v[i][k]) & 0x7fffffffu);
  }
  if (whole) {
#pragma unroll
    for (int i = 1; i < N; i++) top[0] = max(top[0], top[i]);
    top[0] = __reduce_max_sync(0xffffffffu, top[0]);
    if (!WARP) {
      if (lane == 0) room[1][warp] = __uint_as_float(top[0]);
      __syncthreads();
      top[0] = __reduce_max_sync(0xffffffffu, lane < (blockDim.x >> 5) ? __float_as_uint(room[1][lane & 15]) : 0u);
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
    if (whole ? i == 0 && t == 0 : (t & (lanes - 1)) == 0) a.scale[row * groups + (whole ? 0 : c / a.group)] = scale;
  }
}

static size_t bytes_of(int type) { return type == KV_F32 ? 4 : type == KV_BF16 ? 2 : 1; }
static bool rows_aligned(const void *p, long long row_stride, int type, int rows, size_t to = 16) {
  return ((reinterpret_cast<uintptr_t>(p) | (rows > 1 ? (uintptr_t)(row_stride * (long long)bytes_of(type)) : 0)) & (to - 1)) == 0;
}

template <typename TX, typename TR> static cudaError_t rms_norm_in_registers(const RmsNorm &a, cudaStream_t s) {
  if (a.dim <= 1024) {
    // a warp a row, of four in a block
    const dim3 grid((a.rows + 3) / 4), block(128);
    if (a.dim <= 256) return launch_k(rms_norm_kernel<TX, TR, 1, true>, grid, block, 0, s, a);
    if (a.dim <= 512) return launch_k(rms_norm_kernel<TX, TR, 2, true>, grid, block, 0, s, a);
    return launch_k(rms_norm_kernel<TX, TR, 4, true>, grid, block, 0, s, a);
  }
  const int n = a.dim <= 4096 ? 1 : a.dim <= 8192 ? 2 : 4;
  const dim3 block((a.dim / 8 + 32 * n - 1) / (32 * n) * 32);
  if (n == 1) return launch_k(rms_norm_kernel<TX, TR, 1, false>, dim3(a.rows), block, 0, s, a);
  if (n == 2) return launch_k(rms_norm_kernel<TX, TR, 2, false>, dim3(a.rows), block, 0, s, a);
  return launch_k(rms_norm_kernel<TX, TR, 4, false>, dim3(a.rows), block, 0, s, a);
}

cudaError_t launch_rms_norm(const RmsNorm &a, cudaStream_t s) {
  const bool eight = kv_is_8bit(a.y_type);
  const bool pieces = a.dim % 8 == 0 && a.dim <= 16384 && rows_aligned(a.x, a.x_rs, a.x_type, a.rows) && rows_aligned(a.gain, 0, a.g_type, 1) &&
                      (!a.res || (rows_aligned(a.res, a.r_rs, a.r_type, a.rows) && rows_aligned(a.sum, a.s_rs, a.r_type, a.rows))) &&
                      rows_aligned(a.y, a.y_rs, a.y_type, a.rows, eight ? 8 : 16) &&
                      (!eight || a.group >= a.dim || a.group == 32 || a.group == 64 || a.group == 128 || a.group == 256);
  if (!pieces) return launch_k(rms_norm_any_kernel, dim3(a.rows), dim3(256), 0, s, a);
  const bool r = a.res && a.r_type == KV_BF16;
  if (a.x_type == KV_F32) return r ? rms_norm_in_registers<float, bf16>(a, s) : rms_norm_in_registers<float, float>(a, s);
  return r || !a.res ? rms_norm_in_registers<bf16, bf16>(a, s) : rms_norm_in_registers<bf16, float>(a, s);
}

// ---------------------------------------------------------------- gradient
// Blocks take rows in turn and keep their own sums for the gain's gradient, which the next launch adds up in the blocks' order.
struct GradPlan {
  int threads, n, blocks;      // threads of a block, eights of a thread
};
// A thread has its columns in every row: eight up to 4096 of them, sixteen up to 8192.  Two blocks an SM of the widest, up to eight of narrow ones.
static GradPlan grad_plan(int rows, int dim) {
  const int n = dim <= 4096 ? 1 : 2, threads = min(512, (dim + 256 * n - 1) / (256 * n) * 32);
  return {threads, n, min(rows, 148 * max(2, min(8, 1024 / threads)))};
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

// Rows of whole eights up to 8192, aligned to 16 bytes, as they lie in memory: the next row is asked for before this one's sums.
template <typename T> struct Raw8;
template <> struct Raw8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float *p) { a = ((const float4 *)p)[0], b = ((const float4 *)p)[1]; }
  __device__ __forceinline__ void floats(float (&y)[8]) const { y[0] = a.x, y[1] = a.y, y[2] = a.z, y[3] = a.w, y[4] = b.x, y[5] = b.y, y[6] = b.z, y[7] = b.w; }
};
template <> struct Raw8<bf16> {
  uint4 u;
  __device__ __forceinline__ void load(const bf16 *p) { u = *(const uint4 *)p; }
  __device__ __forceinline__ void floats(float (&y)[8]) const { unpack2(u.x, y[0], y[1]), unpack2(u.y, y[2], y[3]), unpack2(u.z, y[4], y[5]), unpack2(u.w, y[6], y[7]); }
};

template <typename TG, typename TX, typename TD, int N>
__global__ void __launch_bounds__(512, 3 - N) rms_norm_grad_kernel(const __grid_constant__ RmsNormGrad a) {
  pdl_wait();
  pdl_trigger();
  __shared__ float2 room[2][16];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  Raw8<TG> g[N];
  Raw8<TX> x[N];
  Raw8<TD> c[N];
  float w[N][8], sum[N][8] = {};
  int at[N];
  bool mine[N];
#pragma unroll
  for (int i = 0; i < N; i++) {
    at[i] = (i * blockDim.x + threadIdx.x) * 8;
    mine[i] = at[i] < a.dim;
#pragma unroll
    for (int k = 0; k < 8; k++) w[i][k] = 0.0f;
    if (!mine[i]) continue;
    if (a.w_type == KV_F32) load8((const float *)a.gain + at[i], w[i]);
    else load8((const bf16 *)a.gain + at[i], w[i]);
  }
  auto load = [&](long long row) {
#pragma unroll
    for (int i = 0; i < N; i++) {
      if (!mine[i]) continue;
      g[i].load((const TG *)a.g + row * a.g_rs + at[i]);
      x[i].load((const TX *)a.x + row * a.x_rs + at[i]);
      if (a.carried) c[i].load((const TD *)a.carried + row * a.c_rs + at[i]);
    }
  };
  long long row = blockIdx.x;
  load(row);
  for (int turn = 0; row < a.rows; row += gridDim.x, turn ^= 1) {
    float gr[N][8], xr[N][8], cr[N][8], ss = 0.0f, dot = 0.0f;
#pragma unroll
    for (int i = 0; i < N; i++) {
#pragma unroll
      for (int k = 0; k < 8; k++) gr[i][k] = xr[i][k] = cr[i][k] = 0.0f;
      if (!mine[i]) continue;
      g[i].floats(gr[i]);
      x[i].floats(xr[i]);
      if (a.carried) c[i].floats(cr[i]);
    }
    if (row + gridDim.x < a.rows) load(row + gridDim.x);
#pragma unroll
    for (int i = 0; i < N; i++)
#pragma unroll
      for (int k = 0; k < 8; k++) ss = fmaf(xr[i][k], xr[i][k], ss), dot = fmaf(gr[i][k] * w[i][k], xr[i][k], dot);
#pragma unroll
    for (int d = 16; d; d >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d), dot += __shfl_xor_sync(0xffffffffu, dot, d);
    if (lane == 0) room[turn][warp] = make_float2(ss, dot);
    __syncthreads();
    const float2 some = lane < warps ? room[turn][lane & 15] : make_float2(0.0f, 0.0f);
    ss = some.x, dot = some.y;
#pragma unroll
    for (int d = 8; d; d >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d), dot += __shfl_xor_sync(0xffffffffu, dot, d);
    ss = __shfl_sync(0xffffffffu, ss, 0), dot = __shfl_sync(0xffffffffu, dot, 0);
    const float u = rsqrtf(ss / a.dim + a.eps), along = dot / a.dim * u * u;
#pragma unroll
    for (int i = 0; i < N; i++) {
      if (!mine[i]) continue;
#pragma unroll
      for (int k = 0; k < 8; k++) {
        sum[i][k] = fmaf(gr[i][k], xr[i][k] * u, sum[i][k]);
        cr[i][k] = fmaf(u, fmaf(-xr[i][k], along, gr[i][k] * w[i][k]), cr[i][k]);
      }
      store8((TD *)a.dx + row * a.d_rs + at[i], cr[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < N; i++)
    if (mine[i]) store8(a.part + (long long)blockIdx.x * a.dim + at[i], sum[i]);
}

// 32 columns a block, blocks' sums in eight runs that are then added in order
__global__ void __launch_bounds__(256) rms_norm_gain_kernel(RmsNormGrad a, int blocks) {
  pdl_wait();
  pdl_trigger();
  __shared__ float some[8][32];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = blockIdx.x * 32 + lane, per = (blocks + 7) / 8;
  float sum = 0.0f;
  if (c < a.dim)
#pragma unroll 8
    for (int b = w * per; b < min(blocks, (w + 1) * per); b++) sum += a.part[(long long)b * a.dim + c];
  some[w][lane] = sum;
  __syncthreads();
  if (w || c >= a.dim) return;
  for (int i = 1; i < 8; i++) sum += some[i][lane];
  store_from_f32(a.dgain, a.w_type, c, sum);
}

size_t rms_norm_grad_scratch_bytes(int rows, int dim) { return (size_t)grad_plan(rows, dim).blocks * dim * sizeof(float); }

template <typename TG, typename TX, typename TD> static cudaError_t rms_norm_grad_in_registers(const RmsNormGrad &a, const GradPlan &p, cudaStream_t s) {
  return p.n == 1 ? launch_k(rms_norm_grad_kernel<TG, TX, TD, 1>, dim3(p.blocks), dim3(p.threads), 0, s, a) : launch_k(rms_norm_grad_kernel<TG, TX, TD, 2>, dim3(p.blocks), dim3(p.threads), 0, s, a);
}
template <typename TG, typename TX> static cudaError_t rms_norm_grad_in_registers(const RmsNormGrad &a, const GradPlan &p, cudaStream_t s) {
  return a.d_type == KV_F32 ? rms_norm_grad_in_registers<TG, TX, float>(a, p, s) : rms_norm_grad_in_registers<TG, TX, bf16>(a, p, s);
}

cudaError_t launch_rms_norm_grad(const RmsNormGrad &a, cudaStream_t s) {
  const GradPlan p = grad_plan(a.rows, a.dim);
  if (a.rows) {
    // what is carried has the output's type, as it has where both are of the residual stream
    const bool pieces = a.dim % 8 == 0 && a.dim <= 8192 && rows_aligned(a.g, a.g_rs, a.g_type, a.rows) && rows_aligned(a.x, a.x_rs, a.x_type, a.rows) &&
                        rows_aligned(a.gain, 0, a.w_type, 1) && rows_aligned(a.dx, a.d_rs, a.d_type, a.rows) &&
                        (!a.carried || (a.c_type == a.d_type && rows_aligned(a.carried, a.c_rs, a.c_type, a.rows)));
    cudaError_t e;
    if (!pieces) e = launch_k(rms_norm_grad_any_kernel, dim3(p.blocks), dim3(256), 0, s, a);
    else if (a.g_type == KV_F32) e = a.x_type == KV_F32 ? rms_norm_grad_in_registers<float, float>(a, p, s) : rms_norm_grad_in_registers<float, bf16>(a, p, s);
    else e = a.x_type == KV_F32 ? rms_norm_grad_in_registers<bf16, float>(a, p, s) : rms_norm_grad_in_registers<bf16, bf16>(a, p, s);
    if (e) return e;
  }
  return launch_k(rms_norm_gain_kernel, dim3((a.dim + 31) / 32), dim3(256), 0, s, a, a.rows ? p.blocks : 0);
}

}  // namespace spec
