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

cudaError_t launch_rms_norm(const RmsNorm &a, cudaStream_t s) { return launch_k(rms_norm_any_kernel, dim3(a.rows), dim3(256), 0, s, a); }

// ---------------------------------------------------------------- gradient
// Blocks take rows in turn and keep their own sums for the gain's gradient, which the next launch adds up in the blocks' order.
constexpr int GRAD_BLOCKS = 592;      // four an SM

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

// 32 columns a block, blocks' sums in eight runs that are then added in order
__global__ void __launch_bounds__(256) rms_norm_gain_kernel(RmsNormGrad a, int blocks) {
  pdl_wait();
  pdl_trigger();
  __shared__ float some[8][32];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = blockIdx.x * 32 + lane, per = (blocks + 7) / 8;
  float sum = 0.0f;
  if (c < a.dim)
    for (int b = w * per; b < min(blocks, (w + 1) * per); b++) sum += a.part[(long long)b * a.dim + c];
  some[w][lane] = sum;
  __syncthreads();
  if (w || c >= a.dim) return;
  for (int i = 1; i < 8; i++) sum += some[i][lane];
  store_from_f32(a.dgain, a.w_type, c, sum);
}

size_t rms_norm_grad_scratch_bytes(int rows, int dim) { return (size_t)min(rows, GRAD_BLOCKS) * dim * sizeof(float); }

cudaError_t launch_rms_norm_grad(const RmsNormGrad &a, cudaStream_t s) {
  const int blocks = min(a.rows, GRAD_BLOCKS);
  if (blocks)
    if (const cudaError_t e = launch_k(rms_norm_grad_any_kernel, dim3(blocks), dim3(256), 0, s, a)) return e;
  return launch_k(rms_norm_gain_kernel, dim3((a.dim + 31) / 32), dim3(256), 0, s, a, blocks);
}

}  // namespace spec
