// Root-mean-square norm of a residual sum, with outputs in 8 bits too, and its gradient.
#pragma once
#include "kv_cache.cuh"

namespace spec {

// s = x + res (x, without res); sum = s in res's type; y = s rsqrt(mean s^2 + eps) gain, in 8 bits codes and scales [rows][groups].  Types: KV_F32, KV_BF16, y's
// also KV_E4M3 and KV_INT8; strides in elements.
struct RmsNorm {
  const void *x, *res, *gain;
  void *sum, *y;
  float *scale;
  long long x_rs, r_rs, s_rs, y_rs;
  int x_type, r_type, g_type, y_type, rows, dim, group;
  float eps;
};
cudaError_t launch_rms_norm(const RmsNorm &a, cudaStream_t s);

// With u = rsqrt(mean x^2 + eps), h = x u: dx = u (g w - h mean(g w h)) + carried, dgain = sum over rows of g h
struct RmsNormGrad {
  const void *g, *x, *gain, *carried;
  void *dx, *dgain;
  long long g_rs, x_rs, c_rs, d_rs;
  int g_type, x_type, w_type, c_type, d_type, rows, dim;
  float eps;
  float *part;           // [blocks][dim]
};
size_t rms_norm_grad_scratch_bytes(int rows, int dim);
cudaError_t launch_rms_norm_grad(const RmsNormGrad &a, cudaStream_t s);

}  // namespace spec
