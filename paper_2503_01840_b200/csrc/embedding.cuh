// Embedding lookup and its gradient.
#pragma once
#include "common.cuh"

namespace spec {

// Ids of 32 or 64 bits.
struct Ids {
  const void *p;
  int wide;
};
// As an int; -1: none; what an int cannot hold becomes -2, which is out of range everywhere
__device__ __forceinline__ int id_at(const Ids &ids, long long i) {
  if (!ids.wide) return ((const int32_t *)ids.p)[i];
  const long long v = ((const long long *)ids.p)[i];
  return v == (int)v ? (int)v : -2;
}

// out[t] = scale * w[ids[t]], zeros for an id of -1; strides in elements
struct Embed {
  const void *w;
  long long w_rs;
  int vocab, dim;
  Ids ids;
  int tokens;
  float scale;
  void *out;
  long long o_rs;
  int32_t *status;
};
cudaError_t launch_embed_rows(const Embed &a, int w_dtype, int out_dtype, cudaStream_t s);

// out[v] (+)= scale * sum over t with ids[t] = v of grad[t], in the order of t
struct EmbedGrad {
  const void *grad;
  long long g_rs;
  int vocab, dim;
  Ids ids;
  int tokens;
  float scale;
  void *out;
  long long o_rs;
  int accumulate;
  void *scratch;
  int32_t *status;
};
size_t embed_grad_scratch_bytes(int tokens, int vocab, int dim);
cudaError_t launch_embed_grad(const EmbedGrad &a, int g_dtype, int out_dtype, cudaStream_t s);

}  // namespace spec
