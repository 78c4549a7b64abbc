// The loss of a student's logits against a teacher's top logits, and its gradient.
#pragma once
#include "embedding.cuh"

namespace spec {

constexpr int DISTILL_MAX_K = 1024;

// Row r: q = softmax(z[r] / T); p over the K entries that the student has (id through the map, where there is one): softmax(values / T) over them, or
// exp(values / T - lse[r]).  loss = sum p (ln p - ln q), or - sum p ln q; dz = grad[r] / T (q sum p - p).  stats: largest logit, sum of exp((z - largest) / T).
// An id several times: the loss is the sum over the entries as they stand, the gradient has the sum of their p.
struct Distill {
  const void *z;
  long long z_rs;
  Ids ids;               // [rows][K]
  const void *values;    // [rows][K]
  const float *lse;      // [rows], or null
  const int32_t *map;    // [map_n], or null
  int rows, vocab, K, map_n, z_type, v_type, kl;
  float temperature;
  const float *grad;     // [rows]; null: 1
  float *loss;           // [rows]; null: the gradient alone, with the statistics given
  float2 *stats;         // [rows], or null
  void *dz;              // null: the loss alone
  long long d_rs;
  int d_type;
  int32_t *status;
};
cudaError_t launch_distill(const Distill &a, cudaStream_t s);

}  // namespace spec
