// Distillation from a teacher's top logits: loss = sum p (ln p - ln q) over the teacher's entries, q the student's softmax; its gradient dz = g / T (q sum p - p).
#include "distill.cuh"

#include <algorithm>

#include "vec.cuh"

namespace spec {

using std::max;
using std::min;

// exp(d / T) as a power of two: log2(e) / T in two parts, so that what is off is the product's rounding alone
struct Base2 {
  float hi, lo;
};
static Base2 base2_of(float temperature) {
  const double c = 1.4426950408889634074 / temperature;      // log2(e) / T
  return {(float)c, (float)(c - (float)c)};
}
__device__ __forceinline__ float power_of_two(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// d below -1e30 counts as that, which is 0 at every temperature up to 1e4: the second part's sign may differ from the first's, and infinities must not meet
__device__ __forceinline__ float exp_of(const Base2 &b, float d) {
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(d) : "f"(-1e30f));
  return power_of_two(fmaf(d, b.hi, d * b.lo));
}

// Maximum and sum of exp relative to it, of what has been seen.  While nothing but -inf has been, the sum is taken relative to 0: of them it stays 0, a NaN shows.
struct Running {
  float m = -INFINITY, s = 0.0f;
};
__device__ __forceinline__ float relative_to(float m) { return m == -INFINITY ? 0.0f : m; }
__device__ __forceinline__ void join(const Base2 &b, Running &a, float m, float s) {
  const float n = relative_to(fmaxf(a.m, m));
  a.s = a.s * exp_of(b, a.m == -INFINITY ? 0.0f : a.m - n) + s * exp_of(b, m == -INFINITY ? 0.0f : m - n);
  a.m = fmaxf(a.m, m);
}

// ---------------------------------------------------------------- a row's entries
struct Entries {
  int *id;               // the student's, -1: none
  float *p, *ln_p, *z;   // z: the student's logit there
};
// Threads of a block fill them in (ids, p, ln p); returns sum p (0: the row has none).  The same for every thread.
__device__ float read_entries(const Distill &a, const Entries &e, long long row, float *room) {
  const float inv_t = 1.0f / a.temperature;
  float top = -INFINITY, sum = 0.0f;
  bool some = false, nan = false;
  for (int k = threadIdx.x; k < a.K; k += blockDim.x) {
    const long long at = row * a.K + k;
    const float v = load_as_f32(a.values, a.v_type, at);
    int id = id_at(a.ids, at);
    if (id != -1) {
      const int n = a.map ? a.map_n : a.vocab;
      if (id < 0 || id >= n) {
        set_status(a.status, ST_BOUNDS, 65, (int)row, id);
        id = -1;
      } else if (a.map) {
        id = a.map[id];
        if (id < -1 || id >= a.vocab) set_status(a.status, ST_BOUNDS, 66, (int)row, id), id = -1;
      }
    }
    if (v == -INFINITY) id = -1;
    e.id[k] = id;
    e.ln_p[k] = v;
    if (id < 0) continue;
    some = true;
    top = fmaxf(top, v);
    nan |= v != v;
  }
  some = __syncthreads_or(some);
  if (!some) return 0.0f;
  if (!a.lse) {                                          // largest of them: by the bits of a monotone key
    top = key_value(block_max(nan ? 0xffffffffu : ordered_key(top), room));
    for (int k = threadIdx.x; k < a.K; k += blockDim.x)
      if (e.id[k] >= 0) sum += expf((e.ln_p[k] - top) * inv_t);
    sum = block_sum(sum, room);
  }
  const float ln_sum = a.lse ? 0.0f : logf(sum), lse = a.lse ? a.lse[row] : 0.0f;
  float all = 0.0f;
  for (int k = threadIdx.x; k < a.K; k += blockDim.x) {
    const float ln_p = a.lse ? e.ln_p[k] * inv_t - lse : (e.ln_p[k] - top) * inv_t - ln_sum, p = e.id[k] >= 0 ? expf(ln_p) : 0.0f;
    e.ln_p[k] = ln_p;
    e.p[k] = p;
    all += p;
  }
  all = block_sum(all, room);
  return all;
}
// what the entries [k] of this thread add to sum p (ln p - ln q), ln q without the logarithm of q's normaliser
__device__ __forceinline__ float entry_loss(const Distill &a, float p, float ln_p, float z, float m) {
  if (p == 0.0f) return 0.0f;
  const float ln_q = (z - m) / a.temperature;
  return p * (a.kl ? ln_p - ln_q : -ln_q);
}

// ---------------------------------------------------------------- any vocabulary, stride and alignment: a block a row, read once for each step
__global__ void __launch_bounds__(512) distill_any_kernel(Distill a, Base2 b) {
  pdl_wait();
  pdl_trigger();
  extern __shared__ float shared[];
  __shared__ float room[32], of_s[16], of_m[16];
  const Entries e{(int *)shared, shared + a.K, shared + 2 * a.K, shared + 3 * a.K};
  const int tid = threadIdx.x;
  const long long row = blockIdx.x, z0 = row * a.z_rs, d0 = row * a.d_rs;
  const float all = read_entries(a, e, row, room);
  bool some = false;
  for (int k = tid; k < a.K; k += 512) some |= e.id[k] >= 0;
  if (!__syncthreads_or(some)) {
    if (a.loss && tid == 0) {
      a.loss[row] = 0.0f;
      if (a.stats) a.stats[row] = make_float2(0.0f, 1.0f);
    }
    if (a.dz)
      for (int c = tid; c < a.vocab; c += 512) store_from_f32(a.dz, a.d_type, d0 + c, 0.0f);
    return;
  }
  for (int k = tid; k < a.K; k += 512) e.z[k] = e.id[k] >= 0 ? load_as_f32(a.z, a.z_type, z0 + e.id[k]) : 0.0f;
  Running r;
  if (a.loss) {
    for (int c = tid; c < a.vocab; c += 512) {
      const float v = load_as_f32(a.z, a.z_type, z0 + c);
      if (v > r.m) r.s *= exp_of(b, r.m == -INFINITY ? 0.0f : r.m - v), r.m = v;
      r.s += exp_of(b, v - relative_to(r.m));
    }
    for (int d = 16; d; d >>= 1) {
      const float m = __shfl_xor_sync(0xffffffffu, r.m, d), s = __shfl_xor_sync(0xffffffffu, r.s, d);
      join(b, r, m, s);
    }
    if ((tid & 31) == 0) of_m[tid >> 5] = r.m, of_s[tid >> 5] = r.s;
    __syncthreads();
    r = Running{};
    for (int w = 0; w < 16; w++) join(b, r, of_m[w], of_s[w]);
    if (r.m == -INFINITY) r.s = NAN;                     // no logit above -inf: there is no softmax
    float loss = 0.0f;
    for (int k = tid; k < a.K; k += 512)
      if (e.id[k] >= 0) loss += entry_loss(a, e.p[k], e.ln_p[k], e.z[k], r.m);
    loss = block_sum(loss, room);
    if (tid == 0) {
      a.loss[row] = loss + all * logf(r.s);
      if (a.stats) a.stats[row] = make_float2(r.m, r.s);
    }
  } else {
    r.m = a.stats[row].x, r.s = a.stats[row].y;
    __syncthreads();
  }
  if (!a.dz) return;
  const float g = (a.grad ? a.grad[row] : 1.0f) / a.temperature, of_q = g * all / r.s;
  for (int c = tid; c < a.vocab; c += 512) store_from_f32(a.dz, a.d_type, d0 + c, of_q * exp_of(b, load_as_f32(a.z, a.z_type, z0 + c) - r.m));
  __syncthreads();
  for (int k = tid; k < a.K; k += 512) {                 // an id's first entry writes for all that name it
    const int id = e.id[k];
    bool first = id >= 0;
    for (int j = 0; first && j < k; j++) first = e.id[j] != id;
    if (!first) continue;
    float p = e.p[k];
    for (int j = k + 1; j < a.K; j++)
      if (e.id[j] == id) p += e.p[j];
    store_from_f32(a.dz, a.d_type, d0 + id, fmaf(of_q, exp_of(b, e.z[k] - r.m), -g * p));
  }
}

cudaError_t launch_distill(const Distill &a, cudaStream_t s) {
  return launch_k(distill_any_kernel, dim3(a.rows), dim3(512), (size_t)a.K * 16, s, a, base2_of(a.temperature));
}

}  // namespace spec
