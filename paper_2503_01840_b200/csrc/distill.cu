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
__device__ __forceinline__ void join_lanes(const Base2 &b, Running &r) {      // lane 0's is the warp's
#pragma unroll
  for (int d = 16; d; d >>= 1) {
    const float m = __shfl_xor_sync(0xffffffffu, r.m, d), s = __shfl_xor_sync(0xffffffffu, r.s, d);
    join(b, r, m, s);
  }
}

// ---------------------------------------------------------------- a row's entries
struct Entries {
  int *id;               // the student's, -1: none
  float *p, *ln_p, *z;   // z: the student's logit there
};
__host__ __device__ constexpr size_t entries_bytes(int K) { return ((size_t)K * 16 + 15) / 16 * 16; }
__device__ __forceinline__ Entries entries_in(char *shared, int K) {
  float *const f = (float *)shared;
  return {(int *)f, f + K, f + 2 * K, f + 3 * K};
}
// One warp fills them in and returns sum p; *none: whether the row has no entry (sum p may be 0 otherwise too, where every p is too small).
__device__ __forceinline__ float read_entries(const Distill &a, const Entries &e, long long row, bool *none) {
  const int lane = threadIdx.x & 31;
  const float inv_t = 1.0f / a.temperature;
  const long long z0 = row * a.z_rs, at = row * a.K;
  float top = -INFINITY;
  bool some = false, nan = false;
#pragma unroll 2
  for (int k = lane; k < a.K; k += 32) {
    int id = id_at(a.ids, at + k);
    const float v = load_as_f32(a.values, a.v_type, at + k);
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
    e.z[k] = id >= 0 ? load_as_f32(a.z, a.z_type, z0 + id) : 0.0f;
    if (id < 0) continue;
    some = true;
    top = fmaxf(top, v);
    nan |= v != v;
  }
  *none = !__any_sync(0xffffffffu, some);
  if (*none) return 0.0f;
  float ln_sum = 0.0f, lse = 0.0f;
  if (a.lse) {
    lse = a.lse[row];
    top = 0.0f;
  } else {
    top = key_value(__reduce_max_sync(0xffffffffu, nan ? 0xffffffffu : ordered_key(top)));
    float sum = 0.0f;
    for (int k = lane; k < a.K; k += 32)
      if (e.id[k] >= 0) sum += expf((e.ln_p[k] - top) * inv_t);
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    ln_sum = logf(sum);
  }
  float all = 0.0f;
  for (int k = lane; k < a.K; k += 32) {
    const float ln_p = (e.ln_p[k] - top) * inv_t - (a.lse ? lse : ln_sum), p = e.id[k] >= 0 ? expf(ln_p) : 0.0f;
    e.ln_p[k] = ln_p;
    e.p[k] = p;
    all += p;
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) all += __shfl_xor_sync(0xffffffffu, all, d);
  return all;
}
// A warp's sum over its lanes' entries of p (ln p - ln q), ln q without the logarithm of q's normaliser
__device__ __forceinline__ float entries_loss(const Distill &a, const Entries &e, float m) {
  float loss = 0.0f;
  for (int k = threadIdx.x & 31; k < a.K; k += 32) {
    const float p = e.p[k], ln_q = (e.z[k] - m) / a.temperature;
    if (e.id[k] >= 0 && p != 0.0f) loss += p * (a.kl ? e.ln_p[k] - ln_q : -ln_q);
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) loss += __shfl_xor_sync(0xffffffffu, loss, d);
  return loss;
}
// The gradient at the entries' ids from c0 to c1: an id's first entry writes for all that name it.  d: of the row
__device__ __forceinline__ void entries_gradient(const Distill &a, const Base2 &b, const Entries &e, float m, float g, float of_q, int c0, int c1, long long d) {
  for (int k = threadIdx.x; k < a.K; k += blockDim.x) {
    const int id = e.id[k];
    if (id < c0 || id >= c1) continue;
    bool first = true;
    for (int j = 0; first && j < k; j++) first = e.id[j] != id;
    if (!first) continue;
    float p = e.p[k];
    for (int j = k + 1; j < a.K; j++)
      if (e.id[j] == id) p += e.p[j];
    store_from_f32(a.dz, a.d_type, d + id, fmaf(of_q, exp_of(b, e.z[k] - m), -g * p));
  }
}

// ---------------------------------------------------------------- any vocabulary: a block a row, read once for each step
__global__ void __launch_bounds__(512) distill_any_kernel(Distill a, Base2 b) {
  pdl_wait();
  pdl_trigger();
  extern __shared__ __align__(16) char shared[];
  __shared__ float of_s[16], of_m[16], mass;
  __shared__ int empty;
  const Entries e = entries_in(shared, a.K);
  const int tid = threadIdx.x;
  const long long row = blockIdx.x, z0 = row * a.z_rs, d0 = row * a.d_rs;
  if (tid < 32) {
    bool none;
    const float all = read_entries(a, e, row, &none);
    if (tid == 0) mass = all, empty = none;
  }
  __syncthreads();
  if (empty) {
    if (a.loss && tid == 0) {
      a.loss[row] = 0.0f;
      if (a.stats) a.stats[row] = make_float2(0.0f, 1.0f);
    }
    if (a.dz)
      for (int c = tid; c < a.vocab; c += 512) store_from_f32(a.dz, a.d_type, d0 + c, 0.0f);
    return;
  }
  const float all = mass;
  Running r;
  if (a.loss) {
    for (int c = tid; c < a.vocab; c += 512) {
      const float v = load_as_f32(a.z, a.z_type, z0 + c);
      if (v > r.m) r.s *= exp_of(b, r.m == -INFINITY ? 0.0f : r.m - v), r.m = v;
      r.s += exp_of(b, v - relative_to(r.m));
    }
    join_lanes(b, r);
    if ((tid & 31) == 0) of_m[tid >> 5] = r.m, of_s[tid >> 5] = r.s;
    __syncthreads();
    r = Running{};
    for (int w = 0; w < 16; w++) join(b, r, of_m[w], of_s[w]);
    if (r.m == -INFINITY) r.s = NAN;                     // no logit above -inf: there is no softmax
    if (tid < 32) {
      const float loss = entries_loss(a, e, r.m);
      if (tid == 0) {
        a.loss[row] = loss + all * logf(r.s);
        if (a.stats) a.stats[row] = make_float2(r.m, r.s);
      }
    }
  } else {
    r.m = a.stats[row].x, r.s = a.stats[row].y;
  }
  if (!a.dz) return;
  const float g = (a.grad ? a.grad[row] : 1.0f) / a.temperature, of_q = g * all / r.s;
  for (int c = tid; c < a.vocab; c += 512) store_from_f32(a.dz, a.d_type, d0 + c, of_q * exp_of(b, load_as_f32(a.z, a.z_type, z0 + c) - r.m));
  __syncthreads();
  entries_gradient(a, b, e, r.m, g, of_q, 0, a.vocab, d0);
}

// ---------------------------------------------------------------- rows held in shared memory
// A cluster of up to eight CTAs has a row, a slice of up to SLICE bytes each, read from memory once: copied to shared memory while a warp looks the entries up, walked for the maximum and the sum, which
// the CTAs exchange, and walked again for the gradient.  Elements keep their place modulo 16 bytes, so any alignment will do; a thread copies and walks the same units of eight.
// Where the statistics are given the CTAs have nothing to exchange and are no cluster.
enum { LOSS = 0, GRADIENT = 1, BOTH = 2 };
struct Slices {
  int n, per;            // slices of a row, elements of one: a multiple of 8
  int whole;             // units of the output are aligned pieces of 16 bytes
  int look_first;        // whether a row is not loaded before it is known that some id of it is not -1
};
constexpr int SLICE = 66 << 10, SLICE_MOST = 200 << 10, CLUSTER_MOST = 8;

__device__ __forceinline__ uint32_t smem_of(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy16(void *to, const void *from) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_of(to)), "l"(from) : "memory"); }
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ float2 of_cta(const float2 *p, int rank) {
  uint32_t at;
  float2 v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_of(p)), "r"(rank));
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(at) : "memory");
  return v;
}

template <typename T, typename O, int MODE>
__global__ void __launch_bounds__(512, 3) distill_rows_kernel(const __grid_constant__ Distill a, const __grid_constant__ Base2 b, const __grid_constant__ Slices sl) {
  pdl_wait();
  pdl_trigger();
  extern __shared__ __align__(16) char shared[];
  __shared__ float2 of_warp[16], mine;
  __shared__ float mass;
  __shared__ int empty;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, NT = blockDim.x;
  const int rank = blockIdx.x % sl.n, c0 = rank * sl.per, n = max(0, min(sl.per, a.vocab - c0));
  const long long row = blockIdx.x / sl.n;
  const T *const z = (const T *)a.z + row * a.z_rs + c0;
  const int shift = (int)((reinterpret_cast<uintptr_t>(z) & 15) / sizeof(T)), units = (shift + n + 7) / 8;
  const Entries e = entries_in(shared, a.K);
  T *const buf = (T *)(shared + entries_bytes(a.K));     // element c of the slice at buf[shift + c]
  bool there = true;
  if (sl.look_first) {
    there = false;
    for (int k = 0; k < a.K && !there; k += 32) there = __any_sync(0xffffffffu, k + lane < a.K && id_at(a.ids, row * a.K + k + lane) != -1);
  }
  const int steps = (units + NT - 1) / NT, quarter = (steps + 3) / 4;
  if (there) {
#pragma unroll
    for (int q = 0; q < 4; q++) {
      for (int i = q * quarter; i < min(steps, (q + 1) * quarter); i++) {
        const int u = i * NT + tid, c = u * 8 - shift;
        if (u >= units) continue;
        if (c >= 0 && c + 8 <= n) {
          copy16(buf + u * 8, z + c);
          if (sizeof(T) == 4) copy16(buf + u * 8 + 4, z + c + 4);
        } else {
#pragma unroll
          for (int x = 0; x < 8; x++) buf[u * 8 + x] = c + x >= 0 && c + x < n ? z[c + x] : from_f32<T>(-INFINITY);
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    }
    if (warp == 0) {
      bool none;
      const float all = read_entries(a, e, row, &none);
      if (lane == 0) mass = all, empty = none;
    }
  } else if (tid == 0) {
    empty = 1;
  }
  Running r;
  if (MODE != GRADIENT && there) {
#pragma unroll
    for (int q = 0; q < 4; q++) {
      if (q == 0) asm volatile("cp.async.wait_group 3;" ::: "memory");
      if (q == 1) asm volatile("cp.async.wait_group 2;" ::: "memory");
      if (q == 2) asm volatile("cp.async.wait_group 1;" ::: "memory");
      if (q == 3) asm volatile("cp.async.wait_group 0;" ::: "memory");
      for (int i = q * quarter; i < min(steps, (q + 1) * quarter); i++) {
        const int u = i * NT + tid;
        if (u >= units) continue;
        float y[8];
        load8(buf + u * 8, y);
        const float top = fmaxf(fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3])), fmaxf(fmaxf(y[4], y[5]), fmaxf(y[6], y[7])));
        if (top > r.m) r.s *= exp_of(b, r.m == -INFINITY ? 0.0f : r.m - top), r.m = top;
        const float m = relative_to(r.m);
        float some = 0.0f;
#pragma unroll
        for (int x = 0; x < 8; x++) some += exp_of(b, y[x] - m);
        r.s += some;
      }
    }
    join_lanes(b, r);
    if (lane == 0) of_warp[warp] = make_float2(r.m, r.s);
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();
  if (MODE != GRADIENT) {
    r = Running{};
    if (there)
      for (int w = 0; w < NT / 32; w++) join(b, r, of_warp[w].x, of_warp[w].y);
    if (sl.n > 1) {                                      // the others have read their row's entries by the end of the wait: the output may be the input
      if (tid == 0) mine = make_float2(r.m, r.s);
      __syncwarp();
      cluster_arrive();
      cluster_wait();
      r = Running{};
      for (int k = 0; k < sl.n; k++) {
        const float2 v = of_cta(&mine, k);
        join(b, r, v.x, v.y);
      }
      cluster_arrive();
    }
    if (r.m == -INFINITY) r.s = NAN;                     // no logit above -inf: there is no softmax
    if (rank == 0 && warp == 0) {
      const float loss = empty ? 0.0f : entries_loss(a, e, r.m) + mass * logf(r.s);
      if (lane == 0) {
        a.loss[row] = loss;
        if (a.stats) a.stats[row] = empty ? make_float2(0.0f, 1.0f) : make_float2(r.m, r.s);
      }
    }
  } else if (!empty) {
    r.m = a.stats[row].x, r.s = a.stats[row].y;
  }
  if (MODE != LOSS) {
    const bool none = empty;
    const float g = none ? 0.0f : (a.grad ? a.grad[row] : 1.0f) / a.temperature, of_q = none ? 0.0f : g * mass / r.s;
    const long long d0 = row * a.d_rs;
    O *const d = (O *)a.dz + d0 + c0;
    if (sl.whole && shift == 0) {
      for (int u = tid; u < units; u += NT) {
        float y[8];
        if (none) {
#pragma unroll
          for (int x = 0; x < 8; x++) y[x] = 0.0f;
        } else {
          load8(buf + u * 8, y);
#pragma unroll
          for (int x = 0; x < 8; x++) y[x] = of_q * exp_of(b, y[x] - r.m);
        }
        if (u * 8 + 8 <= n) {
          store8(d + u * 8, y);
        } else {
#pragma unroll
          for (int x = 0; x < 8; x++)
            if (u * 8 + x < n) d[u * 8 + x] = from_f32<O>(y[x]);
        }
      }
    } else {
      for (int c = tid; c < n; c += NT) d[c] = from_f32<O>(none ? 0.0f : of_q * exp_of(b, to_f32(buf[shift + c]) - r.m));
    }
    if (!none) {
      __syncthreads();
      entries_gradient(a, b, e, r.m, g, of_q, c0, c0 + n, d0);
    }
  }
  __syncwarp();
  if (MODE != GRADIENT && sl.n > 1) cluster_wait();      // nobody leaves while its numbers may be read
}

// Slices of about SLICE bytes, so that three CTAs are on an SM; smaller ones where rows alone do not fill the SMs twice, down to 2 KB.
static bool slices_of(const Distill &a, Slices *sl) {
  const size_t e = a.z_type == 0 ? 4 : 2, row = (size_t)a.vocab * e;
  const int most = a.loss ? CLUSTER_MOST : 64;
  int n = (int)min<size_t>((row + SLICE - 1) / SLICE, most);
  while (n < most && n < 8 && (long long)a.rows * n < 2 * 148 && row / (n + 1) >= 2048) n++;
  sl->n = n;
  sl->per = (int)(((a.vocab + n - 1LL) / n + 7) / 8 * 8);
  sl->whole = a.dz && pieces_aligned(a.dz, a.rows > 1 ? a.d_rs : 0, a.d_type == 0 ? 4 : 2);
  sl->look_first = (long long)a.rows * n > 4 * 148;
  return (size_t)sl->per * e <= SLICE_MOST && (long long)a.rows * n <= INT32_MAX;
}

template <typename T, typename O, int MODE> static cudaError_t rows_in_shared(const Distill &a, const Base2 &b, const Slices &sl, cudaStream_t s) {
  static SmemLimit limit;
  const int units = sl.per / 8 + 1, threads = units <= 256 ? 128 : units <= 1024 ? 256 : 512;
  const size_t smem = entries_bytes(a.K) + (size_t)units * 8 * sizeof(T);
  if (smem > 46 << 10 && !limit.ensure(distill_rows_kernel<T, O, MODE>, (int)smem)) return cudaErrorInvalidValue;
  if (!launch_allowed()) return cudaSuccess;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(a.rows * sl.n)), cfg.blockDim = dim3(threads), cfg.dynamicSmemBytes = smem, cfg.stream = s;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = sl.n, at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = MODE != GRADIENT && sl.n > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, distill_rows_kernel<T, O, MODE>, a, b, sl);
}
template <typename T, typename O> static cudaError_t rows_in_shared(const Distill &a, const Base2 &b, const Slices &sl, cudaStream_t s) {
  return a.loss ? rows_in_shared<T, O, BOTH>(a, b, sl, s) : rows_in_shared<T, O, GRADIENT>(a, b, sl, s);
}

cudaError_t launch_distill(const Distill &a, cudaStream_t s) {
  const Base2 b = base2_of(a.temperature);
  Slices sl;
  if (!slices_of(a, &sl)) return launch_k(distill_any_kernel, dim3(a.rows), dim3(512), entries_bytes(a.K), s, a, b);
  if (a.z_type == 0) {
    if (!a.dz) return rows_in_shared<float, float, LOSS>(a, b, sl, s);
    return a.d_type == 0 ? rows_in_shared<float, float>(a, b, sl, s) : rows_in_shared<float, bf16>(a, b, sl, s);
  }
  if (!a.dz) return rows_in_shared<bf16, bf16, LOSS>(a, b, sl, s);
  return a.d_type == 0 ? rows_in_shared<bf16, float>(a, b, sl, s) : rows_in_shared<bf16, bf16>(a, b, sl, s);
}

}  // namespace spec
