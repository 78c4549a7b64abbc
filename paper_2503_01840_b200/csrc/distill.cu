// Distillation from a teacher's top logits: loss = sum p (ln p - ln q) over the teacher's entries, q the student's softmax; its gradient dz = g / T (q sum p - p).
#include "distill.cuh"

#include <algorithm>

#include "vec.cuh"

namespace spec {

using std::max;
using std::min;

// exp(d / T) = 2^(d c), c = log2(e) / T.  c's own rounding is 2^-25 of the exponent at most, as much as the product's is.  Pairs of 32-bit numbers take one instruction.
typedef unsigned long long Pair;
__device__ __forceinline__ Pair pair(float a, float b) {
  Pair p;
  asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "f"(a), "f"(b));
  return p;
}
__device__ __forceinline__ void unpair(Pair p, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p)); }
__device__ __forceinline__ Pair add(Pair a, Pair b) {
  Pair p;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(p) : "l"(a), "l"(b));
  return p;
}
__device__ __forceinline__ Pair mul(Pair a, Pair b) {
  Pair p;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(p) : "l"(a), "l"(b));
  return p;
}
__device__ __forceinline__ float power_of_two(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float exp_of(float c, float d) { return power_of_two(d * c); }
// exp((y - m) / T) of eight
__device__ __forceinline__ void exp_of(float c, float m, const float (&y)[8], Pair (&e)[4]) {
#pragma unroll
  for (int i = 0; i < 4; i++) {
    float a, b;
    unpair(mul(add(pair(y[2 * i], y[2 * i + 1]), pair(-m, -m)), pair(c, c)), a, b);
    e[i] = pair(power_of_two(a), power_of_two(b));
  }
}

// Maximum and sum of exp relative to it, of what has been seen.  While nothing but -inf has been, the sum is taken relative to 0: of them it stays 0, a NaN shows.
struct Running {
  float m = -INFINITY, s = 0.0f;
};
__device__ __forceinline__ float relative_to(float m) { return m == -INFINITY ? 0.0f : m; }
// of a warp's lanes, the same for all of them
__device__ __forceinline__ void join_lanes(float b, Running &r) {
  const float m = key_value(__reduce_max_sync(0xffffffffu, ordered_key(r.m)));
  float s = r.s * exp_of(b, r.m == -INFINITY ? 0.0f : r.m - m);
#pragma unroll
  for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
  r = Running{m, s};
}

// ---------------------------------------------------------------- a row's entries
struct Entries {
  int *id;               // the student's, -1: none
  float *p, *ln_p, *z;   // z: the student's logit there
};
__host__ __device__ constexpr int fours(int K) { return (K + 3) / 4 * 4; }
__host__ __device__ constexpr size_t entries_bytes(int K) { return (size_t)fours(K) * 16; }
__device__ __forceinline__ Entries entries_in(char *shared, int K) {
  float *const f = (float *)shared;
  return {(int *)f, f + fours(K), f + 2 * fours(K), f + 3 * fours(K)};
}
// One warp fills them in and returns sum p; *none: whether the row has no entry (sum p may be 0 otherwise too, where every p is too small).
__device__ __forceinline__ float read_entries(const Distill &a, const Entries &e, long long row, bool *none) {
  const int lane = threadIdx.x & 31;
  const float inv_t = 1.0f / a.temperature;
  const long long z0 = row * a.z_rs, at = row * a.K;
  float top = -INFINITY;
  bool some = false, nan = false;
  if (lane < fours(a.K) - a.K) e.id[a.K + lane] = -1;
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
__device__ __forceinline__ void entries_gradient(const Distill &a, float b, const Entries &e, float m, float g, float of_q, int c0, int c1, long long d) {
  for (int k = threadIdx.x; k < a.K; k += blockDim.x) {
    const int id = e.id[k];
    if (id < c0 || id >= c1) continue;
    float p = e.p[k];
    bool first = true;
    for (int j = 0; j < a.K; j += 4) {
      const int4 o = *(const int4 *)(e.id + j);
      if (o.x != id && o.y != id && o.z != id && o.w != id) continue;
      for (int x = j; x < j + 4; x++) {
        if (e.id[x] != id) continue;
        first &= x >= k;
        if (x > k) p += e.p[x];
      }
    }
    if (first) store_from_f32(a.dz, a.d_type, d + id, fmaf(of_q, exp_of(b, e.z[k] - m), -g * p));
  }
}

// ---------------------------------------------------------------- any vocabulary: a block a row, read once for each step
__global__ void __launch_bounds__(512) distill_any_kernel(Distill a, float b) {
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
    r = (tid & 31) < 16 ? Running{of_m[tid & 31], of_s[tid & 31]} : Running{};
    join_lanes(b, r);
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
  int ahead;             // rows that are under way at a time: those after them have their entries fetched into L2
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

// the largest of eight; of NaN and a number the number
__device__ __forceinline__ float largest(const float *p) {
  float y[8];
  load8(p, y);
  return fmaxf(fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3])), fmaxf(fmaxf(y[4], y[5]), fmaxf(y[6], y[7])));
}
__device__ __forceinline__ float largest(const bf16 *p) {
  const uint4 u = *(const uint4 *)p;
  const __nv_bfloat162 a = *(const __nv_bfloat162 *)&u.x, b = *(const __nv_bfloat162 *)&u.y, c = *(const __nv_bfloat162 *)&u.z, d = *(const __nv_bfloat162 *)&u.w;
  const __nv_bfloat162 m = __hmax2(__hmax2(a, b), __hmax2(c, d));
  return fmaxf(__low2float(m), __high2float(m));
}

constexpr int WALKERS = 256;      // threads that copy and walk; another warp looks the entries up and takes the loss

template <typename T, typename O, int MODE>
__global__ void __launch_bounds__(WALKERS + 32, 3) distill_rows_kernel(const __grid_constant__ Distill a, float b, const __grid_constant__ Slices sl) {
  pdl_wait();
  pdl_trigger();
  extern __shared__ __align__(16) char shared[];
  __shared__ float2 of_warp[WALKERS / 32], mine;
  __shared__ float mass;
  __shared__ int empty;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const bool walks = tid < WALKERS;
  const int rank = blockIdx.x % sl.n, c0 = rank * sl.per, n = max(0, min(sl.per, a.vocab - c0));
  const long long row = blockIdx.x / sl.n;
  const T *const z = (const T *)a.z + row * a.z_rs + c0;
  const int shift = (int)((reinterpret_cast<uintptr_t>(z) & 15) / sizeof(T)), units = (shift + n + 7) / 8;
  const Entries e = entries_in(shared, a.K);
  T *const buf = (T *)(shared + entries_bytes(a.K));     // element c of the slice at buf[shift + c]
  if (sl.ahead && !walks && row + sl.ahead < a.rows) {
    const long long at = (row + sl.ahead) * a.K;
    for (int k = lane * 32; k < a.K * (a.ids.wide ? 2 : 1); k += 1024) asm volatile("prefetch.global.L2 [%0];" ::"l"((const char *)a.ids.p + at * (a.ids.wide ? 8 : 4) + k * 4));
    for (int k = lane * 32; k < a.K; k += 1024) asm volatile("prefetch.global.L2 [%0];" ::"l"((const char *)a.values + (at + k) * (a.v_type == 0 ? 4 : 2)));
  }
  bool there = true;
  if (sl.look_first) {
    there = false;
    for (int k = 0; k < a.K && !there; k += 32) there = __any_sync(0xffffffffu, k + lane < a.K && id_at(a.ids, row * a.K + k + lane) != -1);
  }
  // steps of a unit a thread; in `inner` ones every unit is whole and in the slice
  const int steps = (units + WALKERS - 1) / WALKERS, inner0 = shift ? 1 : 0, inner1 = max(inner0, (shift + n) / 8 / WALKERS), quarter = (steps + 3) / 4;
  if (there && walks) {
#pragma unroll
    for (int q = 0; q < 4; q++) {
      for (int i = q * quarter; i < min(steps, (q + 1) * quarter); i++) {
        const int u = i * WALKERS + tid, c = u * 8 - shift;
        if ((i >= inner0 && i < inner1) || (u < units && c >= 0 && c + 8 <= n)) {
          copy16(buf + u * 8, z + c);
          if (sizeof(T) == 4) copy16(buf + u * 8 + 4, z + c + 4);
        } else if (u < units) {
#pragma unroll
          for (int x = 0; x < 8; x++) buf[u * 8 + x] = c + x >= 0 && c + x < n ? z[c + x] : from_f32<T>(-INFINITY);
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    }
  } else if (there) {
    bool none;
    const float all = read_entries(a, e, row, &none);
    if (lane == 0) mass = all, empty = none;
  } else if (tid == 0) {
    empty = 1;
  }
  Running r;
  if (MODE != GRADIENT && there && walks) {
    auto seen = [&](int u) {
      float y[8];
      load8(buf + u * 8, y);
      const float top = largest(buf + u * 8);
      if (top > r.m) r.s *= exp_of(b, r.m == -INFINITY ? 0.0f : r.m - top), r.m = top;
      Pair p[4];
      exp_of(b, relative_to(r.m), y, p);
      float even, odd;
      unpair(add(add(p[0], p[1]), add(p[2], p[3])), even, odd);
      r.s += even + odd;
    };
#pragma unroll
    for (int q = 0; q < 4; q++) {
      if (q == 0) asm volatile("cp.async.wait_group 3;" ::: "memory");
      if (q == 1) asm volatile("cp.async.wait_group 2;" ::: "memory");
      if (q == 2) asm volatile("cp.async.wait_group 1;" ::: "memory");
      if (q == 3) asm volatile("cp.async.wait_group 0;" ::: "memory");
      int i = q * quarter;
      const int end = min(steps, (q + 1) * quarter);
      for (; i + 2 <= end && (i + 1 < inner1 || (i + 1) * WALKERS + WALKERS <= units); i += 2) {     // two units at a time
        float y[8], w[8];
        const T *const at = buf + (i * WALKERS + tid) * 8;
        load8(at, y);
        load8(at + WALKERS * 8, w);
        const float top = fmaxf(largest(at), largest(at + WALKERS * 8));
        if (top > r.m) r.s *= exp_of(b, r.m == -INFINITY ? 0.0f : r.m - top), r.m = top;
        const float m = relative_to(r.m);
        Pair p[4], o[4];
        exp_of(b, m, y, p);
        exp_of(b, m, w, o);
        float even, odd;
        unpair(add(add(add(p[0], p[1]), add(p[2], p[3])), add(add(o[0], o[1]), add(o[2], o[3]))), even, odd);
        r.s += even + odd;
      }
      for (; i < end; i++)
        if (i * WALKERS + tid < units) seen(i * WALKERS + tid);
    }
    join_lanes(b, r);
    if (lane == 0) of_warp[warp] = make_float2(r.m, r.s);
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();
  if (MODE != GRADIENT) {
    r = Running{};
    if (there && lane < WALKERS / 32) r = Running{of_warp[lane].x, of_warp[lane].y};
    join_lanes(b, r);
    if (sl.n > 1) {                                      // the others have read their row's entries by the end of the wait: the output may be the input
      if (tid == 0) mine = make_float2(r.m, r.s);
      __syncwarp();
      cluster_arrive();
      cluster_wait();
      r = Running{};
      if (lane < sl.n) {
        const float2 v = of_cta(&mine, lane);
        r = Running{v.x, v.y};
      }
      __syncwarp();
      cluster_arrive();
      join_lanes(b, r);
    }
    if (r.m == -INFINITY) r.s = NAN;                     // no logit above -inf: there is no softmax
    if (rank == 0 && !walks) {
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
    if (!walks) {
    } else if (none) {
      if (sl.whole) {
        const float y[8] = {};
        for (int u = tid; u < n / 8; u += WALKERS) store8(d + u * 8, y);
        for (int c = n / 8 * 8 + tid; c < n; c += WALKERS) d[c] = from_f32<O>(0.0f);
      } else {
        for (int c = tid; c < n; c += WALKERS) d[c] = from_f32<O>(0.0f);
      }
    } else if (sl.whole && shift == 0) {
#pragma unroll 2
      for (int u = tid; u < n / 8; u += WALKERS) {
        float y[8];
        load8(buf + u * 8, y);
        Pair p[4];
        exp_of(b, r.m, y, p);
#pragma unroll
        for (int x = 0; x < 4; x++) unpair(mul(p[x], pair(of_q, of_q)), y[2 * x], y[2 * x + 1]);
        store8(d + u * 8, y);
      }
      for (int c = n / 8 * 8 + tid; c < n; c += WALKERS) d[c] = from_f32<O>(of_q * exp_of(b, to_f32(buf[c]) - r.m));
    } else {
      for (int c = tid; c < n; c += WALKERS) d[c] = from_f32<O>(of_q * exp_of(b, to_f32(buf[shift + c]) - r.m));
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
  sl->ahead = sl->look_first ? 3 * 148 / n : 0;
  return (size_t)sl->per * e <= SLICE_MOST && (long long)a.rows * n <= INT32_MAX;
}

template <typename T, typename O, int MODE> static cudaError_t rows_in_shared(const Distill &a, float b, const Slices &sl, cudaStream_t s) {
  static SmemLimit limit;
  const int units = sl.per / 8 + 1;
  const size_t smem = entries_bytes(a.K) + (size_t)units * 8 * sizeof(T);
  if (smem > 46 << 10 && !limit.ensure(distill_rows_kernel<T, O, MODE>, (int)smem)) return cudaErrorInvalidValue;
  if (!launch_allowed()) return cudaSuccess;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(a.rows * sl.n)), cfg.blockDim = dim3(WALKERS + 32), cfg.dynamicSmemBytes = smem, cfg.stream = s;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = sl.n, at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = MODE != GRADIENT && sl.n > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, distill_rows_kernel<T, O, MODE>, a, b, sl);
}
template <typename T, typename O> static cudaError_t rows_in_shared(const Distill &a, float b, const Slices &sl, cudaStream_t s) {
  return a.loss ? rows_in_shared<T, O, BOTH>(a, b, sl, s) : rows_in_shared<T, O, GRADIENT>(a, b, sl, s);
}

cudaError_t launch_distill(const Distill &a, cudaStream_t s) {
  const float b = (float)(1.4426950408889634 / a.temperature);
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
