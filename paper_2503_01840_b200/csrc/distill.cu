// Distillation from a teacher's top logits: loss = sum p (ln p - ln q) over the teacher's entries, q the student's softmax; its gradient dz = g / T (q sum p - p).
#include "distill.cuh"

#include <algorithm>

#include "vec.cuh"

namespace spec {

using std::max;
using std::min;

// exp(d / T) = 2^(d c), c = log2(e) / T.  c's own rounding is 2^-25 of the exponent at most, as much as the product's is.
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
  float *p, *ln_p;
  float *write;          // for the gradient: p of all entries with this id at the first of them, -1 at the others
  int *table;            // of the ids, or of the places of their first entries
};
__host__ __device__ constexpr int table_bits(int K) { return K <= 16 ? 6 : K <= 64 ? 8 : K <= 256 ? 10 : 12; }      // four places an entry, or more
__host__ __device__ constexpr size_t entries_bytes(int K) { return (size_t)K * 16 + ((size_t)4 << table_bits(K)); }      // the table, and what lies behind it, aligned to 16
__device__ __forceinline__ Entries entries_in(char *shared, int K) {
  float *const f = (float *)shared;
  return {(int *)f, f + K, f + 2 * K, f + 3 * K, (int *)f + 4 * K};
}
// One warp fills them in and returns sum p; *none: whether the row has no entry (sum p may be 0 otherwise too, where every p is too small).
__device__ __forceinline__ float read_entries(const Distill &a, const Entries &e, long long row, bool *none) {
  const int lane = threadIdx.x & 31;
  const float inv_t = 1.0f / a.temperature;
  const long long at = row * a.K;
  float top = -INFINITY;
  bool some = false, nan = false;
#pragma unroll 1
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
#pragma unroll 1
    for (int k = lane; k < a.K; k += 32)
      if (e.id[k] >= 0) sum += expf((e.ln_p[k] - top) * inv_t);
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    ln_sum = logf(sum);
  }
  float all = 0.0f;
#pragma unroll 1
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
// What the same warp does next for the gradient: entries with one id become one, its first.  A table of the ids tells whether there is anything to do.
// Loss and gradient of 8192 x 32000 bf16 with 64, 200, 1024 entries a row 195 / 275 / 1053 us; the last of them repeating the first 197 / 324 / 1401, each one's id twice 213 / 391 / 2017.
// (Comparing every entry with every other 324 / 2015 / 60234, and 320 / 1700 / 39449.)
__device__ __forceinline__ void merge_entries(const Entries &e, int K) {
  const int lane = threadIdx.x & 31, bits = table_bits(K), mask = (1 << bits) - 1;
  for (int k = lane; k <= mask >> 2; k += 32) ((int4 *)e.table)[k] = make_int4(-1, -1, -1, -1);
  __syncwarp();
  bool twice = false;
#pragma unroll 1
  for (int k = lane; k < K; k += 32) {
    const int id = e.id[k];
    e.write[k] = id < 0 ? -1.0f : e.p[k];
    if (id < 0) continue;
    int at = (int)((uint32_t)id * 2654435769u >> (32 - bits));      // 2^32 over the golden ratio spreads neighbours
    for (;;) {                                           // ends: a table is at most a quarter full
      const int was = atomicCAS(e.table + at, -1, id);
      twice |= was == id;
      if (was < 0 || was == id) break;
      at = (at + 1) & mask;
    }
  }
  __syncwarp();
  if (!__any_sync(0xffffffffu, twice)) return;
  // Again with the entries' places in the table, 32 entries at a time: the lowest lane of an id looks for the id's first entry, or is it, and adds its lanes' probabilities in turn.
  for (int k = lane; k <= mask >> 2; k += 32) ((int4 *)e.table)[k] = make_int4(-1, -1, -1, -1);
  __syncwarp();
#pragma unroll 1
  for (int k0 = 0; k0 < K; k0 += 32) {
    const int k = k0 + lane, id = k < K ? e.id[k] : -1;
    const uint32_t same = __match_any_sync(0xffffffffu, id);
    const bool leads = id >= 0 && (same & ((1u << lane) - 1)) == 0;
    const float p = id >= 0 ? e.p[k] : 0.0f;
    int first = k;
    if (leads) {
      int at = (int)((uint32_t)id * 2654435769u >> (32 - bits));
      for (;;) {                                         // ends as above; other lanes put other ids in
        const int was = atomicCAS(e.table + at, -1, k);
        if (was < 0) break;
        if (e.id[was] == id) {
          first = was;
          break;
        }
        at = (at + 1) & mask;
      }
    }
    __syncwarp();
    float sum = first == k ? p : e.write[first];
#pragma unroll 1
    for (uint32_t rest = __reduce_or_sync(0xffffffffu, leads ? first == k ? same & (same - 1) : same : 0u); rest; rest &= rest - 1) {
      const int j = __ffs(rest) - 1;
      const float other = __shfl_sync(0xffffffffu, p, j);
      if ((same >> j & 1) && (j != lane || first != k)) sum += other;
    }
    if (leads) e.write[first] = sum;
    if (id >= 0 && (!leads || first != k)) e.write[k] = -1.0f;
    __syncwarp();
  }
}
// A warp's sum over its lanes' entries of p (ln p - ln q), ln q without the logarithm of q's normaliser; z(id): the student's logit
template <typename F> __device__ __forceinline__ float entries_loss(const Distill &a, const Entries &e, float m, F z) {
  float loss = 0.0f;
#pragma unroll 1
  for (int k = threadIdx.x & 31; k < a.K; k += 32) {
    const float p = e.p[k];
    if (e.id[k] < 0 || p == 0.0f) continue;
    const float ln_q = (z(e.id[k]) - m) / a.temperature;
    loss += p * (a.kl ? e.ln_p[k] - ln_q : -ln_q);
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) loss += __shfl_xor_sync(0xffffffffu, loss, d);
  return loss;
}

// ---------------------------------------------------------------- any vocabulary: a block a row, read once for each step
__global__ void __launch_bounds__(512) distill_any_kernel(Distill a, float b) {
  pdl_wait();
  pdl_trigger();
  extern __shared__ __align__(16) char shared[];
  __shared__ float of_s[16], of_m[16], mass;
  __shared__ int empty;
  const Entries e = entries_in(shared, a.K);
  float *const kept = (float *)(shared + entries_bytes(a.K));     // the logits at the entries: the output may be the input
  const int tid = threadIdx.x;
  const long long row = blockIdx.x, z0 = row * a.z_rs, d0 = row * a.d_rs;
  if (tid < 32) {
    bool none;
    const float all = read_entries(a, e, row, &none);
    if (tid == 0) mass = all, empty = none;
    for (int k = tid; k < a.K; k += 32) kept[k] = e.id[k] >= 0 ? load_as_f32(a.z, a.z_type, z0 + e.id[k]) : 0.0f;
    if (a.dz) merge_entries(e, a.K);
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
  } else {
    r.m = a.stats[row].x, r.s = a.stats[row].y;
  }
  // loss and gradient at the entries, whose list gives the place
  if (tid < 32) {
    float loss = 0.0f;
    for (int k = tid; k < a.K; k += 32) {
      if (e.id[k] < 0 || e.p[k] == 0.0f) continue;
      const float ln_q = (kept[k] - r.m) / a.temperature;
      loss += e.p[k] * (a.kl ? e.ln_p[k] - ln_q : -ln_q);
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) loss += __shfl_xor_sync(0xffffffffu, loss, d);
    if (a.loss && tid == 0) {
      a.loss[row] = loss + all * logf(r.s);
      if (a.stats) a.stats[row] = make_float2(r.m, r.s);
    }
  }
  if (!a.dz) return;
  const float g = (a.grad ? a.grad[row] : 1.0f) / a.temperature, of_q = g * all / r.s;
  for (int c = tid; c < a.vocab; c += 512) store_from_f32(a.dz, a.d_type, d0 + c, of_q * exp_of(b, load_as_f32(a.z, a.z_type, z0 + c) - r.m));
  __syncthreads();
  for (int k = tid; k < a.K; k += 512)
    if (e.id[k] >= 0 && !(e.write[k] < 0.0f)) store_from_f32(a.dz, a.d_type, d0 + e.id[k], fmaf(of_q, exp_of(b, kept[k] - r.m), -g * e.write[k]));
}

// ---------------------------------------------------------------- rows held in shared memory
// A cluster of up to eight CTAs has a row, a slice of up to SLICE bytes each, read from memory once: copied to shared memory, walked for the maximum and the sum, which the CTAs
// exchange, and walked again for the gradient.  Where the statistics are given the CTAs have nothing to exchange and are no cluster.  Elements keep their place modulo 16 bytes, so any
// alignment will do; a thread copies and walks the same units of eight and waits for its own copies alone.  Meanwhile another warp looks the entries up (some four microseconds, most of
// them waiting), takes the loss, and writes over what the walkers wrote at the entries' ids.
// The gradient from statistics is bound by bytes: 2048 rows of 128256 fp32 to bf16 241 us, 6.5 TB/s, a copy's rate.  Loss and gradient at once wait, load, walk and write in turn, three
// CTAs an SM side by side: 8192 rows of 32000 bf16, a tenth of them without entries, 187 us, 5.4 TB/s, 82 % of a copy's; two exponentials an element are 116 us of its unit's time.
// Slices of 44 KB and four CTAs 292 / 259 us (clusters wait for one another), of 100 KB 196 / 247; 384 walkers 206 / 269.  CTAs that stay, with the next row's entries and copies under way,
// 244 / 299: their one look-up warp is what they wait for.  Rows that have no id are not read: 233 us without that, and 210 without the next entries' way into L2.  Loops stay rolled: two warps'
// paths have to stay in the instruction cache together, and the same loops unrolled, with fewer checks, take 205 to 218 us.  One unit a thread at a time 193 us, four 188.
enum { LOSS = 0, GRADIENT = 1, BOTH = 2 };
struct Slices {
  int n, per;            // slices of a row, elements of one: a multiple of 8
  int whole;             // units of the output are aligned pieces of 16 bytes
  int look_first;        // whether a row is not loaded before it is known that some id of it is not -1
  int ahead;             // rows that are under way at a time, if there are more: the entries of the row that far on go to L2
};
constexpr int SLICE = 66 << 10, SHARED_MOST = 224 << 10, CLUSTER_MOST = 8;

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ float2 of_cta(const float2 *p, int rank) {
  uint32_t at;
  float2 v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_of(p)), "r"(rank));
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(at) : "memory");
  return v;
}

// the largest of eight (of NaN and a number the number)
__device__ __forceinline__ float largest(const Raw8<float> &x) { return fmaxf(fmaxf(fmaxf(x.a.x, x.a.y), fmaxf(x.a.z, x.a.w)), fmaxf(fmaxf(x.b.x, x.b.y), fmaxf(x.b.z, x.b.w))); }
__device__ __forceinline__ float largest(const Raw8<bf16> &x) {
  const __nv_bfloat162 a = *(const __nv_bfloat162 *)&x.u.x, b = *(const __nv_bfloat162 *)&x.u.y, c = *(const __nv_bfloat162 *)&x.u.z, d = *(const __nv_bfloat162 *)&x.u.w;
  const __nv_bfloat162 m = __hmax2(__hmax2(a, b), __hmax2(c, d));
  return fmaxf(__low2float(m), __high2float(m));
}

constexpr int WALKERS = 256;      // threads that copy and walk; another warp looks the entries up and takes the loss
constexpr int UNITS = 2;          // that a thread walks at a time

// The part of N units in a thread's maximum and sum
template <int N, typename T> __device__ __forceinline__ Running walk(const Raw8<T> (&x)[N], float b, Running r) {
  float top = largest(x[0]);
#pragma unroll
  for (int i = 1; i < N; i++) top = fmaxf(top, largest(x[i]));
  if (top > r.m) r.s *= exp_of(b, r.m == -INFINITY ? 0.0f : r.m - top), r.m = top;
  const float m = relative_to(r.m);
  Pair s[4];
#pragma unroll
  for (int i = 0; i < N; i++) {
    float y[8];
    Pair p[4];
    x[i].floats(y);
    exp_of(b, m, y, p);
#pragma unroll
    for (int k = 0; k < 4; k++) s[k] = i ? add(s[k], p[k]) : p[k];
  }
  float even, odd;
  unpair(add(add(s[0], s[1]), add(s[2], s[3])), even, odd);
  r.s += even + odd;
  return r;
}

// an element of another CTA's shared memory, at the place that p has in this one's
__device__ __forceinline__ float of_cta(const float *p, int rank) {
  uint32_t at;
  float v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_of(p)), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ float of_cta(const bf16 *p, int rank) {
  uint32_t at;
  uint16_t v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_of(p)), "r"(rank));
  asm volatile("ld.shared::cluster.u16 %0, [%1];" : "=h"(v) : "r"(at) : "memory");
  return __uint_as_float((uint32_t)v << 16);
}
// the walkers have written the row's gradient: they go on, the other warp waits for them
__device__ __forceinline__ void written_arrive() {
  __syncwarp();
  asm volatile("bar.arrive 1, %0;" ::"n"(WALKERS + 32) : "memory");
}
__device__ __forceinline__ void written_wait() {
  __syncwarp();
  asm volatile("bar.sync 1, %0;" ::"n"(WALKERS + 32) : "memory");
}

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
  // what is needed later is asked for now, for this row and for the one that comes to this place on the SM next
  const float grad = MODE != LOSS && a.grad ? a.grad[row] : 1.0f;
  const float2 stats = MODE == GRADIENT ? a.stats[row] : make_float2(0.0f, 1.0f);
  if (!walks && sl.ahead && row + sl.ahead < a.rows) {
    const long long at = (row + sl.ahead) * a.K;
    const int ids = a.ids.wide ? 8 : 4, values = a.v_type == 0 ? 4 : 2;
    for (int k = lane * 32; k < a.K; k += 1024) {
      for (int x = 0; x < ids / 4 && k + 16 * x < a.K; x++) asm volatile("prefetch.global.L2 [%0];" ::"l"((const char *)a.ids.p + (at + k) * ids + x * 128));
      asm volatile("prefetch.global.L2 [%0];" ::"l"((const char *)a.values + (at + k) * values));
    }
  }
  const int steps = (units + WALKERS - 1) / WALKERS, quarter = (steps + 3) / 4;      // a unit of each thread a step
  auto copy_quarters = [&](int q0, int q1) {
#pragma unroll 1
    for (int q = q0; q < q1; q++) {
#pragma unroll 1
      for (int i = q * quarter; i < min(steps, (q + 1) * quarter); i++) {
        const int u = i * WALKERS + tid, c = u * 8 - shift;
        if (c >= 0 && c + 8 <= n) {
          copy8(buf + u * 8, z + c);
        } else if (u < units) {
#pragma unroll 1
          for (int x = 0; x < 8; x++) buf[u * 8 + x] = c + x >= 0 && c + x < n ? z[c + x] : from_f32<T>(-INFINITY);
        }
      }
      copies_commit();
    }
  };
  bool there = true;
  if (sl.look_first) {
    there = false;
#pragma unroll 1
    for (int k = 0; k < a.K && !there; k += 32) there = __any_sync(0xffffffffu, k + lane < a.K && id_at(a.ids, row * a.K + k + lane) != -1);
  }
  if (there && walks) {
    copy_quarters(0, 4);
  } else if (!walks) {
    bool none = true;
    if (there) {
      const float all = read_entries(a, e, row, &none);
      if (lane == 0) mass = all;
      if (MODE != LOSS && !none) merge_entries(e, a.K);
    }
    if (lane == 0) empty = none;
  }
  Running r;
  if (MODE != GRADIENT && there && walks) {
#pragma unroll 1
    for (int q = 0; q < 4; q++) {
      if (q == 0) copies_but<3>();
      if (q == 1) copies_but<2>();
      if (q == 2) copies_but<1>();
      if (q == 3) copies_but<0>();
      int i = q * quarter;
      const int end = min(steps, (q + 1) * quarter);
#pragma unroll 1
      for (; i + UNITS <= end && (i + UNITS) * WALKERS <= units; i += UNITS) {
        Raw8<T> x[UNITS];
#pragma unroll
        for (int k = 0; k < UNITS; k++) x[k].take(buf + ((i + k) * WALKERS + tid) * 8);
        r = walk<UNITS>(x, b, r);
      }
#pragma unroll 1
      for (; i < end; i++)
        if (i * WALKERS + tid < units) {
          Raw8<T> x[1];
          x[0].take(buf + (i * WALKERS + tid) * 8);
          r = walk<1>(x, b, r);
        }
    }
    join_lanes(b, r);
    if (lane == 0) of_warp[warp] = make_float2(r.m, r.s);
  }
  copies_but<0>();
  __syncthreads();
  const bool none = empty, joint = MODE != GRADIENT && sl.n > 1;
  if (MODE == GRADIENT) {
    r = Running{stats.x, stats.y};
  } else {
    r = Running{};
    if (there && lane < WALKERS / 32) r = Running{of_warp[lane].x, of_warp[lane].y};
    join_lanes(b, r);
    if (joint) {
      if (tid == 0) mine = make_float2(r.m, r.s);
      __syncwarp();
      cluster_arrive();
      cluster_wait();
      r = Running{};
      if (lane < sl.n) {
        const float2 v = of_cta(&mine, lane);
        r = Running{v.x, v.y};
      }
      join_lanes(b, r);
      if (walks) cluster_arrive();
    }
    if (r.m == -INFINITY) r.s = NAN;                     // no logit above -inf: there is no softmax
  }
  const float g = none ? 0.0f : grad / a.temperature, of_q = none ? 0.0f : g * mass / r.s;
  if (!walks) {                                          // while the others write
    if (MODE != GRADIENT && rank == 0) {
      auto logit = [&](int id) {
        if (!joint) return to_f32(buf[shift + id]);
        const int k = id / sl.per;
        return of_cta(buf + shift + (id - k * sl.per), k);
      };
      const float loss = none ? 0.0f : entries_loss(a, e, r.m, logit) + mass * logf(r.s);
      if (lane == 0) {
        a.loss[row] = loss;
        if (a.stats) a.stats[row] = none ? make_float2(0.0f, 1.0f) : make_float2(r.m, r.s);
      }
    }
    if (MODE != LOSS) {
      if (!none)
#pragma unroll 1
        for (int k = lane; k < a.K; k += 32) {           // what is written over theirs
          const int id = e.id[k];
          const float p = e.write[k];
          if (id >= c0 && id < c0 + n && !(p < 0.0f)) e.write[k] = fmaf(of_q, exp_of(b, to_f32(buf[shift + id - c0]) - r.m), -g * p);
          else e.id[k] = -1;
        }
      written_wait();
      if (!none)
#pragma unroll 1
        for (int k = lane; k < a.K; k += 32)
          if (e.id[k] >= 0) store_from_f32(a.dz, a.d_type, row * a.d_rs + e.id[k], e.write[k]);
    }
    __syncwarp();
    if (joint) cluster_arrive(), cluster_wait();         // nobody leaves while its numbers may be read
    return;
  }
  if (MODE != LOSS) {
    O *const d = (O *)a.dz + row * a.d_rs + c0;
    if (none) {
      if (sl.whole) {
        const float y[8] = {};
#pragma unroll 1
        for (int u = tid; u < n / 8; u += WALKERS) store8(d + u * 8, y);
        for (int c = n / 8 * 8 + tid; c < n; c += WALKERS) d[c] = from_f32<O>(0.0f);
      } else {
  #pragma unroll 1
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
#pragma unroll 1
      for (int c = n / 8 * 8 + tid; c < n; c += WALKERS) d[c] = from_f32<O>(of_q * exp_of(b, to_f32(buf[c]) - r.m));
    } else {
#pragma unroll 2
      for (int c = tid; c < n; c += WALKERS) d[c] = from_f32<O>(of_q * exp_of(b, to_f32(buf[shift + c]) - r.m));
    }
  }
  if (MODE != LOSS) written_arrive();
  __syncwarp();
  if (joint) cluster_wait();
}

// ---------------------------------------------------------------- the loss alone, of many rows
// A CTA a row, walked once as it comes from memory.  Bytes bound it in fp32: 2048 rows of 128256 154 us, 6.8 TB/s, a copy's rate; in bf16 unpacking and exponentials come near them: 8192 rows
// of 32000 109 us, 4.8 TB/s; 96 us, 4.9 TB/s of what is read, where a tenth of the rows have no entry and are not.  Where the first and the last of these took 155 / 103, by clusters through
// shared memory as above 315 / 132, four CTAs an SM 165 / 115, six 181 / 103.
template <typename T>
__global__ void __launch_bounds__(WALKERS + 32, 5) distill_loss_kernel(const __grid_constant__ Distill a, float b) {
  pdl_wait();
  pdl_trigger();
  extern __shared__ __align__(16) char shared[];
  __shared__ float2 of_warp[WALKERS / 32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long row = blockIdx.x;
  const T *const z = (const T *)a.z + row * a.z_rs;
  const Entries e = entries_in(shared, a.K);
  // a row without an id is not read
  bool there = false;
  for (int k = 0; k < a.K && !there; k += 32) there = __any_sync(0xffffffffu, k + lane < a.K && id_at(a.ids, row * a.K + k + lane) != -1);
  float all = 0.0f;
  bool none = true;
  if (!there) {
  } else if (tid >= WALKERS) {
    all = read_entries(a, e, row, &none);
  } else {
    // units of eight, aligned; what lies before and behind them an element a thread
    const int head = min(a.vocab, (int)((16 - (reinterpret_cast<uintptr_t>(z) & 15)) % 16 / sizeof(T))), units = (a.vocab - head) / 8, tail = head + units * 8;
    Running r;
    const int c = tid < head ? tid : tid < head + a.vocab - tail ? tail + tid - head : -1;      // fewer than 16
    if (c >= 0) r.m = to_f32(z[c]), r.s = exp_of(b, r.m - relative_to(r.m));
    if (r.m != r.m) r = Running{-INFINITY, NAN};
    constexpr int U = sizeof(T) == 4 ? 2 : 4;            // 64 bytes of a thread under way: with 128 of fp32 registers spill (238 us)
    for (int u = tid; u < units; u += U * WALKERS) {
      Raw8<T> x[U][1];
#pragma unroll
      for (int i = 0; i < U; i++)
        if (u + i * WALKERS < units) x[i][0].take(z + head + (u + i * WALKERS) * 8);
#pragma unroll
      for (int i = 0; i < U; i++)
        if (u + i * WALKERS < units) r = walk<1>(x[i], b, r);
    }
    join_lanes(b, r);
    if (lane == 0) of_warp[warp] = make_float2(r.m, r.s);
  }
  __syncthreads();
  if (tid < WALKERS) return;
  Running r;
  if (!none && lane < WALKERS / 32) r = Running{of_warp[lane].x, of_warp[lane].y};
  join_lanes(b, r);
  if (r.m == -INFINITY) r.s = NAN;
  const float loss = none ? 0.0f : entries_loss(a, e, r.m, [&](int id) { return to_f32(z[id]); }) + all * logf(r.s);
  if (lane) return;
  a.loss[row] = loss;
  if (a.stats) a.stats[row] = none ? make_float2(0.0f, 1.0f) : make_float2(r.m, r.s);
}

// Slices of about SLICE bytes, so that three CTAs are on an SM; smaller ones where rows alone do not fill the SMs twice, down to 2 KB.
static bool slices_of(const Distill &a, Slices *sl) {
  const size_t e = a.z_type == 0 ? 4 : 2, row = (size_t)a.vocab * e;
  const size_t most = a.loss ? CLUSTER_MOST : INT32_MAX;
  int n = (int)min((row + SLICE - 1) / SLICE, most);
  while (n < CLUSTER_MOST && (long long)a.rows * n < 2 * 148 && row / (n + 1) >= 2048) n++;
  sl->n = n;
  sl->per = (int)(((a.vocab + n - 1LL) / n + 7) / 8 * 8);
  sl->whole = a.dz && pieces_aligned(a.dz, a.rows > 1 ? a.d_rs : 0, a.d_type == 0 ? 4 : 2);
  sl->look_first = (long long)a.rows * n > 4 * 148;
  sl->ahead = sl->look_first ? 3 * 148 / n : 0;
  return (size_t)sl->per * e + entries_bytes(a.K) <= SHARED_MOST && (long long)a.rows * n <= INT32_MAX;
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
  const float b = (float)(1.4426950408889634 / a.temperature);      // log2(e) / T
  if (!a.dz && a.rows >= 2 * 148)
    return a.z_type == 0 ? launch_k(distill_loss_kernel<float>, dim3(a.rows), dim3(WALKERS + 32), entries_bytes(a.K), s, a, b)
                         : launch_k(distill_loss_kernel<bf16>, dim3(a.rows), dim3(WALKERS + 32), entries_bytes(a.K), s, a, b);
  Slices sl;
  if (!slices_of(a, &sl)) return launch_k(distill_any_kernel, dim3(a.rows), dim3(512), entries_bytes(a.K) + (size_t)a.K * 4, s, a, b);
  if (a.z_type == 0) {
    if (!a.dz) return rows_in_shared<float, float, LOSS>(a, b, sl, s);
    return a.d_type == 0 ? rows_in_shared<float, float>(a, b, sl, s) : rows_in_shared<float, bf16>(a, b, sl, s);
  }
  if (!a.dz) return rows_in_shared<bf16, bf16, LOSS>(a, b, sl, s);
  return a.d_type == 0 ? rows_in_shared<bf16, float>(a, b, sl, s) : rows_in_shared<bf16, bf16>(a, b, sl, s);
}

}  // namespace spec
