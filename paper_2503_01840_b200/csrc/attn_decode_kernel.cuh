// Attention of one new token per sequence over the paged cache:
//   out = sum_t p_t v_t / sum_t p_t,  p_t = exp(scale q.k_t - max),  lse = max + log sum_t p_t,   t < length of the sequence.
//
// Every key and value is read once and used for the few query heads that share it, so the cache's bytes bound it.  They are dealt out
// evenly: all tiles of TILE positions, of every sequence and KV head one after the other, are cut into equal runs for the CTAs
// (one wave of them), a CTA's run into equal runs for its warps.  A warp walks its run with a softmax state of its own; what is left
// of a (sequence, head) that several warps share is joined in shared memory, and of one that several CTAs share by the CTA that
// finishes last, out of the workspace, in the order of the positions whoever that is: the result does not depend on timing.
#pragma once
#include "attn_decode.cuh"

namespace spec {

constexpr int DA_MAX_CTAS = 304;           // CTAs of a launch, at most
constexpr int DA_PART_FLOATS = 8 * 256 + 16 * 2;      // a partial state: O of heads x hd <= 2048 elements, then (max, sum) of up to 16 heads

// workspace: partial states of each CTA's first and last segment, and a counter per CTA for the segment that starts in it
struct DaArgs {
  DecodeAttn a;
  int page_shift;               // log2 of the page size, or -1
  int heads, chunks;            // query heads a warp takes together, and how many such chunks share a KV head
  float *part;                  // [CTAs][2][DA_PART_FLOATS]
  unsigned *count;              // [CTAs], zero between calls
};

__host__ __device__ constexpr int da_part_floats(int heads, int hd) { return heads * hd + (2 * heads + 3) / 4 * 4; }

// A run of tiles of one (sequence, chunk of heads)
struct DaSeg {
  int b, v;                     // sequence; KV head * chunks + chunk
  int t0, t1, tiles;            // tiles t0 .. t1 - 1 of `tiles`
};

__device__ __forceinline__ float da_exp2(float x) { return exp2f(x); }
__device__ __forceinline__ float da_ref(float m) { return m == -INFINITY ? 0.0f : m; }      // keeps inf - inf out of a row whose scores are all -inf

__device__ __forceinline__ float da_inverse(float l) { return l == 0.0f ? 0.0f : 1.0f / l; }      // a row whose scores are all -inf gives 0

// first row (of hd elements) of a position of KV head g; -1 where the page is none of the pool's
__device__ __forceinline__ int da_row(const DaArgs &p, int b, int g, int pos) {
  const KvCache &c = p.a.cache;
  const int at = p.page_shift >= 0 ? pos >> p.page_shift : pos / c.page_size;
  const int page = c.table[(size_t)b * c.pages_per_seq + at];
  if (page < 0 || page >= c.num_pages) {
    set_status(p.a.status, ST_BOUNDS, 63, b, page);
    return -1;
  }
  return (page * c.G + g) * c.page_size + (pos - at * c.page_size);
}

// ---------------------------------------------------------------- the kernel
// tiles before sequence b, for every b; -1 and lengths past the cache are reported and clamped
__device__ __forceinline__ int da_length(const DaArgs &p, int b) {
  const int len = p.a.len[b];
  const long long cap = (long long)p.a.cache.pages_per_seq * p.a.cache.page_size;
  if (len < 0 || len > cap) {
    set_status(p.a.status, ST_BOUNDS, 62, b, len);
    return len < 0 ? 0 : (int)cap;
  }
  return len;
}

__device__ __forceinline__ void da_store(const DaArgs &p, bool f32, size_t at, float4 o) {
  if (f32) *(float4 *)((float *)p.a.out + at) = o;
  else {
    const __nv_bfloat162 lo = __floats2bfloat162_rn(o.x, o.y), hi = __floats2bfloat162_rn(o.z, o.w);
    *(uint2 *)((bf16 *)p.a.out + at) = make_uint2(*(const uint32_t *)&lo, *(const uint32_t *)&hi);
  }
}

// smem: int before[batch + 1] (tiles before each sequence), then per warp the body's floats and two partial states
template <typename Body>
__global__ void __launch_bounds__(Body::WARPS * 32, 1) decode_attn_kernel(DaArgs p, int q_f32) {
  pdl_wait();
  pdl_trigger();
  constexpr int W = Body::WARPS, THREADS = W * 32, TILE = Body::TILE;
  extern __shared__ __align__(16) char smem[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, B = p.a.batch, hd = p.a.cache.hd, group = p.a.H / p.a.cache.G;
  const int heads = p.heads, part_floats = da_part_floats(heads, hd);     // O [heads][hd], then (max, sum) [heads]
  int *before = (int *)smem;
  float *mem = (float *)(smem + ((size_t)(B + 1) * 4 + 15) / 16 * 16);
  float *warp_mem = mem + warp * Body::warp_smem_floats(hd);
  float *states = mem + W * Body::warp_smem_floats(hd);                  // [2 W][part_floats]
  __shared__ int scan[W];
  __shared__ DaSeg seg[2 * W];                                           // of the partial states; b = -1: none
  __shared__ unsigned last;

  // ---- tiles before each sequence: a run of sequences per thread, then a scan over the threads
  {
    const int per = (B + THREADS - 1) / THREADS, b0 = min(B, tid * per), b1 = min(B, b0 + per);
    int sum = 0;
    for (int b = b0; b < b1; b++) sum += (da_length(p, b) + TILE - 1) / TILE;
    int inc = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += x;
    }
    if (lane == 31) scan[warp] = inc;
    __syncthreads();
    int at = inc - sum;
    for (int w = 0; w < warp; w++) at += scan[w];
    for (int b = b0; b < b1; b++) {
      before[b] = at;
      at += (da_length(p, b) + TILE - 1) / TILE;
    }
    if (tid == THREADS - 1) before[B] = at;
    if (lane < 2) seg[2 * warp + lane].b = -1;
    __syncthreads();
  }
  const int VH = p.a.cache.G * p.chunks;
  const long long total = (long long)before[B] * VH;
  const int cta = blockIdx.x, N = (int)min((long long)gridDim.x, max(total, 1ll));      // CTAs that take part: a tile each at least
  const int c0 = cta < N ? (int)(total * cta / N) : 0, c1 = cta < N ? (int)(total * (cta + 1) / N) : 0;
  const int w0 = c0 + (int)((long long)(c1 - c0) * warp / W), w1 = c0 + (int)((long long)(c1 - c0) * (warp + 1) / W);
  auto out_at = [&](const DaSeg &s, int h) {                             // element of the output of a segment's head h
    return ((size_t)s.b * p.a.H + (s.v / p.chunks) * group + (s.v % p.chunks) * heads + h) * hd;
  };
  auto have = [&](const DaSeg &s) { return min(heads, group - (s.v % p.chunks) * heads); };

  // ---- sequences without a position
  for (int b = cta; b < B; b += gridDim.x)
    if (before[b + 1] == before[b]) {
      for (int i = tid * 4; i < p.a.H * hd; i += THREADS * 4) da_store(p, q_f32, (size_t)b * p.a.H * hd + i, make_float4(0.f, 0.f, 0.f, 0.f));
      if (p.a.lse)
        for (int h = tid; h < p.a.H; h += THREADS) p.a.lse[(size_t)b * p.a.H + h] = -INFINITY;
    }

  // ---- this warp's tiles
  int slot = 0;
  for (int u = w0; u < w1;) {
    DaSeg s;
    int lo = 0, hi = B;                                                  // the last sequence with before * VH <= u: it has tiles
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if ((long long)before[mid] * VH <= u) lo = mid;
      else hi = mid;
    }
    s.b = lo;
    s.tiles = before[lo + 1] - before[lo];
    const int r = u - before[lo] * VH;
    s.v = r / s.tiles;
    s.t0 = r - s.v * s.tiles;
    s.t1 = min(s.tiles, s.t0 + (w1 - u));
    u += s.t1 - s.t0;
    Body body;
    body.init(p, s, q_f32, warp_mem, lane);
    body.run(p, s, da_length(p, s.b), lane);
    const int nh = have(s);
    if (s.t0 == 0 && s.t1 == s.tiles) {
      body.each(hd, lane, [&](int h, int d, float4 o, float l) {
        if (h >= nh) return;
        const float f = da_inverse(l);
        da_store(p, q_f32, out_at(s, h) + d, make_float4(o.x * f, o.y * f, o.z * f, o.w * f));
      }, [&](int h, float m, float l) {
        if (h < nh && p.a.lse) p.a.lse[out_at(s, h) / hd] = (da_ref(m) + log2f(l)) * 0.693147180559945309f;
      });
    } else {
      float *st = states + (size_t)(2 * warp + slot) * part_floats;
      body.each(hd, lane, [&](int h, int d, float4 o, float) {
        if (h < heads) *(float4 *)(st + h * hd + d) = o;
      }, [&](int h, float m, float l) {
        if (h < heads) *(float2 *)(st + heads * hd + 2 * h) = make_float2(m, l);
      });
      if (lane == 0) seg[2 * warp + slot] = s;
      slot++;                                                            // only a run's first and last segment can be parts
    }
  }
  __syncthreads();

  // ---- what this CTA's warps share: partial states i .. j of one segment, in the order of the positions
  const int hv = hd / 4;
  // joins n states; st(k): the k-th.  Writes the output, or to `to` a joined state.
  auto join = [&](const DaSeg &s, int n, auto st, float *to) {
    const int nh = have(s);
    for (int i = tid; i < nh * hv; i += THREADS) {
      const int h = i / hv, d = (i - h * hv) * 4;
      float m = -INFINITY, l = 0.0f;
      for (int k = 0; k < n; k++) m = fmaxf(m, st(k)[heads * hd + 2 * h]);
      const float ref = da_ref(m);
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int k = 0; k < n; k++) {
        const float *x = st(k);
        const float2 ml = *(const float2 *)(x + heads * hd + 2 * h);
        const float4 y = *(const float4 *)(x + h * hd + d);
        const float f = da_exp2(ml.x - ref);
        l = fmaf(ml.y, f, l);
        o.x = fmaf(y.x, f, o.x), o.y = fmaf(y.y, f, o.y), o.z = fmaf(y.z, f, o.z), o.w = fmaf(y.w, f, o.w);
      }
      if (to) {
        *(float4 *)(to + h * hd + d) = o;
        if (d == 0) *(float2 *)(to + heads * hd + 2 * h) = make_float2(m, l);
      } else {
        const float f = da_inverse(l);
        da_store(p, q_f32, out_at(s, h) + d, make_float4(o.x * f, o.y * f, o.z * f, o.w * f));
        if (d == 0 && p.a.lse) p.a.lse[out_at(s, h) / hd] = (ref + log2f(l)) * 0.693147180559945309f;
      }
    }
  };
  for (int i = 0; i < 2 * W;) {
    if (seg[i].b < 0) { i++; continue; }
    DaSeg s = seg[i];
    int j = i, n = 0;
    short at[2 * W];
    while (j < 2 * W && (seg[j].b < 0 || (seg[j].b == s.b && seg[j].v == s.v))) {
      if (seg[j].b >= 0) {
        s.t1 = seg[j].t1;
        at[n++] = (short)j;
      }
      j++;
    }
    i = j;
    auto mine = [&](int k) { return states + (size_t)at[k] * part_floats; };
    if (s.t0 == 0 && s.t1 == s.tiles) {
      join(s, n, mine, nullptr);
      continue;
    }
    // other CTAs have the rest of it: the one that starts it keeps its count
    float *const part = p.part;
    join(s, n, mine, part + (size_t)(2 * cta + (s.t0 == 0)) * DA_PART_FLOATS);
    const long long u0 = (long long)before[s.b] * VH + (long long)s.v * s.tiles;
    const int first = (int)(((u0 + 1) * N - 1) / total), final_ = (int)(((u0 + s.tiles) * N - 1) / total);
    __threadfence();
    __syncthreads();
    if (tid == 0) last = atomicAdd(p.count + first, 1u) == (unsigned)(final_ - first);
    __syncthreads();
    if (last) {
      __threadfence();
      if (tid == 0) p.count[first] = 0;                                  // as the next call wants it
      join(s, final_ - first + 1, [&](int k) { return part + (size_t)(2 * (first + k) + (k == 0)) * DA_PART_FLOATS; }, nullptr);
    }
    __syncthreads();
  }
}

constexpr size_t DA_SMEM = 224 * 1024;
inline size_t da_smem_bytes(int batch, int warps, int own_floats, int heads, int hd) {
  return ((size_t)(batch + 1) * 4 + 15) / 16 * 16 + sizeof(float) * warps * (own_floats + 2 * da_part_floats(heads, hd));
}
template <typename Body> static cudaError_t launch(const DaArgs &p, bool q_f32, int ctas, cudaStream_t s) {
  static SmemLimit limit;
  const long long tiles = ((long long)p.a.cache.pages_per_seq * p.a.cache.page_size + Body::TILE - 1) / Body::TILE;
  if (tiles * p.a.batch * p.a.cache.G * p.chunks > INT32_MAX) return cudaErrorNotSupported;
  const size_t smem = da_smem_bytes(p.a.batch, Body::WARPS, Body::warp_smem_floats(p.a.cache.hd), p.heads, p.a.cache.hd);
  if (smem > DA_SMEM || !limit.ensure(decode_attn_kernel<Body>, (int)smem)) return cudaErrorInvalidValue;
  return launch_k(decode_attn_kernel<Body>, dim3(ctas), dim3(Body::WARPS * 32), smem, s, p, (int)q_f32);
}

cudaError_t launch_decode_fma(const DaArgs &p, int fmt, bool q_f32, int ctas, cudaStream_t s);
cudaError_t launch_decode_mma(const DaArgs &p, int fmt, int ctas, cudaStream_t s);

}  // namespace spec
