// Attention of one new token per sequence over the paged cache:
//   out = sum_t p_t v_t / sum_t p_t,  p_t = exp(scale q.k_t - max),  lse = max + log sum_t p_t,   t < length of the sequence.
//
// Every key and value is read once and used for the few query heads that share it, so the cache's bytes bound it.  They are dealt out
// evenly: all tiles of TILE positions, of every sequence and KV head one after the other, are cut into equal runs for the CTAs
// (one wave of them), a CTA's run into equal runs for its warps.  A warp walks its run with a softmax state of its own; what is left
// of a (sequence, head) that several warps share is joined in shared memory, and of one that several CTAs share by the CTA that
// finishes last, out of the workspace, in the order of the positions whoever that is: the result does not depend on timing.
#include "attn_decode.cuh"

#include <algorithm>

namespace spec {

constexpr int DA_MAX_CTAS = 304;           // CTAs of a launch, at most
constexpr int DA_PART_FLOATS = 8 * 256 + 16 * 2;      // a partial state: O of heads x hd <= 2048 elements, then (max, sum) of up to 16 heads

// workspace: partial states of each CTA's first and last segment, and a counter per CTA for the segment that starts in it
size_t decode_attn_workspace_bytes() { return (size_t)DA_MAX_CTAS * (2 * DA_PART_FLOATS * sizeof(float) + 64); }

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

// first row (of hd elements) of a position of KV head g; positions past the sequence or pages outside the pool: -1
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

// ---------------------------------------------------------------- plain-FMA body
// A lane takes a position's whole score; then LPT lanes share a position's values, DV vectors of four dimensions each.
template <int FMT_, int HP_, int DCLASS> struct FmaBody {
  static constexpr int FMT = FMT_, HP = HP_, TILE = 32, WARPS = 8;
  static constexpr int LPT = DCLASS == 64 ? 16 : 32, NV = DCLASS == 256 ? 2 : 1, PER = 32 / LPT;
  typedef typename KvElem<FMT>::type E;
  static constexpr int VEC = 16 / sizeof(E);
  static __host__ __device__ int warp_smem_floats(int hd) { return HP * hd + 64; }

  float m[HP], l[HP], acc[HP][NV][4];
  float *qs;                    // [HP][hd], times scale * log2 e

  __device__ void init(const DaArgs &p, const DaSeg &sg, bool q_f32, float *mem, int lane) {
    qs = mem;
    const int hd = p.a.cache.hd, group = p.a.H / p.a.cache.G, h0 = (sg.v / p.chunks) * group + (sg.v % p.chunks) * p.heads;
    const int have = min(p.heads, group - (sg.v % p.chunks) * p.heads);
    __syncwarp();
    for (int i = lane; i < HP * hd; i += 32) {
      const int h = i / hd;
      const size_t at = (size_t)sg.b * p.a.q_ts + (size_t)(h0 + h) * hd + (i - h * hd);
      qs[i] = h < have ? (q_f32 ? ((const float *)p.a.q)[at] : to_f32(((const bf16 *)p.a.q)[at])) * (p.a.scale * 1.44269504088896341f) : 0.0f;
    }
    __syncwarp();
#pragma unroll
    for (int h = 0; h < HP; h++) {
      m[h] = -INFINITY, l[h] = 0.0f;
#pragma unroll
      for (int j = 0; j < NV; j++)
#pragma unroll
        for (int e = 0; e < 4; e++) acc[h][j][e] = 0.0f;
    }
  }

  static __device__ __forceinline__ void unpack(const uint4 &u, float (&x)[VEC]) {
    const E *e = (const E *)&u;
#pragma unroll
    for (int i = 0; i < VEC; i++) x[i] = kv_decode<FMT>(e[i]);
  }

  __device__ void run(const DaArgs &p, const DaSeg &sg, int len, int lane) {
    const KvCache &c = p.a.cache;
    const int hd = c.hd, g = sg.v / p.chunks;
    const E *K = (const E *)c.k, *V = (const E *)c.v;
    for (int t = sg.t0; t < sg.t1; t++) {
      const int pos = t * TILE + lane, n = min(TILE, len - t * TILE);
      const int row = pos < len ? da_row(p, sg.b, g, pos) : -1;
      float s[HP];
#pragma unroll
      for (int h = 0; h < HP; h++) s[h] = 0.0f;
      float vsc = 1.0f;
      if (row >= 0) {
        const uint4 *kr = (const uint4 *)(K + (size_t)row * hd);
#pragma unroll 4
        for (int i = 0; i < hd / VEC; i++) {
          float x[VEC];
          unpack(kr[i], x);
#pragma unroll
          for (int h = 0; h < HP; h++)
#pragma unroll
            for (int e = 0; e < VEC; e += 4) {
              const float4 w = *(const float4 *)(qs + h * hd + i * VEC + e);
              s[h] = fmaf(w.x, x[e], fmaf(w.y, x[e + 1], fmaf(w.z, x[e + 2], fmaf(w.w, x[e + 3], s[h]))));
            }
        }
        if constexpr (kv_is_8bit(FMT)) {
          const float ksc = c.ks[row];
          vsc = c.vs[row];
#pragma unroll
          for (int h = 0; h < HP; h++) s[h] *= ksc;
        }
      }
#pragma unroll
      for (int h = 0; h < HP; h++) {
        if (row < 0) s[h] = -INFINITY;
        float mx = s[h];
#pragma unroll
        for (int o = 16; o; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
        mx = fmaxf(mx, m[h]);
        const float f = da_exp2(m[h] - da_ref(mx));
        s[h] = da_exp2(s[h] - da_ref(mx));
        m[h] = mx;
        l[h] = l[h] * f + s[h];                                // each lane its own positions' sum
#pragma unroll
        for (int j = 0; j < NV; j++)
#pragma unroll
          for (int e = 0; e < 4; e++) acc[h][j][e] *= f;
        s[h] *= vsc;
      }
      const int dim = (lane % LPT) * 4;
#pragma unroll 4
      for (int j = 0; j < n; j += PER) {
        const int from = PER == 1 ? j : j + lane / LPT;
        const int r = __shfl_sync(0xffffffffu, row, from);
        float x[NV][4];
#pragma unroll
        for (int i = 0; i < NV; i++) {
          const int d = dim + i * 128;
#pragma unroll
          for (int e = 0; e < 4; e++) x[i][e] = 0.0f;
          if (r >= 0 && d < hd) {
            struct alignas(4 * sizeof(E)) Four { E e[4]; };
            const Four u = *(const Four *)(V + (size_t)r * hd + d);
#pragma unroll
            for (int e = 0; e < 4; e++) x[i][e] = kv_decode<FMT>(u.e[e]);
          }
        }
#pragma unroll
        for (int h = 0; h < HP; h++) {
          const float w = __shfl_sync(0xffffffffu, s[h], from);
          if (r < 0) continue;
#pragma unroll
          for (int i = 0; i < NV; i++)
#pragma unroll
            for (int e = 0; e < 4; e++) acc[h][i][e] = fmaf(w, x[i][e], acc[h][i][e]);
        }
      }
    }
#pragma unroll
    for (int h = 0; h < HP; h++) {
#pragma unroll
      for (int o = 16; o; o >>= 1) l[h] += __shfl_xor_sync(0xffffffffu, l[h], o);
      if constexpr (PER == 2) {
#pragma unroll
        for (int e = 0; e < 4; e++) acc[h][0][e] += __shfl_xor_sync(0xffffffffu, acc[h][0][e], 16);
      }
    }
  }

  // f(head, dimension, four values of O) by the lanes that hold them; stat(head, max, sum) by lane 0
  template <typename F, typename G> __device__ void each(int hd, int lane, F f, G stat) {
#pragma unroll
    for (int h = 0; h < HP; h++) {
      if (lane < LPT)
#pragma unroll
        for (int i = 0; i < NV; i++)
          if (lane * 4 + i * 128 < hd) f(h, lane * 4 + i * 128, make_float4(acc[h][i][0], acc[h][i][1], acc[h][i][2], acc[h][i][3]));
      if (lane == 0) stat(h, m[h], l[h]);
    }
  }
};

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
      body.each(hd, lane, [&](int h, int d, float4 o) {
        if (h >= nh) return;
        const float f = body.l[h] > 0.0f ? 1.0f / body.l[h] : body.l[h] == 0.0f ? 0.0f : NAN;
        da_store(p, q_f32, out_at(s, h) + d, make_float4(o.x * f, o.y * f, o.z * f, o.w * f));
      }, [&](int h, float m, float l) {
        if (h < nh && p.a.lse) p.a.lse[out_at(s, h) / hd] = (da_ref(m) + log2f(l)) * 0.693147180559945309f;
      });
    } else {
      float *st = states + (size_t)(2 * warp + slot) * part_floats;
      body.each(hd, lane, [&](int h, int d, float4 o) {
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
        const float f = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : NAN;
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
template <typename Body> static size_t smem_bytes(int batch, int heads, int hd) {
  return ((size_t)(batch + 1) * 4 + 15) / 16 * 16 + sizeof(float) * Body::WARPS * (Body::warp_smem_floats(hd) + 2 * da_part_floats(heads, hd));
}
template <typename Body> static cudaError_t launch(const DaArgs &p, bool q_f32, int ctas, cudaStream_t s) {
  static SmemLimit limit;
  const long long tiles = ((long long)p.a.cache.pages_per_seq * p.a.cache.page_size + Body::TILE - 1) / Body::TILE;
  if (tiles * p.a.batch * p.a.cache.G * p.chunks > INT32_MAX) return cudaErrorNotSupported;
  const size_t smem = smem_bytes<Body>(p.a.batch, p.heads, p.a.cache.hd);
  if (smem > DA_SMEM || !limit.ensure(decode_attn_kernel<Body>, (int)smem)) return cudaErrorInvalidValue;
  return launch_k(decode_attn_kernel<Body>, dim3(ctas), dim3(Body::WARPS * 32), smem, s, p, (int)q_f32);
}

template <int FMT, int HP> static cudaError_t fma_by_hd(const DaArgs &p, bool q_f32, int ctas, cudaStream_t s) {
  const int hd = p.a.cache.hd;
  if (hd <= 64) return launch<FmaBody<FMT, HP, 64>>(p, q_f32, ctas, s);
  if (hd <= 128) return launch<FmaBody<FMT, HP, 128>>(p, q_f32, ctas, s);
  return launch<FmaBody<FMT, HP, 256>>(p, q_f32, ctas, s);
}
template <int FMT> static cudaError_t fma_by_heads(const DaArgs &p, bool q_f32, int ctas, cudaStream_t s) {
  if (p.heads <= 1) return fma_by_hd<FMT, 1>(p, q_f32, ctas, s);
  if (p.heads <= 2) return fma_by_hd<FMT, 2>(p, q_f32, ctas, s);
  if (p.heads <= 4) return fma_by_hd<FMT, 4>(p, q_f32, ctas, s);
  return fma_by_hd<FMT, 8>(p, q_f32, ctas, s);
}

cudaError_t launch_decode_attn(const DecodeAttn &a, int dtype, int fmt, cudaStream_t s) {
  DaArgs p{};
  p.a = a;
  p.page_shift = (a.cache.page_size & (a.cache.page_size - 1)) == 0 ? __builtin_ctz(a.cache.page_size) : -1;
  const int group = a.H / a.cache.G;
  // up to eight heads at a time, fewer where a large batch's table leaves no room for their partial states
  int most = 8;
  while (most > 1 && smem_bytes<FmaBody<KV_F32, 8, 256>>(a.batch, most, a.cache.hd) > DA_SMEM) most /= 2;
  p.chunks = (group + most - 1) / most;
  p.heads = (group + p.chunks - 1) / p.chunks;
  p.part = (float *)a.workspace;
  p.count = (unsigned *)(p.part + (size_t)DA_MAX_CTAS * 2 * DA_PART_FLOATS);
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return e;
  const int ctas = std::min(sms, DA_MAX_CTAS);
  const bool q_f32 = dtype == KV_F32;
  switch (fmt) {
    case KV_F32: return fma_by_heads<KV_F32>(p, q_f32, ctas, s);
    case KV_BF16: return fma_by_heads<KV_BF16>(p, q_f32, ctas, s);
    case KV_E4M3: return fma_by_heads<KV_E4M3>(p, q_f32, ctas, s);
    default: return fma_by_heads<KV_INT8>(p, q_f32, ctas, s);
  }
}

}  // namespace spec
