// Rotary positions, writing keys and values into the paged cache (rotated and quantised on the way), reading positions of it back.
//
// Rotation: the pair (a, b) of a head's dimensions at position p becomes m (a cos t - b sin t, b cos t + a sin t), t = p f; its
// gradient is the transposed matrix, -t for t.  Quantisation, for each token and head: scale = max(amax / top, 2^-120) over the
// rotated 32-bit values, code = round(x / scale).  A row with an infinity or a NaN gets a scale of NaN and reads
// back as NaN throughout.
#include "kv_cache.cuh"

#include <algorithm>

namespace spec {

using std::max;
using std::min;

constexpr int ROPE_THREADS = 256, ROPE_MAX_HD = 256;

// ---------------------------------------------------------------- any head size up to 256, any strides
// A block per token, a warp per head: a lane holds dimensions lane, lane + 32, ...
template <typename T, int FMT>
__global__ void __launch_bounds__(ROPE_THREADS) rope_append_any_kernel(RopeAppend a) {
  pdl_wait();
  pdl_trigger();
  typedef typename KvElem<FMT>::type E;
  __shared__ float2 cs[ROPE_MAX_HD / 2];
  const int t = blockIdx.x, lane = threadIdx.x & 31, half = a.rope.half, hd = a.hd;
  if (half) {
    const int pos = a.pos[t];
    for (int i = threadIdx.x; i < half; i += ROPE_THREADS) cs[i] = rope_angle(a.rope, pos, i);
  }
  __shared__ int row0;
  if (threadIdx.x == 0) row0 = a.k.p ? kv_row(a.cache, a.seq[t], a.kvpos[t], a.status, t) : -1;
  __syncthreads();
  const int G = a.k.p ? a.cache.G : 0;
  for (int i = threadIdx.x >> 5; i < a.H + 2 * G; i += ROPE_THREADS / 32) {
    const int kind = i < a.H ? 0 : i < a.H + G ? 1 : 2, h = kind == 0 ? i : kind == 1 ? i - a.H : i - a.H - G;
    if (kind && row0 < 0) continue;
    const HeadView &src = kind == 0 ? a.q : kind == 1 ? a.k : a.v;
    const T *x = (const T *)src.p + t * src.ts + h * src.hs;
    float y[ROPE_MAX_HD / 32];
    uint32_t top = 0;                                    // bits of the largest magnitude: NaN counts as the largest of all
#pragma unroll
    for (int j = 0; j < ROPE_MAX_HD / 32; j++) {
      const int d = lane + j * 32;
      if (d >= hd) continue;
      const float v = to_f32(x[d]);
      y[j] = v;
      if (kind < 2 && d < 2 * half) {
        const bool second = a.rope.interleaved ? d & 1 : d >= half;
        const float2 c = cs[a.rope.interleaved ? d >> 1 : second ? d - half : d];
        const float w = to_f32(x[a.rope.interleaved ? d ^ 1 : second ? d - half : d + half]);
        y[j] = second ? fmaf(v, c.x, w * c.y) : fmaf(v, c.x, -(w * c.y));
      }
      top = max(top, __float_as_uint(y[j]) & 0x7fffffffu);
    }
    __syncwarp();                                        // the output may be the input
    if (kind == 0) {
      T *o = (T *)a.q_out + t * a.qo_ts + h * a.qo_hs;
#pragma unroll
      for (int j = 0; j < ROPE_MAX_HD / 32; j++)
        if (lane + j * 32 < hd) o[lane + j * 32] = from_f32<T>(y[j]);
      continue;
    }
    const size_t row = (uint32_t)(row0 + h * a.cache.page_size);
    E *o = (E *)(kind == 1 ? a.cache.k : a.cache.v) + row * hd;
    if constexpr (kv_is_8bit(FMT)) {
      const float scale = kv_scale<FMT>(__reduce_max_sync(0xffffffffu, top)), inv = 1.0f / scale;
#pragma unroll
      for (int j = 0; j < ROPE_MAX_HD / 32; j++)
        if (lane + j * 32 < hd) o[lane + j * 32] = (E)kv_encode4<FMT>(y[j] * inv, 0.0f, 0.0f, 0.0f);
      if (lane == 0) (kind == 1 ? a.cache.ks : a.cache.vs)[row] = scale;
    } else {
#pragma unroll
      for (int j = 0; j < ROPE_MAX_HD / 32; j++)
        if (lane + j * 32 < hd) o[lane + j * 32] = from_f32<E>(y[j]);
    }
  }
}

// ---------------------------------------------------------------- heads of whole 16-byte pieces
// A head is shared by LH lanes, a power of two, each with two 16-byte pieces: the two whose elements pair up in the half layout,
// neighbours in the interleaved one and past the rotated dimensions.  So a pair never leaves a lane, and a head's largest magnitude is LH
// lanes' exchange.  A block takes some heads of some tokens; their cosines and sines are formed once, in shared memory.
// Bytes bound it: a thread asks for its first U heads before it forms the angles.  Measured: 16384 tokens of 40 heads of 128 in bf16 57 us
// (5.9 TB/s, 92 % of a copy's rate), 4096 of 80 heads in fp32 53 us (6.3 TB/s); with keys and values to e4m3 as well, 16384 of 32 + 8 + 8 heads,
// 69 us (5.4 TB/s): the look-ups of the cache rows stand before a block's first store.  One head under way a thread and six blocks an SM; with two and five
// 61 / 53 / 72 us, one and eight 57 / 54 / 82; with two rounds a block instead of six 64 / 53 / 94, two heads and eight rounds 62 / 53 / 74; one wave of blocks that walk tokens with
// copies to shared memory four heads ahead 59 / 81 / 79; with 64-bit offsets 59 / 54 / 74.
__device__ __forceinline__ void unpack_piece(uint4 u, float (&y)[4]) {
  y[0] = __uint_as_float(u.x), y[1] = __uint_as_float(u.y), y[2] = __uint_as_float(u.z), y[3] = __uint_as_float(u.w);
}
__device__ __forceinline__ void unpack_piece(uint4 u, float (&y)[8]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; i++) y[2 * i] = __uint_as_float(w[i] << 16), y[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
}
__device__ __forceinline__ uint4 pack_piece(const float (&y)[4]) {
  return make_uint4(__float_as_uint(y[0]), __float_as_uint(y[1]), __float_as_uint(y[2]), __float_as_uint(y[3]));
}
__device__ __forceinline__ uint4 pack_piece(const float (&y)[8]) {
  return make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
}
struct RopeGrid {
  int per_block, heads;         // tokens and heads of a block
  int lh_shift;                 // log2 of LH
  uint32_t by_heads, by_half;   // ceil(2^32 / heads), / pairs: quotients of the small numbers here by a product
  int q_ts, q_hs, k_ts, k_hs, v_ts, v_hs, o_ts, o_hs;      // strides: within a block offsets are 32-bit, which halves their instructions
};
constexpr int ROPE_MAX_TOKENS = 16;

template <int N> __device__ __forceinline__ void turn_neighbours(float (&y)[N], const float (&c)[N / 2], const float (&s)[N / 2]) {
#pragma unroll
  for (int i = 0; i < N; i += 2) {
    const float p = y[i], q = y[i + 1];
    y[i] = fmaf(p, c[i / 2], -(q * s[i / 2])), y[i + 1] = fmaf(q, c[i / 2], p * s[i / 2]);
  }
}

template <typename T, int FMT, bool INTER, int U>
__global__ void __launch_bounds__(ROPE_THREADS, 6) rope_append_kernel(const __grid_constant__ RopeAppend a, const __grid_constant__ RopeGrid gr) {
  pdl_wait();
  pdl_trigger();
  typedef typename KvElem<FMT>::type E;
  constexpr int VE = 16 / sizeof(T);
  extern __shared__ __align__(16) float trig[];          // [tokens][cos half | sin half]
  __shared__ int rows[ROPE_MAX_TOKENS];
  const int tid = threadIdx.x, hd = a.hd, half = a.rope.half, G = a.k.p ? a.cache.G : 0;
  const int t0 = blockIdx.x * gr.per_block, nt = min(gr.per_block, a.tokens - t0), h0 = blockIdx.y * gr.heads, nh = min(gr.heads, a.H + 2 * G - h0);
  const int l = tid & ((1 << gr.lh_shift) - 1), slot = tid >> gr.lh_shift, step = ROPE_THREADS >> gr.lh_shift;
  // this lane's two pieces of a head (in elements), and whether they turn
  const bool paired = !INTER && l * VE < half;
  const int d0 = paired ? l * VE : 2 * l * VE, d1 = paired ? half + l * VE : d0 + VE;
  const bool turn0 = INTER ? d0 < 2 * half : paired, turn1 = INTER ? d1 < 2 * half : paired;

  const T *const q = (const T *)a.q.p + (long long)t0 * a.q.ts, *const k = (const T *)a.k.p + (long long)t0 * a.k.ts, *const v = (const T *)a.v.p + (long long)t0 * a.v.ts;
  T *const q_out = (T *)a.q_out + (long long)t0 * a.qo_ts;
  uint4 x[U][2];
  int of_t[U], of_h[U];                                  // token and head; token -1: there is none
  auto load = [&](int j0) {
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int j = j0 + u * step, t = (int)__umulhi((uint32_t)j, gr.by_heads), i = j - t * gr.heads, h = h0 + i;
      of_t[u] = -1, of_h[u] = h;
      if (t >= nt || i >= nh) continue;
      of_t[u] = t;
      const T *p = h < a.H ? q + (t * gr.q_ts + h * gr.q_hs) : h < a.H + G ? k + (t * gr.k_ts + (h - a.H) * gr.k_hs) : v + (t * gr.v_ts + (h - a.H - G) * gr.v_hs);
      x[u][0] = *(const uint4 *)(p + d0), x[u][1] = *(const uint4 *)(p + d1);
    }
  };
  load(slot);
  for (int i = tid; i < nt * half; i += ROPE_THREADS) {
    const int t = (int)__umulhi((uint32_t)i, gr.by_half), pair = i - t * half;
    const float2 c = rope_angle(a.rope, a.pos[t0 + t], pair);
    trig[t * 2 * half + pair] = c.x;
    trig[t * 2 * half + half + pair] = c.y;
  }
  if (G && tid < nt) rows[tid] = kv_row(a.cache, a.seq[t0 + tid], a.kvpos[t0 + tid], a.status, t0 + tid);
  __syncthreads();
  const int most = nt * gr.heads;
  for (int j0 = slot; j0 < most; j0 += U * step) {
    if (j0 != slot) load(j0);
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int t = of_t[u], h = of_h[u];
      if (t < 0) continue;
      float y0[VE], y1[VE];
      unpack_piece(x[u][0], y0);
      unpack_piece(x[u][1], y1);
      if (h < a.H + G) {
        const float *cs = trig + t * 2 * half, *sn = cs + half;
        if constexpr (INTER) {
          struct alignas(2 * VE) Some { float f[VE / 2]; };
          if (turn0) turn_neighbours(y0, (*(const Some *)(cs + d0 / 2)).f, (*(const Some *)(sn + d0 / 2)).f);
          if (turn1) turn_neighbours(y1, (*(const Some *)(cs + d1 / 2)).f, (*(const Some *)(sn + d1 / 2)).f);
        } else if (paired) {
#pragma unroll
          for (int i = 0; i < VE; i += 4) {
            const float4 c = *(const float4 *)(cs + d0 + i), s = *(const float4 *)(sn + d0 + i);
            const float cc[4] = {c.x, c.y, c.z, c.w}, ss[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
            for (int e = 0; e < 4; e++) {
              const float p = y0[i + e], q = y1[i + e];
              y0[i + e] = fmaf(p, cc[e], -(q * ss[e])), y1[i + e] = fmaf(q, cc[e], p * ss[e]);
            }
          }
        }
      }
      if (h < a.H) {
        T *o = q_out + (t * gr.o_ts + h * gr.o_hs);
        *(uint4 *)(o + d0) = pack_piece(y0);
        *(uint4 *)(o + d1) = pack_piece(y1);
        continue;
      }
      if (rows[t] < 0) continue;                         // all lanes of a head alike
      const bool key = h < a.H + G;
      const size_t row = (uint32_t)(rows[t] + (key ? h - a.H : h - a.H - G) * a.cache.page_size);
      E *o = (E *)(key ? a.cache.k : a.cache.v) + row * hd;
      if constexpr (kv_is_8bit(FMT)) {
        uint32_t top = 0;                                // bits of the largest magnitude: NaN counts as the largest of all
#pragma unroll
        for (int i = 0; i < VE; i++) top = max(top, max(__float_as_uint(y0[i]) & 0x7fffffffu, __float_as_uint(y1[i]) & 0x7fffffffu));
        const uint32_t group = (gr.lh_shift == 5 ? 0xffffffffu : ((1u << (1 << gr.lh_shift)) - 1)) << (tid & 31 & ~((1 << gr.lh_shift) - 1));
        for (int d = 1; d < 1 << gr.lh_shift; d <<= 1) top = max(top, __shfl_xor_sync(group, top, d));
        const float scale = kv_scale<FMT>(top), inv = 1.0f / scale;
#pragma unroll
        for (int i = 0; i < VE; i++) y0[i] *= inv, y1[i] *= inv;
        if constexpr (VE == 8) {
          *(uint2 *)(o + d0) = make_uint2(kv_encode4<FMT>(y0[0], y0[1], y0[2], y0[3]), kv_encode4<FMT>(y0[4], y0[5], y0[6], y0[7]));
          *(uint2 *)(o + d1) = make_uint2(kv_encode4<FMT>(y1[0], y1[1], y1[2], y1[3]), kv_encode4<FMT>(y1[4], y1[5], y1[6], y1[7]));
        } else {
          *(uint32_t *)(o + d0) = kv_encode4<FMT>(y0[0], y0[1], y0[2], y0[3]);
          *(uint32_t *)(o + d1) = kv_encode4<FMT>(y1[0], y1[1], y1[2], y1[3]);
        }
        if (l == 0) (key ? a.cache.ks : a.cache.vs)[row] = scale;
      } else {                                           // of the keys' own type
        *(uint4 *)(o + d0) = pack_piece(y0);
        *(uint4 *)(o + d1) = pack_piece(y1);
      }
    }
  }
}

static bool whole_pieces(const void *p, long long ts, long long hs, size_t e) {      // and strides whose offsets in a block stay below 2^31
  const long long most = 1 << 26, heads = 1 << 18;
  if (ts > most || ts < -most || hs > heads || hs < -heads) return false;
  return ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ts * (long long)e) | (uintptr_t)(hs * (long long)e)) & 15) == 0;
}

// Few tokens: a round's heads a block (of several tokens where one has fewer heads than that and every SM has a block), so that no thread has a second round to wait
// for; many (more than 1184 rounds, eight for each SM): about six rounds a block.  One head goes as two of which the second is not there: ceil(2^32 / 1) is no 32-bit number.  us of 16384 tokens of one head of
// 64 / 128 in bf16: a token a block 22.2 / 20.8, sixteen 4.3 / 6.1; of 64 tokens of two heads: sixteen a block 2.5, one 1.8.
RopePlan rope_plan(int tokens, int heads, int step) {
  const long long rounds = ((long long)tokens * heads + step - 1) / step;
  const int slots = max(2, heads);
  if (rounds > 1184) return {max(1, min(ROPE_MAX_TOKENS, 6 * step / slots)), slots};
  const int h = min(slots, step);
  return {min(min(ROPE_MAX_TOKENS, step / h), (tokens + 147) / 148), h};
}

template <typename T, int FMT> static cudaError_t rope_append(const RopeAppend &a, cudaStream_t s) {
  constexpr int VE = 16 / sizeof(T);
  const int G = a.k.p ? a.cache.G : 0, all = a.H + 2 * G, lh = a.hd / (2 * VE);
  const bool pieces = a.hd % (2 * VE) == 0 && (lh & (lh - 1)) == 0 && lh <= 32 && (a.rope.interleaved ? 2 * a.rope.half : a.rope.half) % VE == 0 &&
                      (!a.H || (whole_pieces(a.q.p, a.q.ts, a.q.hs, sizeof(T)) && whole_pieces(a.q_out, a.qo_ts, a.qo_hs, sizeof(T)))) &&
                      (!G || (whole_pieces(a.k.p, a.k.ts, a.k.hs, sizeof(T)) && whole_pieces(a.v.p, a.v.ts, a.v.hs, sizeof(T))));
  if (!pieces || all > 4096) return launch_k(rope_append_any_kernel<T, FMT>, dim3(a.tokens), dim3(ROPE_THREADS), 0, s, a);
  RopeGrid gr;
  gr.lh_shift = __builtin_ctz(lh);
  const int step = ROPE_THREADS / lh;                    // heads of a round of the block
  constexpr int U = 1;
  const RopePlan plan = rope_plan(a.tokens, all, step);
  gr.heads = plan.heads;
  gr.per_block = plan.per_block;
  gr.by_half = a.rope.half > 1 ? (uint32_t)((0x100000000ull + a.rope.half - 1) / a.rope.half) : 0;
  gr.q_ts = (int)a.q.ts, gr.q_hs = (int)a.q.hs, gr.k_ts = (int)a.k.ts, gr.k_hs = (int)a.k.hs, gr.v_ts = (int)a.v.ts, gr.v_hs = (int)a.v.hs;
  gr.o_ts = (int)a.qo_ts, gr.o_hs = (int)a.qo_hs;
  gr.by_heads = (uint32_t)((0x100000000ull + gr.heads - 1) / gr.heads);
  const dim3 grid((a.tokens + gr.per_block - 1) / gr.per_block, (all + gr.heads - 1) / gr.heads);
  const size_t smem = (size_t)gr.per_block * 2 * a.rope.half * sizeof(float);
  if (a.rope.interleaved) return launch_k(rope_append_kernel<T, FMT, true, U>, grid, dim3(ROPE_THREADS), smem, s, a, gr);
  return launch_k(rope_append_kernel<T, FMT, false, U>, grid, dim3(ROPE_THREADS), smem, s, a, gr);
}

cudaError_t launch_rope_append(const RopeAppend &a, int dtype, int fmt, cudaStream_t s) {
  if (dtype == KV_F32) return fmt == KV_E4M3 ? rope_append<float, KV_E4M3>(a, s) : fmt == KV_INT8 ? rope_append<float, KV_INT8>(a, s) : rope_append<float, KV_F32>(a, s);
  return fmt == KV_E4M3 ? rope_append<bf16, KV_E4M3>(a, s) : fmt == KV_INT8 ? rope_append<bf16, KV_INT8>(a, s) : rope_append<bf16, KV_BF16>(a, s);
}

// ---------------------------------------------------------------- reading back
// Row r of the output is position kvpos[r] of sequence seq[r], zeros where there is none.  A thread takes eight elements, so that a
// warp's stores of bf16 are whole lines; a block some rows, whose places in the pool are looked up once.  Bytes bound it: 16384 tokens
// of 8 heads of 128 from e4m3 21 us (4.8 TB/s), 8000 of 40 heads from int8 52 us (4.8 TB/s).  Two, four and eight items a thread under way, with as many
// blocks an SM as that leaves room for: 21 / 23 / 24 us.
constexpr int READ_MAX_ROWS = 64;      // 256 / the least items a row (4)
struct ReadGrid { int rows, items; uint32_t by_items, by_hd8; };         // rows of a block, eights of a row (keys, then values); ceil(2^32 / items), / a head's eights

template <int FMT, typename T>
__global__ void __launch_bounds__(256, 8) kv_read_kernel(KvRead a, ReadGrid gr) {
  pdl_wait();
  pdl_trigger();
  typedef typename KvElem<FMT>::type E;
  const int hd8 = a.cache.hd / 8, r0 = blockIdx.x * gr.rows, nr = min(gr.rows, a.rows - r0);
  __shared__ int at[READ_MAX_ROWS];
  if (threadIdx.x < nr) at[threadIdx.x] = kv_row(a.cache, a.seq[r0 + threadIdx.x], a.kvpos[r0 + threadIdx.x], a.status, r0 + threadIdx.x);
  __syncthreads();
  const int half = gr.items / 2, n = nr * gr.items;
  T *const k_out = (T *)a.k_out + (size_t)r0 * half * 8, *const v_out = (T *)a.v_out + (size_t)r0 * half * 8;
  typedef typename Four<FMT>::raw Raw;
  struct alignas(sizeof(E) == 4 ? 16 : 8 * sizeof(E)) Eight { Raw e[2]; };
  constexpr int U = 2;                                   // in flight
  for (int i0 = threadIdx.x; i0 < n; i0 += U * 256) {
    Eight x[U];
    float sc[U];
    T *to[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int i = i0 + u * 256;
      const int r = (int)__umulhi((uint32_t)i, gr.by_items), e = i - r * gr.items, kv = e >= half, w = e - kv * half;
      const int h = (int)__umulhi((uint32_t)w, gr.by_hd8), d = (w - h * hd8) * 8;
      to[u] = nullptr;
      if (i >= n) continue;
      to[u] = (kv ? v_out : k_out) + (uint32_t)(r * half + w) * 8;
      const size_t row = (uint32_t)(at[r] + h * a.cache.page_size);
      x[u] = Eight{};
      sc[u] = 0.0f;
      if (at[r] < 0) continue;
      x[u] = *(const Eight *)((const E *)(kv ? a.cache.v : a.cache.k) + row * a.cache.hd + d);
      if constexpr (kv_is_8bit(FMT)) sc[u] = (kv ? a.cache.vs : a.cache.ks)[row];
    }
#pragma unroll
    for (int u = 0; u < U; u++) {
      if (!to[u]) continue;
      float4 lo = kv_decode_four<FMT>(x[u].e[0]), hi = kv_decode_four<FMT>(x[u].e[1]);
      if constexpr (kv_is_8bit(FMT)) {
        lo.x *= sc[u], lo.y *= sc[u], lo.z *= sc[u], lo.w *= sc[u];
        hi.x *= sc[u], hi.y *= sc[u], hi.z *= sc[u], hi.w *= sc[u];
      }
      if constexpr (sizeof(T) == 4) {
        ((float4 *)to[u])[0] = lo;
        ((float4 *)to[u])[1] = hi;
      } else {
        *(uint4 *)to[u] = make_uint4(pack_bf16(lo.x, lo.y), pack_bf16(lo.z, lo.w), pack_bf16(hi.x, hi.y), pack_bf16(hi.z, hi.w));
      }
    }
  }
}

template <int FMT> static cudaError_t kv_read(const KvRead &a, int out_dtype, cudaStream_t s) {
  ReadGrid gr;
  gr.items = 2 * a.cache.G * (a.cache.hd / 8);
  // one wave of blocks (eight an SM) where there is enough to do, and about 4096 items each where there is more: a block's look-ups come before
  // everything else it does
  gr.rows = max(max(1, 256 / gr.items), min(min(READ_MAX_ROWS, (a.rows + 1183) / 1184), max(1, 4096 / gr.items)));
  gr.by_items = (uint32_t)((0x100000000ull + gr.items - 1) / gr.items);
  gr.by_hd8 = (uint32_t)((0x100000000ull + a.cache.hd / 8 - 1) / (a.cache.hd / 8));
  const dim3 grid((a.rows + gr.rows - 1) / gr.rows);
  if (out_dtype == KV_F32) return launch_k(kv_read_kernel<FMT, float>, grid, dim3(256), 0, s, a, gr);
  return launch_k(kv_read_kernel<FMT, bf16>, grid, dim3(256), 0, s, a, gr);
}

cudaError_t launch_kv_read(const KvRead &a, int fmt, int out_dtype, cudaStream_t s) {
  return fmt == KV_F32 ? kv_read<KV_F32>(a, out_dtype, s) : fmt == KV_BF16 ? kv_read<KV_BF16>(a, out_dtype, s)
       : fmt == KV_E4M3 ? kv_read<KV_E4M3>(a, out_dtype, s) : kv_read<KV_INT8>(a, out_dtype, s);
}

}  // namespace spec
