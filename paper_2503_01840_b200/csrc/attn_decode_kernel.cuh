// Attention of one new token per sequence over the paged cache:
//   out = sum_t p_t v_t / sum_t p_t,  p_t = exp(scale q.k_t - max),  lse = max + log sum_t p_t,   t < length of the sequence.
//
// Every key and value is read once for up to 16 of the query heads that share it (a chunk; eight with few sequences, large heads or plain FMAs), so the cache's bytes bound it.  They are dealt out
// evenly: all tiles of TILE positions, of every sequence and KV head (a segment) one after the other, are cut into equal runs for the CTAs
// (one wave of them), a CTA's run into equal runs for its warps.  A warp walks its run with a softmax state of its own; what is left
// of a (sequence, head) that several warps share is joined in shared memory, and of one that several CTAs share by the CTA that
// finishes last, out of the workspace, in the order of the positions whoever that is: the result does not depend on timing.
#pragma once
#include "attn_decode.cuh"

namespace spec {

// Work is counted in tiles, and the beginning of a segment (queries, page, first keys: nothing is under way meanwhile) as so many more.  us with 0 / 1 / 2 / 3:
// one sequence of 16384 18.6 / 17.5 / 17.4 / 17.7, 8 of 700 to 1500 14.0 / 12.6 / 12.7 / 13.3, 4 of 1000 to 8000 17.6 / 16.3 / 16.2 / 16.1, 64 of 256 to 2048
// 42.1 / 41.8 / 41.4 / 40.9.
constexpr int DA_START = 2;
// Bodies of 16 columns take a KV head's heads by halves where there are fewer units than this a CTA, as the lengths on the device say: the join of 16 heads' states by 8 warps then costs more than
// the second walk.  us whole / by halves, heads of 128 in e4m3, sequences x KV heads, tables of 65536 positions: 40 x 1 with 16 query heads of 100 to 400 (3 units) 19.5 / 10.8, of 1000 to 2000 (13)
// 23.7 / 20.6, 60 x 1 (20) 25.2 / 22.6, 16 x 2 of 4096 (28) 27.2 / 26.2, 64 x 2 of 256 to 2048 (33) 30.7 / 35.1; bf16, 15 x 2 of 500 to 1500 (13) 21.6 / 17.2, 16 x 2 of 4096 (56) 29.5 / 33.0.
constexpr int DA_HALVE_BELOW = 24;
constexpr int DA_MAX_CTAS = 160;           // CTAs of a launch, at most
constexpr int DA_PART_FLOATS = 8 * 256 + 16 * 2;      // a partial state: O of heads x hd <= 2048 elements, then (max, sum) of up to 16 heads

// How the heads of a KV head go together
struct DaDeal {
  int heads, chunks;            // query heads a warp takes together, and how many such chunks share a KV head
  int vheads, segs;             // KV heads x chunks; segments of the call
  int whole;                    // segments that a CTA gets at most where they stay whole (0: they do not)
};

// workspace: partial states of each CTA's first and last segment, and a counter per CTA for the segment that starts in it
struct DaArgs {
  DecodeAttn a;
  int page_shift;               // log2 of the page size, or -1
  int q_f32;                    // queries and output in fp32
  int group;                    // query heads per KV head
  int spare;                    // tiles that a CTA may have beyond its share where segments stay whole
  DaDeal deal;
  DaDeal halves;                // bodies of 16 columns: where there are fewer units than halve_below (a KV head's heads as one chunk)
  int halve_below;
  unsigned *count;              // [CTAs], zero between calls
  float *part;                  // [CTAs][2][part_floats], close together: another page of memory costs a walk of the page tables
};

__host__ __device__ constexpr int da_part_floats(int heads, int hd) { return heads * hd + (2 * heads + 3) / 4 * 4; }

// A run of tiles of one (sequence, chunk of heads)
struct DaSeg {
  int b, kv;                    // sequence, KV head
  int head, have;               // its chunk's first query head, and how many there are
  int t0, t1, tiles;            // tiles t0 .. t1 - 1 of `tiles`
  int u0;                       // the first of them, in units over all segments
};

// States of one segment that are joined: `mask` of those that stand `stride` floats apart from `from`, the first `skew` further on; into `to`, or
// where that is null into rows `row` .. of the output
struct DaRun {
  const float *from;
  float *to;
  int row, heads, stride, skew;
  uint32_t mask;
};

__device__ __forceinline__ float da_exp2(float x) { return exp2f(x); }
__device__ __forceinline__ float da_ref(float m) { return m == -INFINITY ? 0.0f : m; }      // keeps inf - inf out of a row whose scores are all -inf

__device__ __forceinline__ float da_inverse(float l) { return l == 0.0f ? 0.0f : 1.0f / l; }      // a row whose scores are all -inf gives 0

// x / d for small quotients (below 2^20) of non-negative numbers, in a third of the instructions of the exact division
__device__ __forceinline__ int da_quotient(int x, int d) {
  const int q = (int)__fdividef((float)x, (float)d), r = x - q * d;
  return q + (r >= d) - (r < 0);
}

__device__ __forceinline__ float warp_max(float x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
  return x;
}
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

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
// a sequence's length; one below zero or past the cache is reported and clamped
__device__ __forceinline__ int da_length(const DaArgs &p, int b) {
  const int len = p.a.len[b];
  const long long cap = (long long)p.a.cache.pages_per_seq * p.a.cache.page_size;
  if (len < 0 || len > cap) {
    set_status(p.a.status, ST_BOUNDS, 62, b, len);
    return len < 0 ? 0 : (int)cap;
  }
  return len;
}

__device__ __forceinline__ void da_store(void *out, bool f32, size_t at, float4 o) {
  if (f32) *(float4 *)((float *)out + at) = o;
  else *(uint2 *)((bf16 *)out + at) = make_uint2(pack_bf16(o.x, o.y), pack_bf16(o.z, o.w));
}

// A warp joins one head of the states (O [heads][hd], then, `stats` floats on, (max, sum) [heads]) whose bits are set in `run`, `stride` floats apart,
// the first `skew` further on: into its rows of the output and of lse, or as a state into `to`.  One piece of code for all joins, kept short: a
// call runs it once or twice, and fetching cold instructions takes longer than what they do.
// (Its arguments are values: fields of the kernel's parameters behind a pointer would be loads, from the L2 after the fence.)
static __device__ __noinline__ void da_join_head(const float *states, int stride, int skew, uint32_t run, int stats, int h, int hd, float *to, void *out, bool f32, float *lse) {
  const int lane = threadIdx.x & 31;
  const int first = __ffs(run) - 1;
  constexpr int U = 8;                                   // states in flight; the first ones are asked for together with the sums
  float4 y[U];
  auto ask = [&](uint32_t left, int d) {
#pragma unroll
    for (int u = 0; u < U; u++) {
      y[u] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (!left) continue;
      const int k = __ffs(left) - 1;
      left &= left - 1;
      if (d < hd) y[u] = *(const float4 *)(states + (size_t)k * stride + (k == first ? skew : 0) + h * hd + d);
    }
  };
  const bool in = (run >> lane) & 1;
  const float2 x = in ? *(const float2 *)(states + (size_t)lane * stride + (lane == first ? skew : 0) + stats + 2 * h) : make_float2(-INFINITY, 0.0f);
  ask(run, lane * 4);
  const float m = warp_max(x.x), f = in ? da_exp2(x.x - da_ref(m)) : 0.0f, l = warp_sum(x.y * f), inv = da_inverse(l);
  for (int d = lane * 4; d - lane * 4 < hd; d += 128) {
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (uint32_t left = run; left;) {
      if (left != run || d >= 128) ask(left, d);
#pragma unroll
      for (int u = 0; u < U; u++) {
        if (!left) continue;
        const float w = __shfl_sync(0xffffffffu, f, __ffs(left) - 1);
        left &= left - 1;
        o.x = fmaf(y[u].x, w, o.x), o.y = fmaf(y[u].y, w, o.y), o.z = fmaf(y[u].z, w, o.z), o.w = fmaf(y[u].w, w, o.w);
      }
    }
    if (d >= hd) continue;
    if (to) *(float4 *)(to + h * hd + d) = o;
    else da_store(out, f32, d, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
  }
  if (lane != 0) return;
  if (to) *(float2 *)(to + stats + 2 * h) = make_float2(m, l);
  else if (lse) *lse = (da_ref(m) + log2f(l)) * 0.693147180559945309f;
}

// smem: int before[batch + 1] (units before each sequence), per warp the body's floats and two partial states
template <typename Body>
__global__ void __launch_bounds__(Body::WARPS * 32, 1) decode_attn_kernel(const __grid_constant__ DaArgs p) {
  pdl_wait();
  pdl_trigger();
  constexpr int W = Body::WARPS, THREADS = W * 32, TILE = Body::TILE;
  extern __shared__ __align__(16) char smem[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, B = p.a.batch, hd = p.a.cache.hd, cta = blockIdx.x;
  int *before = (int *)smem;
  float *mem = (float *)(smem + ((size_t)(B + 1) * 4 + 15) / 16 * 16);
  float *warp_mem = mem + warp * Body::warp_smem_floats(hd);
  float *const states = mem + W * Body::warp_smem_floats(hd);            // [2 W][part_floats]
  __shared__ int2 scan[W];
  __shared__ DaSeg seg[2 * W];                                           // of the partial states; b = -1: none
  __shared__ DaRun runs[2 * W];
  __shared__ int to_do[3];

  // ---- units (tiles and beginnings) before each sequence, their sum, and the longest sequence's.  Up to 32 sequences: a lane each in every warp, and no barrier
  // on the way to the first load; more: a run of them per thread, a scan over the threads, and a table.
  const bool few = B <= 32;
  auto units_of = [&](int len) { return len ? (len - 1) / TILE + 1 + DA_START : 0; };      // (len + TILE - 1 may be none of an int)
  int total, longest = 0, my_before = 0, my_tiles = 0;
  if (few) {
    my_tiles = lane < B ? units_of(da_length(p, lane)) : 0;
    int inc = my_tiles;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += x;
    }
    my_before = inc - my_tiles;
    total = __shfl_sync(0xffffffffu, inc, 31);
    longest = __reduce_max_sync(0xffffffffu, my_tiles);
  } else {
    const int per = (B + THREADS - 1) / THREADS, b0 = min(B, tid * per), b1 = min(B, b0 + per);
    int sum = 0, most = 0;
    for (int b = b0; b < b1; b++) {
      const int t = units_of(da_length(p, b));
      sum += t;
      most = max(most, t);
    }
    int inc = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += x;
    }
    most = __reduce_max_sync(0xffffffffu, most);
    if (lane == 31) scan[warp] = make_int2(inc, most);
    __syncthreads();
    int at = inc - sum;
    for (int w = 0; w < W; w++) {
      if (w < warp) at += scan[w].x;
      longest = max(longest, scan[w].y);
    }
    for (int b = b0; b < b1; b++) {
      before[b] = at;
      at += units_of(da_length(p, b));
    }
    if (tid == THREADS - 1) before[B] = at;
    __syncthreads();
    total = before[B];
  }
  bool halved = false;
  if constexpr (Body::HALVES) halved = total * p.a.cache.G < p.halve_below;
  const DaDeal &deal = halved ? p.halves : p.deal;
  const int heads = deal.heads, chunks = deal.chunks, VH = deal.vheads, part_floats = da_part_floats(heads, hd);      // a state: O [heads][hd], then (max, sum) [heads]
  total *= VH;
  if (lane < 2) seg[2 * warp + lane].b = -1;
  // (units before sequence b, those of each of its segments); all lanes ask for the same one
  auto tiles_of = [&](int b) {
    if (few) return make_int2(__shfl_sync(0xffffffffu, my_before, b), __shfl_sync(0xffffffffu, my_tiles, b));
    return make_int2(before[b], before[b + 1] - before[b]);
  };

  // The units are dealt out evenly: each of N CTAs has total / N, the first total % N one more.  (32-bit quotients: 64-bit ones take
  // microseconds here.)  At least eight tiles a CTA: states that CTAs share cost more to join than those of a CTA's warps.
  const int N = max(1, min((int)gridDim.x, (total + 7) >> 3));
  const int each = total / N, more = total - each * N;
  auto begin_of = [&](int i) { return i * each + min(i, more); };
  auto cta_of = [&](int u) { return u < more * (each + 1) ? u / (each + 1) : more + (u - more * (each + 1)) / each; };
  int c0 = cta < N ? begin_of(cta) : 0, c1 = cta < N ? begin_of(cta + 1) : 0;
  // Joining states of several CTAs takes six microseconds, in which a CTA reads `spare` tiles.  Where no CTA gets that many more than its
  // share when segments stay whole, they do.
  if (deal.whole && ((long long)deal.whole * longest - p.spare) * (int)gridDim.x <= total) {
    auto start_of = [&](int j) {
      const int b = da_quotient(j, VH);
      if (b >= B) return total;
      const int2 t = tiles_of(b);
      return t.x * VH + (j - b * VH) * t.y;
    };
    c0 = start_of((int)((unsigned)deal.segs * (unsigned)cta / gridDim.x));
    c1 = start_of((int)((unsigned)deal.segs * (unsigned)(cta + 1) / gridDim.x));
  }
  const int w0 = c0 + (int)((unsigned)(c1 - c0) * (unsigned)warp / W), w1 = c0 + (int)((unsigned)(c1 - c0) * (unsigned)(warp + 1) / W);

  // ---- sequences without a position
  for (int b = cta; b < B; b += gridDim.x)
    if (tiles_of(b).y == 0) {
      for (int i = tid * 4; i < p.a.H * hd; i += THREADS * 4) da_store(p.a.out, p.q_f32, (size_t)b * p.a.H * hd + i, make_float4(0.f, 0.f, 0.f, 0.f));
      if (p.a.lse)
        for (int h = tid; h < p.a.H; h += THREADS) p.a.lse[(size_t)b * p.a.H + h] = -INFINITY;
    }

  // ---- this warp's tiles
  int slot = 0;
  for (int u = w0; u < w1;) {
    DaSeg s;
    if (few) {                                                           // the last sequence with before * VH <= u: it has tiles
      s.b = __popc(__ballot_sync(0xffffffffu, lane < B && my_before * VH <= u)) - 1;
    } else {
      int lo = 0, hi = B;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (before[mid] * VH <= u) lo = mid;
        else hi = mid;
      }
      s.b = lo;
    }
    const int2 t = tiles_of(s.b);
    const int r = u - t.x * VH, v = da_quotient(r, t.y), x = r - v * t.y, end = min(t.y, x + (w1 - u));      // units x .. end - 1 of the segment's
    s.kv = chunks == 1 ? v : da_quotient(v, chunks);
    const int before_it = (v - s.kv * chunks) * heads;                   // query heads of the chunks before this one
    s.head = s.kv * p.group + before_it;
    s.have = min(heads, p.group - before_it);
    s.tiles = t.y - DA_START;
    s.t0 = max(x - DA_START, 0);
    s.t1 = end - DA_START;
    s.u0 = u - x + DA_START;
    u += end - x;
    if (s.t1 <= s.t0) continue;                                          // nothing but its beginning
    Body body;
    body.run(p, s, da_length(p, s.b), warp_mem, lane);
    const bool whole = s.t0 == 0 && s.t1 == s.tiles;
    float *st = states + (size_t)(2 * warp + (whole ? 1 : slot)) * part_floats;
    __syncwarp();
    body.each(hd, lane, [&](int h, int d, float4 o) {
      if (h < heads) *(float4 *)(st + h * hd + d) = o;
    }, [&](int h, float m, float l) {
      if (h < heads) *(float2 *)(st + heads * hd + 2 * h) = make_float2(m, l);
    });
    if (whole) {                                                         // the slot is free again until the run's last segment
      __syncwarp();
      const size_t row = (size_t)s.b * p.a.H + s.head;
      for (int h = 0; h < s.have; h++)
        da_join_head(st, part_floats, 0, 1u, heads * hd, h, hd, nullptr, (char *)p.a.out + (row + h) * hd * (p.q_f32 ? 4 : 2), p.q_f32, p.a.lse ? p.a.lse + row + h : nullptr);
    } else {
      if (lane == 0) seg[2 * warp + slot] = s;
      slot++;                                                            // only a run's first and last segment can be parts
    }
  }
  __syncthreads();

  // ---- joins: of the states that this CTA's warps share (level 0); of those that CTAs share, 32 at a time, by the CTA that comes last (1);
  // of what that leaves where a segment has more (2).  All levels run the same code, a warp a run and head by turns: code that only the
  // last CTA ran took it microseconds to fetch.  (Eight or sixteen at a time, and level 2 for the rest: 21.4 us against 18.4 for one sequence of 16384.)
  static_assert(2 * W <= 32, "a lane per partial state");
  constexpr int SHIFT = 5;                                               // states of a part
  static_assert(DA_MAX_CTAS / (1 << SHIFT) + 2 <= 2 * W, "room for the parts of level 1");
  auto make_run = [&](int at, const DaSeg &s, const float *from, int stride, int skew, uint32_t mask, float *to) {
    runs[at] = DaRun{from, to, s.b * p.a.H + s.head, s.have, stride, skew, mask};
  };
  int n_runs = 0, n_open = 0;
  DaSeg open_seg{};                                                      // lanes 0 and 1 of warp 0: what other CTAs have the rest of
  if (warp == 0) {
    // lane i looks at partial state i; a run of one segment's states begins where the one before it is another's
    const DaSeg mine = lane < 2 * W ? seg[lane] : DaSeg{-1, 0, 0, 0, 0, 0, 0, 0};
    const uint32_t some = __ballot_sync(0xffffffffu, mine.b >= 0), below = (1u << lane) - 1;
    const int prev = (some & below) ? 31 - __clz(some & below) : lane;
    const int pu = __shfl_sync(0xffffffffu, mine.u0, prev);
    const bool begins = mine.b >= 0 && (prev == lane || pu != mine.u0);
    const uint32_t all = __ballot_sync(0xffffffffu, begins), after = all & ~below & ~(1u << lane);
    const uint32_t run = some & ~below & (after ? (1u << (__ffs(after) - 1)) - 1 : 0xffffffffu);
    const int t1 = __shfl_sync(0xffffffffu, mine.t1, begins ? 31 - __clz(run) : lane);
    const bool open = begins && (mine.t0 != 0 || t1 != mine.tiles);
    if (begins)
      make_run(__popc(all & below), mine, states, part_floats, 0, run, open ? p.part + (size_t)(2 * cta + (mine.t0 == 0)) * part_floats : nullptr);
    // at most two are open: the first run, which began in an earlier CTA, and the last
    const uint32_t opens = __ballot_sync(0xffffffffu, open);
    n_open = __popc(opens);
    const int from = lane == 0 ? __ffs(opens) - 1 : 31 - __clz(opens);
    open_seg.b = __shfl_sync(0xffffffffu, mine.b, from & 31), open_seg.head = __shfl_sync(0xffffffffu, mine.head, from & 31);
    open_seg.have = __shfl_sync(0xffffffffu, mine.have, from & 31), open_seg.tiles = __shfl_sync(0xffffffffu, mine.tiles, from & 31);
    open_seg.u0 = __shfl_sync(0xffffffffu, mine.u0, from & 31);
    if (lane == 0) to_do[0] = __popc(all), to_do[1] = n_open;
  }
  __syncthreads();
  n_runs = to_do[0];
  n_open = to_do[1];
  bool mine_last = false;                                                // lanes 0 and 1 of warp 0 again
  int shared_from = 0, shared_by = 0;
#pragma unroll 1
  for (int level = 0;; level++) {
    const int per = heads <= 1 ? 0 : 32 - __clz(heads - 1);              // heads of a run: a power of two, so that no quotient is taken
#pragma unroll 1
    for (int j = warp; j < n_runs << per; j += W) {
      const DaRun r = runs[j >> per];
      const int h = j & ((1 << per) - 1);
      if (h >= r.heads) continue;
      da_join_head(r.from, r.stride, r.skew, r.mask, heads * hd, h, hd, r.to, (char *)p.a.out + (size_t)(r.row + h) * hd * (p.q_f32 ? 4 : 2), p.q_f32,
                   p.a.lse ? p.a.lse + r.row + h : nullptr);
    }
    if (n_open == 0 || level == 2) return;
    __syncthreads();                                                     // the block's states are written
    if (warp == 0) {
      int parts = 0;
      if (level == 0) {                                                  // the CTA that starts a segment keeps its count
        if (lane < n_open) {
          shared_from = cta_of(open_seg.u0);
          shared_by = cta_of(open_seg.u0 + open_seg.tiles - 1) - shared_from + 1;
          __threadfence();
          mine_last = atomicAdd(p.count + shared_from, 1u) == (unsigned)(shared_by - 1);
          if (mine_last) p.count[shared_from] = 0;                       // as the next call wants it
          __threadfence();
        }
        parts = mine_last ? (shared_by + (1 << SHIFT) - 1) >> SHIFT : 0;
      } else {
        parts = mine_last && shared_by > 1 << SHIFT ? 1 : 0;
      }
      const int other = __shfl_sync(0xffffffffu, parts, 0), first_slot = lane == 0 ? 0 : other;
      if (level == 0) {
        // a CTA's state stands where its number says, but for the first CTA, whose last segment it is
        for (int i = 0; i < parts; i++) {
          const int k0 = i << SHIFT, k = min(1 << SHIFT, shared_by - k0);
          make_run(first_slot + i, open_seg, p.part + (size_t)2 * (shared_from + k0) * part_floats, 2 * part_floats, i == 0 ? part_floats : 0, k == 32 ? 0xffffffffu : (1u << k) - 1,
                   parts == 1 ? nullptr : states + (size_t)(first_slot + i) * part_floats);
        }
      } else if (parts) {
        const int k = (shared_by + (1 << SHIFT) - 1) >> SHIFT;
        const int slots = lane == 0 ? 0 : to_do[2];
        make_run(first_slot, open_seg, states + (size_t)slots * part_floats, part_floats, 0, k == 32 ? 0xffffffffu : (1u << k) - 1, nullptr);
      }
      const int sum = __shfl_sync(0xffffffffu, parts, 0) + __shfl_sync(0xffffffffu, parts, 1);
      if (lane == 0) {
        to_do[0] = sum;
        if (level == 0) to_do[2] = parts;                                // where the second segment's states begin
      }
    }
    __syncthreads();
    n_runs = to_do[0];
    if (n_runs == 0) return;
  }
}

constexpr size_t DA_SMEM = 224 * 1024;
// What a CTA reads in the time that a join over CTAs takes.  us with none / 128 / 256 / 512 KB: 64 sequences of 10 to 100 tokens, 40 heads 32.2 / 32.3 /
// 24.8 / 24.7; 32 of 100 to 400, 8 heads 16.7 / 14.1 / 14.2 / 14.2; 8 of 700 to 1500 16.7 / 16.7 / 16.6 / 17.2.
constexpr int DA_SPARE_BYTES = 256 * 1024;
// warps of the bodies: as many as their registers leave room for
constexpr int da_mma_warps(int hd, int bytes, int columns, int groups) { return hd * bytes * groups <= 128 && columns == 8 ? 16 : 8; }
constexpr int da_fma_warps(int hd, int heads) { return heads <= 4 && hd <= 128 ? 16 : 8; }
inline size_t da_smem_bytes(int batch, int warps, int own_floats, int heads, int hd) {
  return ((size_t)(batch + 1) * 4 + 15) / 16 * 16 + sizeof(float) * warps * (own_floats + 2 * da_part_floats(heads, hd));
}
template <typename Body> static cudaError_t launch(DaArgs p, int ctas, cudaStream_t s) {
  static SmemLimit limit;
  const long long tiles = ((long long)p.a.cache.pages_per_seq * p.a.cache.page_size + Body::TILE - 1) / Body::TILE;
  const long long units = (tiles + DA_START) * p.a.batch * p.a.cache.G;
  if (units * p.deal.chunks > (1 << 30)) return cudaErrorNotSupported;
  // (with fewer segments than half the CTAs the others stay without work: one user at 613 tokens 12.3 us dealt out evenly, 13.0 whole)
  for (DaDeal *d : {&p.deal, &p.halves}) d->whole = d->segs * 2 >= ctas && d->segs < (1 << 24) ? (d->segs + ctas - 1) / ctas : 0;
  p.halve_below = Body::HALVES && units * p.halves.chunks <= (1 << 30) ? p.halve_below * ctas : 0;
  p.spare = DA_SPARE_BYTES / (Body::TILE * p.a.cache.hd * 2 * (int)sizeof(typename Body::E));
  const size_t smem = da_smem_bytes(p.a.batch, Body::WARPS, Body::warp_smem_floats(p.a.cache.hd), p.deal.heads, p.a.cache.hd);
  if (smem > DA_SMEM || !limit.ensure(decode_attn_kernel<Body>, (int)smem)) return cudaErrorInvalidValue;
  return launch_k(decode_attn_kernel<Body>, dim3(ctas), dim3(Body::WARPS * 32), smem, s, p);
}

cudaError_t launch_decode_fma(const DaArgs &p, int fmt, int ctas, cudaStream_t s);
cudaError_t launch_decode_mma(const DaArgs &p, int fmt, const DecodePlan &plan, int ctas, cudaStream_t s);

}  // namespace spec
