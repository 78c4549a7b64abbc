// Embedding lookup, out[t] = scale w[ids[t]], and its gradient, dw[v] = scale * sum of grad[t] over the t with ids[t] = v, summed in 32 bits in an
// order that depends on the ids alone.
#include "embedding.cuh"

#include <algorithm>

#include "vec.cuh"

namespace spec {

using std::max;
using std::min;

// ---------------------------------------------------------------- lookup
// any width, stride and alignment: a block per token and 1024 columns
__global__ void __launch_bounds__(256) embed_any_kernel(Embed a, int w_dtype, int out_dtype) {
  pdl_wait();
  pdl_trigger();
  const int t = blockIdx.x, id = id_at(a.ids, t);
  const bool there = id >= 0 && id < a.vocab;
  if (!there && id != -1 && threadIdx.x == 0) set_status(a.status, ST_BOUNDS, 64, t, id);
  for (int c = blockIdx.y * 1024 + threadIdx.x; c < min(a.dim, (int)(blockIdx.y + 1) * 1024); c += 256)
    store_from_f32(a.out, out_dtype, (long long)t * a.o_rs + c, there ? load_as_f32(a.w, w_dtype, (long long)id * a.w_rs + c) * a.scale : 0.0f);
}

// Widths of whole eights, aligned to 16 bytes: a thread has up to four units of eight under way.  A block has 1024 units of a token, or as many tokens as make 1024.
// Bytes bound it: 16384 tokens of 8192 in bf16 66 us, 8.1 TB/s as counted: rows that several tokens ask for come from L2.  512 units 70 us, 2048 78.
constexpr int LOOK_UNITS = 1024;
struct EmbedGrid {
  int units, tokens;     // of a token; of a block
  uint32_t by_units;     // ceil(2^32 / units), where a block has several tokens
};
template <typename TW, typename TO>
__global__ void __launch_bounds__(256) embed_kernel(const __grid_constant__ Embed a, const __grid_constant__ EmbedGrid gr) {
  pdl_wait();
  pdl_trigger();
  constexpr int U = LOOK_UNITS / 256;
  const int t0 = blockIdx.x * gr.tokens, u0 = blockIdx.y * LOOK_UNITS, n = gr.tokens == 1 ? min(LOOK_UNITS + 0, gr.units - u0) : min(gr.tokens, a.tokens - t0) * gr.units;
  int token[U], unit[U], id[U];
#pragma unroll
  for (int k = 0; k < U; k++) {
    const int i = threadIdx.x + k * 256;
    token[k] = -1;
    if (i >= n) continue;
    const int q = gr.tokens == 1 ? 0 : (int)__umulhi((uint32_t)i, gr.by_units);
    token[k] = t0 + q, unit[k] = u0 + i - q * gr.units;
    id[k] = id_at(a.ids, token[k]);
    if (id[k] >= 0 && id[k] < a.vocab) continue;
    if (id[k] != -1 && unit[k] == 0) set_status(a.status, ST_BOUNDS, 64, token[k], id[k]);
    id[k] = -1;
  }
  Raw8<TW> x[U];
#pragma unroll
  for (int k = 0; k < U; k++)
    if (token[k] >= 0 && id[k] >= 0) x[k].take((const TW *)a.w + (long long)id[k] * a.w_rs + unit[k] * 8);
#pragma unroll
  for (int k = 0; k < U; k++) {
    if (token[k] < 0) continue;
    float y[8] = {};
    if (id[k] >= 0) {
      x[k].floats(y);
#pragma unroll
      for (int c = 0; c < 8; c++) y[c] *= a.scale;
    }
    store8((TO *)a.out + (long long)token[k] * a.o_rs + unit[k] * 8, y);
  }
}

static size_t bytes_of(int dtype) { return dtype == 0 ? 4 : 2; }

cudaError_t launch_embed_rows(const Embed &a, int w_dtype, int out_dtype, cudaStream_t s) {
  if (a.dim % 8 || a.dim < 16 || !pieces_aligned(a.w, a.vocab > 1 ? a.w_rs : 0, bytes_of(w_dtype)) || !pieces_aligned(a.out, a.tokens > 1 ? a.o_rs : 0, bytes_of(out_dtype)))
    return launch_k(embed_any_kernel, dim3(a.tokens, (a.dim + 1023) / 1024), dim3(256), 0, s, a, w_dtype, out_dtype);
  EmbedGrid gr;
  gr.units = a.dim / 8;
  gr.tokens = max(1, min(LOOK_UNITS / gr.units, a.tokens / 296));      // every SM has two blocks before one has two tokens
  gr.by_units = (uint32_t)((0x100000000ull + gr.units - 1) / gr.units);
  const dim3 grid((a.tokens + gr.tokens - 1) / gr.tokens, gr.tokens == 1 ? (gr.units + LOOK_UNITS - 1) / LOOK_UNITS : 1);
  if (w_dtype == 0) return out_dtype == 0 ? launch_k(embed_kernel<float, float>, grid, dim3(256), 0, s, a, gr) : launch_k(embed_kernel<float, bf16>, grid, dim3(256), 0, s, a, gr);
  return out_dtype == 0 ? launch_k(embed_kernel<bf16, float>, grid, dim3(256), 0, s, a, gr) : launch_k(embed_kernel<bf16, bf16>, grid, dim3(256), 0, s, a, gr);
}

// ---------------------------------------------------------------- gradient: the tokens in the order of their ids
// A block owns a range of the vocabulary.  It reads all ids, which are few and stay in L2: how many lie below its range is where its tokens begin in the sorted
// order, so blocks need nothing from one another and one launch sorts.  Warps walk segments of the ids: counting first, then writing those of the range
// one behind another, in the tokens' order, to `list`; one warp deals them to their rows' places, 32 at a time (16384 tokens of one id: some 13 us).
constexpr int SORT_THREADS = 512, SORT_WARPS = SORT_THREADS / 32, SORT_MAX_ROWS = 4096, SORT_NEAR = 1024;

struct EmbedSort {
  int rows;              // of the vocabulary a block
  int32_t *order, *id;   // tokens by id, and the ids
  int2 *list;            // (token, row of the block's range) of the ranges, unsorted
  int32_t *count;        // tokens with a row
  uint32_t *present;     // a bit for each row of the vocabulary that a token has; null: rows without are zeroed here
};

__global__ void __launch_bounds__(SORT_THREADS) embed_sort_kernel(EmbedGrad a, EmbedSort so, int out_dtype) {
  pdl_wait();
  pdl_trigger();
  __shared__ int have[SORT_MAX_ROWS], place[SORT_MAX_ROWS], below[SORT_WARPS], mine[SORT_WARPS], upto[SORT_WARPS];
  __shared__ int2 near_by[SORT_NEAR];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, lo = blockIdx.x * so.rows, n_rows = min(so.rows, a.vocab - lo);
  for (int i = threadIdx.x; i < n_rows; i += SORT_THREADS) have[i] = 0;
  __syncthreads();
  // a warp's segment, in steps of 32 ids
  const long long steps = (a.tokens + 31LL) / 32, per = (steps + SORT_WARPS - 1) / SORT_WARPS, s0 = min((long long)warp * per, steps), s1 = min(s0 + per, steps);
  int less = 0, in = 0;
  constexpr int U = 8;                                   // steps under way
  for (long long s = s0; s < s1; s += U) {
    int id[U];
#pragma unroll
    for (int k = 0; k < U; k++) {
      const long long t = (s + k) * 32 + lane;
      id[k] = s + k < s1 && t < a.tokens ? id_at(a.ids, t) : -1;
    }
#pragma unroll
    for (int k = 0; k < U; k++) {
      if (id[k] < 0 || id[k] >= a.vocab) {
        if (id[k] != -1 && blockIdx.x == 0) set_status(a.status, ST_BOUNDS, 64, (int)((s + k) * 32 + lane), id[k]);
        continue;
      }
      less += id[k] < lo;
      if (id[k] >= lo && id[k] - lo < n_rows) in++, atomicAdd(&have[id[k] - lo], 1);
    }
  }
  less = __reduce_add_sync(0xffffffffu, less);
  in = __reduce_add_sync(0xffffffffu, in);
  if (lane == 0) below[warp] = less, mine[warp] = in;
  __syncthreads();
  int base = 0, before_me = 0, total = 0;
  for (int w = 0; w < SORT_WARPS; w++) {
    base += below[w];
    if (w < warp) before_me += mine[w];
    total += mine[w];
  }
  if (threadIdx.x == 0 && lo + n_rows == a.vocab) *so.count = base + total;
  if (total) {
    int2 *const list = total <= SORT_NEAR ? near_by : so.list + base;      // long ones in memory
    if (in) {
      int at = before_me;
      for (long long s = s0; s < s1; s += U) {
        int id[U];
#pragma unroll
        for (int k = 0; k < U; k++) {
          const long long t = (s + k) * 32 + lane;
          id[k] = s + k < s1 && t < a.tokens ? id_at(a.ids, t) : -1;
        }
#pragma unroll
        for (int k = 0; k < U; k++) {
          const bool hit = id[k] >= lo && id[k] - lo < n_rows;
          const uint32_t hits = __ballot_sync(0xffffffffu, hit);
          if (hit) list[at + __popc(hits & ((1u << lane) - 1))] = make_int2((int)((s + k) * 32 + lane), id[k] - lo);
          at += __popc(hits);
        }
      }
    }
    // where each row's tokens begin
    constexpr int EACH = SORT_MAX_ROWS / SORT_THREADS;
    const int each = (n_rows + SORT_THREADS - 1) / SORT_THREADS, r0 = threadIdx.x * each;
    int first[EACH], sum = 0;
#pragma unroll
    for (int k = 0; k < EACH; k++) {
      first[k] = sum;
      if (k < each && r0 + k < n_rows) sum += have[r0 + k];
    }
    int run = sum;
    for (int d = 1; d < 32; d <<= 1) {
      const int o = __shfl_up_sync(0xffffffffu, run, d);
      if (lane >= d) run += o;
    }
    if (lane == 31) upto[warp] = run;
    __syncthreads();
    run += base - sum;
    for (int w = 0; w < warp; w++) run += upto[w];
#pragma unroll
    for (int k = 0; k < EACH; k++)
      if (k < each && r0 + k < n_rows) place[r0 + k] = run + first[k];
    __syncthreads();
    if (warp == 0)
      for (int i = 0; i < total; i += 32) {
        const bool there = i + lane < total;
        const int2 e = there ? list[i + lane] : make_int2(0, -1);
        const uint32_t same = __match_any_sync(0xffffffffu, e.y);
        const int rank = __popc(same & ((1u << lane) - 1));
        int at = there ? place[e.y] : 0;
        __syncwarp();
        if (there && rank == 0) place[e.y] = at + __popc(same);
        __syncwarp();
        if (there) so.order[at + rank] = e.x, so.id[at + rank] = lo + e.y;
      }
  }
  if (so.present) {                                      // a block's range is whole words
    for (int i = threadIdx.x; i < (n_rows + 31) / 32 * 32; i += SORT_THREADS) {
      const uint32_t bits = __ballot_sync(0xffffffffu, i < n_rows && have[i]);
      if (lane == 0) so.present[(lo + i) / 32] = bits;
    }
  } else if (!a.accumulate) {
    for (int r = warp; r < n_rows; r += SORT_WARPS) {
      if (have[r]) continue;
      for (int c = lane; c < a.dim; c += 32) store_from_f32(a.out, out_dtype, (lo + r) * a.o_rs + c, 0.0f);
    }
  }
}

// ---------------------------------------------------------------- gradient: sums of runs of equal ids
// The sorted tokens are cut into chunks, whatever ids they have: no id, however frequent, makes a block longer than another.  A run inside a chunk is written where
// it belongs; what a chunk has of a run that goes over its ends goes to `part` (slot 0: of a run that began before, 1: of one that begins here and goes on),
// and the chunk in which a run begins adds those up, in order, in the next launch.  Blocks behind the chunks' write the zeros of rows without tokens, which are most of the bytes:
// 8192 tokens of 128256 x 4096 bf16 176 us (1111 MB, 6.3 TB/s, 96 % of a copy's rate); by the sorting blocks before them 199.  Chunks of 16 tokens 2 us more, of 64 4 more.
// Few tokens go by 16s: 2003 of 4096 x 256 fp32 16.4 us (three launches one behind the other), by 32s 18.5.
struct EmbedRuns {
  int per_chunk, chunks;
  const int32_t *order, *id, *count;
  float *part;           // [chunks][2][dim]
  const uint32_t *present;
  int zeroing;           // blocks that write zeros to rows without tokens, behind the others
};
constexpr int CHUNK_MAX = 64;

__device__ __forceinline__ void embed_grad_out(const EmbedGrad &a, int out_dtype, int id, int c, float sum) {
  const long long at = id * a.o_rs + c;
  store_from_f32(a.out, out_dtype, at, a.accumulate ? fmaf(sum, a.scale, load_as_f32(a.out, out_dtype, at)) : sum * a.scale);
}

template <typename TO> __device__ __forceinline__ void embed_grad_out8(const EmbedGrad &a, int id, int c, const float (&sum)[8]) {
  TO *const at = (TO *)a.out + id * a.o_rs + c;
  float y[8] = {};
  if (a.accumulate) load8(at, y);
#pragma unroll
  for (int e = 0; e < 8; e++) y[e] = a.accumulate ? fmaf(sum[e], a.scale, y[e]) : sum[e] * a.scale;
  store8(at, y);
}

__global__ void __launch_bounds__(128) embed_runs_any_kernel(EmbedGrad a, EmbedRuns r, int g_dtype, int out_dtype) {
  pdl_wait();
  pdl_trigger();
  __shared__ int token[CHUNK_MAX], id[CHUNK_MAX + 2];
  const int n = *r.count, p0 = blockIdx.x * r.per_chunk, m = min(r.per_chunk, n - p0);
  if (m <= 0) return;
  for (int i = threadIdx.x; i < m; i += 128) token[i] = r.order[p0 + i];
  for (int i = threadIdx.x; i < m + 2; i += 128) id[i] = p0 + i - 1 >= 0 && p0 + i - 1 < n ? r.id[p0 + i - 1] : -1;
  __syncthreads();
  const int c = blockIdx.y * 128 + threadIdx.x;
  if (c >= a.dim) return;
  float sum = 0.0f;
  bool began = id[0] != id[1];                           // whether the run under way began in this chunk
  for (int i = 0; i < m; i++) {
    sum += load_as_f32(a.grad, g_dtype, token[i] * a.g_rs + c);
    const int me = id[i + 1];
    if (i + 1 < m && id[i + 2] == me) continue;
    const bool ends = id[i + 2] != me;
    if (began && ends) embed_grad_out(a, out_dtype, me, c, sum);
    else r.part[(2LL * blockIdx.x + began) * a.dim + c] = sum;
    sum = 0.0f;
    began = true;
  }
}

// Widths of whole eights, aligned to 16 bytes: eight columns a thread, eight tokens of them under way
template <typename TG, typename TO>
__global__ void __launch_bounds__(128) embed_runs_kernel(const __grid_constant__ EmbedGrad a, const __grid_constant__ EmbedRuns r) {
  pdl_wait();
  pdl_trigger();
  const int slabs = (a.dim + 1023) / 1024, chunk = blockIdx.x / slabs;
  if (chunk >= r.chunks) {
    const int words = a.dim * (int)sizeof(TO) / 16;
    for (int v = blockIdx.x - slabs * r.chunks; v < a.vocab; v += r.zeroing) {
      if (r.present[v >> 5] >> (v & 31) & 1) continue;
      uint4 *const p = (uint4 *)((TO *)a.out + v * a.o_rs);
      for (int i = threadIdx.x; i < words; i += 128) p[i] = make_uint4(0, 0, 0, 0);
    }
    return;
  }
  __shared__ int token[CHUNK_MAX], id[CHUNK_MAX + 2];
  const int n = *r.count, p0 = chunk * r.per_chunk, m = min(r.per_chunk, n - p0);
  if (m <= 0) return;
  for (int i = threadIdx.x; i < m; i += 128) token[i] = r.order[p0 + i];
  for (int i = threadIdx.x; i < m + 2; i += 128) id[i] = p0 + i - 1 >= 0 && p0 + i - 1 < n ? r.id[p0 + i - 1] : -1;
  __syncthreads();
  const int c = ((blockIdx.x - chunk * slabs) * 128 + threadIdx.x) * 8;
  if (c >= a.dim) return;
  constexpr int U = 8;
  float sum[8] = {};
  bool began = id[0] != id[1];
  for (int i0 = 0; i0 < m; i0 += U) {
    Raw8<TG> x[U];
#pragma unroll
    for (int k = 0; k < U; k++)
      if (i0 + k < m) x[k].take((const TG *)a.grad + token[i0 + k] * a.g_rs + c);
#pragma unroll
    for (int k = 0; k < U; k++) {
      const int i = i0 + k;
      if (i >= m) continue;
      float y[8];
      x[k].floats(y);
#pragma unroll
      for (int e = 0; e < 8; e++) sum[e] += y[e];
      const int me = id[i + 1];
      const bool ends = id[i + 2] != me;
      if (i + 1 < m && !ends) continue;
      if (began && ends) embed_grad_out8<TO>(a, me, c, sum);
      else store8(r.part + (2LL * chunk + began) * a.dim + c, sum);
#pragma unroll
      for (int e = 0; e < 8; e++) sum[e] = 0.0f;
      began = true;
    }
  }
}

template <typename TO>
__global__ void __launch_bounds__(128) embed_join_eights_kernel(const __grid_constant__ EmbedGrad a, const __grid_constant__ EmbedRuns r) {
  pdl_wait();
  pdl_trigger();
  const int n = *r.count, k = blockIdx.x, p1 = (k + 1) * r.per_chunk;
  if (p1 >= n) return;
  const int me = r.id[p1 - 1];
  if (r.id[p1] != me || (k > 0 && r.id[k * r.per_chunk] == me && r.id[k * r.per_chunk - 1] == me)) return;
  int last = k + 1;                                      // the run's last chunk: ids are sorted
  for (bool more = true; more;) {
    const int j = last + 1 + (threadIdx.x & 31);
    const uint32_t on = __ballot_sync(0xffffffffu, j < r.chunks && (long long)j * r.per_chunk < n && r.id[j * r.per_chunk] == me);
    more = on == 0xffffffffu;
    last += more ? 32 : __ffs(~on) - 1;
  }
  const int c = (blockIdx.y * 128 + threadIdx.x) * 8;
  if (c >= a.dim) return;
  float sum[8];
  load8(r.part + (2LL * k + 1) * a.dim + c, sum);
#pragma unroll 8
  for (int j = k + 1; j <= last; j++) {
    float y[8];
    load8(r.part + 2LL * j * a.dim + c, y);
#pragma unroll
    for (int e = 0; e < 8; e++) sum[e] += y[e];
  }
  embed_grad_out8<TO>(a, me, c, sum);
}

__global__ void __launch_bounds__(128) embed_join_kernel(EmbedGrad a, EmbedRuns r, int out_dtype) {
  pdl_wait();
  pdl_trigger();
  const int n = *r.count, k = blockIdx.x, p1 = (k + 1) * r.per_chunk;
  if (p1 >= n) return;
  const int me = r.id[p1 - 1];
  if (r.id[p1] != me || (k > 0 && r.id[k * r.per_chunk] == me && r.id[k * r.per_chunk - 1] == me)) return;      // no run goes on here, or it began before
  const int c = blockIdx.y * 128 + threadIdx.x;
  if (c >= a.dim) return;
  float sum = r.part[(2LL * k + 1) * a.dim + c];
  for (int j = k + 1; j < r.chunks && j * r.per_chunk < n && r.id[j * r.per_chunk] == me; j++) sum += r.part[2LL * j * a.dim + c];
  embed_grad_out(a, out_dtype, me, c, sum);
}

static size_t up(size_t n) { return (n + 255) / 256 * 256; }
static int chunk_of(int tokens) { return tokens >= 4096 ? 32 : 16; }

size_t embed_grad_scratch_bytes(int tokens, int vocab, int dim) {
  const size_t T = tokens, chunks = (T + chunk_of(tokens) - 1) / chunk_of(tokens);
  return up(4 * T) * 2 + up(8 * T) + 256 + up(((size_t)vocab + 31) / 32 * 4) + chunks * 2 * dim * 4;
}

cudaError_t launch_embed_grad(const EmbedGrad &a, int g_dtype, int out_dtype, cudaStream_t s) {
  const bool eights = a.tokens && a.dim % 8 == 0 && pieces_aligned(a.out, a.vocab > 1 ? a.o_rs : 0, bytes_of(out_dtype)) && pieces_aligned(a.grad, a.tokens > 1 ? a.g_rs : 0, bytes_of(g_dtype));
  char *p = (char *)a.scratch;
  EmbedSort so;
  so.count = (int32_t *)p, p += 256;
  so.order = (int32_t *)p, p += up(4 * (size_t)a.tokens);
  so.id = (int32_t *)p, p += up(4 * (size_t)a.tokens);
  so.list = (int2 *)p, p += up(8 * (size_t)a.tokens);
  so.present = eights && !a.accumulate ? (uint32_t *)p : nullptr, p += up(((size_t)a.vocab + 31) / 32 * 4);
  so.rows = min(SORT_MAX_ROWS, (a.vocab / 296 + 32) / 32 * 32);      // two blocks an SM
  if (const cudaError_t e = launch_k(embed_sort_kernel, dim3((a.vocab + so.rows - 1) / so.rows), dim3(SORT_THREADS), 0, s, a, so, out_dtype)) return e;
  if (a.tokens == 0) return cudaSuccess;
  EmbedRuns r;
  r.per_chunk = chunk_of(a.tokens);
  r.chunks = (int)(((long long)a.tokens + r.per_chunk - 1) / r.per_chunk);
  r.order = so.order, r.id = so.id, r.count = so.count, r.part = (float *)p, r.present = so.present;
  // about 48 KB of zeros a block, and blocks for every SM: 128256 x 4096 bf16 for 8192 tokens 176 us so, 198 with 2368 blocks that stay, 184 with one for each of two rows
  r.zeroing = so.present ? (int)min<long long>(a.vocab, max(592LL, (long long)a.vocab * a.dim * (long long)bytes_of(out_dtype) / (48 << 10))) : 0;
  const dim3 grid(r.chunks, (a.dim + 127) / 128);
  if (!eights) {
    if (const cudaError_t e = launch_k(embed_runs_any_kernel, grid, dim3(128), 0, s, a, r, g_dtype, out_dtype)) return e;
    return launch_k(embed_join_kernel, grid, dim3(128), 0, s, a, r, out_dtype);
  }
  const int slabs = (a.dim + 1023) / 1024;
  if ((long long)r.chunks * slabs + r.zeroing > INT32_MAX) return cudaErrorNotSupported;
  const dim3 runs(r.chunks * slabs + r.zeroing), join(r.chunks, slabs);
  const cudaError_t e = g_dtype == 0 ? (out_dtype == 0 ? launch_k(embed_runs_kernel<float, float>, runs, dim3(128), 0, s, a, r) : launch_k(embed_runs_kernel<float, bf16>, runs, dim3(128), 0, s, a, r))
                                     : (out_dtype == 0 ? launch_k(embed_runs_kernel<bf16, float>, runs, dim3(128), 0, s, a, r) : launch_k(embed_runs_kernel<bf16, bf16>, runs, dim3(128), 0, s, a, r));
  if (e) return e;
  return out_dtype == 0 ? launch_k(embed_join_eights_kernel<float>, join, dim3(128), 0, s, a, r) : launch_k(embed_join_eights_kernel<bf16>, join, dim3(128), 0, s, a, r);
}

}  // namespace spec
