// Single-token attention on plain FMAs: fp32 caches, and head sizes that the tensor-core body is not made for.  16 sequences of 4096 positions,
// 8 KV heads of 128 for 32 query heads in fp32: 114 us, 4.7 TB/s (231 with a lane a position's keys, whose loads touch 32 lines each, and loads
// that stand behind conditions).
#include "attn_decode_kernel.cuh"

namespace spec {

// Eight lanes share a position's keys; then LPT lanes share a position's values, NV vectors of four dimensions each.
template <int FMT_, int HP_, int DCLASS> struct FmaBody {
  static constexpr int FMT = FMT_, HP = HP_, TILE = 32, WARPS = da_fma_warps(DCLASS, HP);
  static constexpr bool HALVES = false;
  static constexpr int LPT = DCLASS == 64 ? 16 : 32, NV = DCLASS == 256 ? 2 : 1, PER = 32 / LPT;
  typedef typename KvElem<FMT>::type E;
  static constexpr int VEC = 16 / sizeof(E), STEPS = DCLASS / VEC / 8 > 0 ? DCLASS / VEC / 8 : 1;      // rounds of eight 16-byte pieces over a row
  static __host__ __device__ int warp_smem_floats(int hd) { return HP * hd + 64; }

  float m[HP], l[HP], acc[HP][NV][4];
  float *qs;                    // [HP][hd], times scale * log2 e

  __device__ __forceinline__ void run(const DaArgs &p, const DaSeg &sg, int len, float *mem, int lane) {
    init(p, sg, mem, lane);
    walk(p, sg, len, lane);
  }

  __device__ __forceinline__ void init(const DaArgs &p, const DaSeg &sg, float *mem, int lane) {
    qs = mem;
    const int hd = p.a.cache.hd;
    __syncwarp();
    for (int i = lane; i < HP * hd; i += 32) {
      const int h = i / hd;
      const size_t at = (size_t)sg.b * p.a.q_ts + (size_t)(sg.head + h) * hd + (i - h * hd);
      qs[i] = h < sg.have ? (p.q_f32 ? ((const float *)p.a.q)[at] : to_f32(((const bf16 *)p.a.q)[at])) * (p.a.scale * 1.44269504088896341f) : 0.0f;
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
    const typename Four<FMT>::raw *r = (const typename Four<FMT>::raw *)&u;
#pragma unroll
    for (int i = 0; i < VEC / 4; i++) {
      const float4 f = kv_decode_four<FMT>(r[i]);
      x[4 * i] = f.x, x[4 * i + 1] = f.y, x[4 * i + 2] = f.z, x[4 * i + 3] = f.w;
    }
  }

  __device__ __forceinline__ void walk(const DaArgs &p, const DaSeg &sg, int len, int lane) {
    const KvCache &c = p.a.cache;
    const int hd = c.hd, g = sg.kv;
    const E *K = (const E *)c.k, *V = (const E *)c.v;
    const int sub = lane & 7, mine = 4 * sub + (lane >> 3);              // this lane's position of a tile
    const int pieces = hd / VEC;
    for (int t = sg.t0; t < sg.t1; t++) {
      const int pos = t * TILE + mine;
      const int row = pos < len ? da_row(p, sg.b, g, pos) : -1;
      float s[HP];
      // four positions at a time, 128 bytes of each by eight lanes: whole lines, where a lane a position asked for 32 at once
#pragma unroll 4
      for (int i = 0; i < 8; i++) {
        const int r = __shfl_sync(0xffffffffu, row, (lane & 24) | i);
        float d[HP];
#pragma unroll
        for (int h = 0; h < HP; h++) d[h] = 0.0f;
        // loads without a condition, so that they are all under way at once: what a position that does not count brings is not used
        const uint4 *const kr = (const uint4 *)(K + (size_t)max(r, 0) * hd);
        uint4 raw[STEPS];
#pragma unroll
        for (int j = 0; j < STEPS; j++) raw[j] = __ldg(kr + min(sub + 8 * j, pieces - 1));
#pragma unroll
        for (int j = 0; j < STEPS; j++) {
          const int at = sub + 8 * j;
          if (at >= pieces) continue;
          float x[VEC];
          unpack(raw[j], x);
#pragma unroll
          for (int h = 0; h < HP; h++)
#pragma unroll
            for (int e = 0; e < VEC; e += 4) {
              const float4 w = *(const float4 *)(qs + h * hd + at * VEC + e);
              d[h] = fmaf(w.x, x[e], fmaf(w.y, x[e + 1], fmaf(w.z, x[e + 2], fmaf(w.w, x[e + 3], d[h]))));
            }
        }
#pragma unroll
        for (int h = 0; h < HP; h++) {
          d[h] += __shfl_xor_sync(0xffffffffu, d[h], 1);
          d[h] += __shfl_xor_sync(0xffffffffu, d[h], 2);
          d[h] += __shfl_xor_sync(0xffffffffu, d[h], 4);
          if (sub == i) s[h] = d[h];
        }
      }
      float vsc = 1.0f;
      if constexpr (kv_is_8bit(FMT))
        if (row >= 0) {
          const float ksc = c.ks[row];
          vsc = c.vs[row];
#pragma unroll
          for (int h = 0; h < HP; h++) s[h] *= ksc;
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
#pragma unroll 1
      for (int j0 = 0; j0 < 32; j0 += 8 * PER) {         // eight of a lane's vectors under way
        typename Four<FMT>::raw raw[8][NV];
        int r[8];
#pragma unroll
        for (int u = 0; u < 8; u++) {
          r[u] = __shfl_sync(0xffffffffu, row, j0 + (PER == 1 ? u : 2 * u + lane / LPT));
          const E *vr = V + (size_t)max(r[u], 0) * hd;
#pragma unroll
          for (int i = 0; i < NV; i++) raw[u][i] = __ldg((const typename Four<FMT>::raw *)(vr + min(dim + i * 128, hd - 4)));
        }
#pragma unroll
        for (int u = 0; u < 8; u++)
#pragma unroll
          for (int h = 0; h < HP; h++) {
            const float w = __shfl_sync(0xffffffffu, s[h], j0 + (PER == 1 ? u : 2 * u + lane / LPT));
            if (r[u] < 0) continue;
#pragma unroll
            for (int i = 0; i < NV; i++) {
              const float4 x = kv_decode_four<FMT>(raw[u][i]);
              acc[h][i][0] = fmaf(w, x.x, acc[h][i][0]), acc[h][i][1] = fmaf(w, x.y, acc[h][i][1]);
              acc[h][i][2] = fmaf(w, x.z, acc[h][i][2]), acc[h][i][3] = fmaf(w, x.w, acc[h][i][3]);
            }
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

  // f(head, dimension, four values of O) by the lanes that hold them; stat(head, max, sum) by one lane
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

template <int FMT, int HP> static cudaError_t fma_by_hd(const DaArgs &p, int ctas, cudaStream_t s) {
  const int hd = p.a.cache.hd;
  if (hd <= 64) return launch<FmaBody<FMT, HP, 64>>(p, ctas, s);
  if (hd <= 128) return launch<FmaBody<FMT, HP, 128>>(p, ctas, s);
  return launch<FmaBody<FMT, HP, 256>>(p, ctas, s);
}
template <int FMT> static cudaError_t fma_by_heads(const DaArgs &p, int ctas, cudaStream_t s) {
  if (p.deal.heads <= 1) return fma_by_hd<FMT, 1>(p, ctas, s);
  if (p.deal.heads <= 2) return fma_by_hd<FMT, 2>(p, ctas, s);
  if (p.deal.heads <= 4) return fma_by_hd<FMT, 4>(p, ctas, s);
  return fma_by_hd<FMT, 8>(p, ctas, s);
}

cudaError_t launch_decode_fma(const DaArgs &p, int fmt, int ctas, cudaStream_t s) {
  switch (fmt) {
    case KV_F32: return fma_by_heads<KV_F32>(p, ctas, s);
    case KV_BF16: return fma_by_heads<KV_BF16>(p, ctas, s);
    case KV_E4M3: return fma_by_heads<KV_E4M3>(p, ctas, s);
    default: return fma_by_heads<KV_INT8>(p, ctas, s);
  }
}

}  // namespace spec
