// Single-token attention on tensor cores: bf16 queries (over 8-bit caches fp32 ones too), head sizes 64, 128 and 256, up to MR = 8 or 16 columns
// of query heads per KV head.  For a group of 16 positions
//   S^T [16 positions][MR heads] = K Q^T,   O^T [hd][MR heads] += V^T P^T     (mma m16n8k16: the cache is the A operand, so no row of it is wasted)
// Lane (g, t) = (lane / 4, lane % 4) holds keys of positions g and g + 8 and values of positions 2t, 2t + 1, 2t + 8, 2t + 9.  Which
// dimension stands at which place of a contraction is free as long as Q agrees, so a lane's keys are whole 16-byte pieces of a row,
// likewise its values (piece g of a row): everything comes straight from global memory into the registers that the MMA reads,
// one tile ahead.  Eight bits become f16, which holds every e4m3 and int8 number; Q becomes f16 times a power of two that puts its
// largest element below 2^15, so that no element that counts loses a bit.  Scales of keys go onto the scores.  Scales of values go onto
// the probabilities: each head's products are multiplied by a power of two that puts its largest so far near 2^6 (f16 holds 2^-24 .. 2^16), and O is divided by it
// in the end.  It follows the products, not the scales: a value's scale far above the others' costs those nothing where its probability is small.
// The reference that probabilities are relative to follows the maximum only where a score passes it by more than 8 (in powers of two), and that power only where a product
// passes 2^15; over 8-bit caches both change by whole powers of two, exactly.
// Over a bf16 cache the MMA has both operands in bf16 (f16 would not hold the values), so probabilities go in two parts of eight bits, one MMA each into the same O: in one part
// they made the output's error against 64 bits 2.3e-3, where its own rounding to bf16 is 1.7e-3.  The tensor pipe has the room; us with one part /
// two: 16 sequences of 4096, 32 / 8 heads of 128 51.3 / 51.3, 16 of 4097 to 32768, 64 / 8 195.8 / 196.2, 128 / 8 60.3 / 60.8, 7 of 16384, 64 / 4 heads of 64 39.4 / 39.7.
//
// Measured: 16 sequences of 4097 to 32768 positions, 64 / 8 heads of 128, in bf16 192 us (6.3 TB/s, 98 % of a copy's rate); 16 of 8192, 32 / 8 heads, in
// bf16 91 us, in e4m3 55 (5.0 TB/s), in int8 57.  What is left there is the ten microseconds around the loop (launch, first loads, joins).
// Tried without a gain: lines of the tile after the next asked for to the L2 (e4m3 56 -> 61 us; heads of 64 28 -> 24 where larger tiles brought 23), one load of
// scales a tile and
// shuffles of them (310 -> 495 instructions a group with the division and the maximum of scales that went along with it).
#include "attn_decode_kernel.cuh"

namespace spec {

__device__ __forceinline__ float da_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
template <bool F16> __device__ __forceinline__ void da_mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (F16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t da_transpose(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint4 da_load16(const void *p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ uint2 da_load8(const void *p) {
  uint2 v;
  asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
  return v;
}
// four 8-bit numbers as two pairs of f16
template <int FMT> __device__ __forceinline__ void da_to_f16(uint32_t x, uint32_t &lo, uint32_t &hi) {
  if constexpr (FMT == KV_E4M3) {
    e4m3_to_f16(x, lo, hi);
  } else {                                               // bits 0x6400 | u are 1024 + u, u = x + 128
    x ^= 0x80808080u;
    const __half2 off = __half2half2(__ushort_as_half(0x6480));
    const uint32_t a = __byte_perm(x, 0x64646464u, 0x4140), b = __byte_perm(x, 0x64646464u, 0x4342);
    const __half2 l = __hsub2(*(const __half2 *)&a, off), h = __hsub2(*(const __half2 *)&b, off);
    lo = *(const uint32_t *)&l;
    hi = *(const uint32_t *)&h;
  }
}

template <int FMT_, int HD, int MR, bool SPLIT, int NG> struct MmaBody {
  static constexpr int FMT = FMT_, NB = MR / 8, TILE = 16 * NG;
  static constexpr bool Q8 = kv_is_8bit(FMT);
  // fp32 queries (8-bit caches): a block of eight columns is four heads' upper eleven bits and the same heads' next eleven, 2^11 times as
  // large, of the queries as of the probabilities; the products are exact, and the two sums are put together in fp32
  static_assert(!SPLIT || Q8, "a bf16 cache has bf16 queries");
  static constexpr int PER_BLOCK = SPLIT ? 4 : 8;       // heads of a block of columns
  typedef typename KvElem<FMT>::type E;
  static constexpr int EB = sizeof(E), KP = HD * EB / 64, VB = HD * EB / 8 < 16 ? HD * EB / 8 : 16, VP = HD * EB / 8 / VB, EP = VB / EB;
  static constexpr int STEPS = HD / 16;
  static constexpr uint32_t FULL = NG == 2 ? 0xffffffffu : 0xffffu;      // all positions of a tile count
  // values a tile ahead as well, where keys and values of a tile are not half a thread's registers
  static constexpr bool V_AHEAD = HD * EB < 512;
  static constexpr int WARPS = da_mma_warps(HD, EB, MR, NG);
  static constexpr bool HALVES = MR == 16;
  static __host__ __device__ int warp_smem_floats(int) { return 0; }

  static constexpr float NONE = -3.40282346638528860e38f;      // the reference before any score: the lowest number, so that none is below it
  float r[NB][2], l[NB][2], o[NB][STEPS][4];             // reference, sum and O of heads 8 n + 2 t and the next
  uint32_t q[NB][STEPS][2];
  float wide[SPLIT ? NB : 1][SPLIT ? STEPS : 1][4];      // queries as they are, until begin()
  float qf[NB][2];                                       // scale * log2 e / the power of two on Q
  float up[Q8 ? NB : 1][2];                              // the power of two on probability times scale, and so on O

  // the dimensions of Q that this lane's piece of a key meets in contraction s, four at a time; heads past the last are zero
  __device__ __forceinline__ void load_queries(const DaArgs &p, const DaSeg &sg, int g, int t) {
#pragma unroll
    for (int n = 0; n < NB; n++) {
      const int h = PER_BLOCK * n + g % PER_BLOCK;
      const bool in = h < sg.have;
      const size_t x = (size_t)sg.b * p.a.q_ts + (size_t)(sg.head + (in ? h : 0)) * HD;
#pragma unroll
      for (int s = 0; s < STEPS; s++) {
        const int d = EB == 1 ? (s / 4) * 64 + t * 16 + (s % 4) * 4 : (s / 2) * 32 + t * 8 + (s % 2) * 4;
        if constexpr (SPLIT) {
          const float4 u = in ? *(const float4 *)((const float *)p.a.q + x + d) : make_float4(0.f, 0.f, 0.f, 0.f);
          wide[n][s][0] = u.x, wide[n][s][1] = u.y, wide[n][s][2] = u.z, wide[n][s][3] = u.w;
        } else {
          const uint2 u = in ? *(const uint2 *)((const bf16 *)p.a.q + x + d) : make_uint2(0, 0);
          q[n][s][0] = u.x, q[n][s][1] = u.y;
        }
      }
    }
  }
  static __device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }
  static __device__ __forceinline__ float inverse_power(float p) { return __uint_as_float(0x7f000000u - __float_as_uint(p)); }      // 1 / p, of a power of two from 2^-126 to 2^126
  // two numbers as f16 (part 0), or what that leaves of them, times 2^11 (part 1); an infinity leaves nothing
  static __device__ __forceinline__ uint32_t part_of(float a, float b, int part) {
    const __half2 hi = __floats2half2_rn(a, b);
    if (!SPLIT || part == 0) return *(const uint32_t *)&hi;
    const float2 u = __half22float2(hi);
    const __half2 lo = __floats2half2_rn(fabsf(u.x) < INFINITY ? (a - u.x) * 2048.0f : 0.0f, fabsf(u.y) < INFINITY ? (b - u.y) * 2048.0f : 0.0f);
    return *(const uint32_t *)&lo;
  }
  __device__ __forceinline__ void begin(const DaArgs &p, int g, int t) {
#pragma unroll
    for (int n = 0; n < NB; n++) {
      float f = p.a.scale * 1.44269504088896341f;
      if constexpr (Q8) {
        float top = 0.0f;
        auto pair = [&](int s, int i) {
          if constexpr (SPLIT) return make_float2(wide[n][s][2 * i], wide[n][s][2 * i + 1]);
          else return __bfloat1622float2(*(const __nv_bfloat162 *)&q[n][s][i]);
        };
#pragma unroll
        for (int s = 0; s < STEPS; s++)
#pragma unroll
          for (int i = 0; i < 2; i++) {
            const float2 v = pair(s, i);
            top = fmaxf(top, fmaxf(fabsf(v.x), fabsf(v.y)));
          }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // 2^(14 - exponent), kept where it and its reciprocal are normal numbers; a head with an infinity is taken as it is
        int e = (int)(__float_as_uint(top) >> 23) - 127;
        e = e > 127 ? 14 : max(e, -100);
        const float up = __uint_as_float((uint32_t)(14 - e + 127) << 23);
        f *= __uint_as_float((uint32_t)(e - 14 + 127) << 23);
#pragma unroll
        for (int s = 0; s < STEPS; s++)
#pragma unroll
          for (int i = 0; i < 2; i++) {
            const float2 v = pair(s, i);
            q[n][s][i] = SPLIT ? part_of(v.x * up, v.y * up, g >> 2) : part_of(v.x * up, v.y * up, 0);
          }
      }
#pragma unroll
      for (int e = 0; e < 2; e++) {
        qf[n][e] = __shfl_sync(0xffffffffu, f, ((2 * t + e) % PER_BLOCK) * 4);
        r[n][e] = NONE, l[n][e] = 0.0f;
        if constexpr (Q8) up[n][e] = 8.507059173023462e37f;       // 2^126
      }
#pragma unroll
      for (int s = 0; s < STEPS; s++)
#pragma unroll
        for (int e = 0; e < 4; e++) o[n][s][e] = 0.0f;
    }
  }

  struct Keys { uint4 x[2][KP]; float ks[2], vs[2]; };   // keys and both scales of positions g and g + 8
  struct Values { uint32_t x[4][VP * VB / 4]; };
  // `row`: of this lane's position of a tile; `at`: 0 or 16, where the group begins
  static __device__ __forceinline__ void load_keys(const KvCache &cc, int row, int at, int g, int t, Keys &k) {
#pragma unroll
    for (int i = 0; i < 2; i++) {
      const uint32_t r = __shfl_sync(0xffffffffu, row, at + g + 8 * i);
      const char *from = (const char *)cc.k + (size_t)r * (HD * EB) + t * 16;
#pragma unroll
      for (int j = 0; j < KP; j++) k.x[i][j] = da_load16(from + j * 64);
      if constexpr (Q8) k.ks[i] = __ldg(cc.ks + r), k.vs[i] = __ldg(cc.vs + r);
    }
  }
  static __device__ __forceinline__ void load_values(const KvCache &cc, int row, int at, int g, int t, Values &v) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const char *from = (const char *)cc.v + (size_t)(uint32_t)__shfl_sync(0xffffffffu, row, at + 2 * t + (i & 1) + 4 * (i & 2)) * (HD * EB) + g * VB;
#pragma unroll
      for (int j = 0; j < VP; j++)
        if constexpr (VB == 16) {
          const uint4 u = da_load16(from + j * 128);
          v.x[i][4 * j] = u.x, v.x[i][4 * j + 1] = u.y, v.x[i][4 * j + 2] = u.z, v.x[i][4 * j + 3] = u.w;
        } else {
          const uint2 u = da_load8(from);
          v.x[i][0] = u.x, v.x[i][1] = u.y;
        }
    }
  }

  __device__ __forceinline__ void run(const DaArgs &p, const DaSeg &sg, int len, float *, int lane) {
    const KvCache &cc = p.a.cache;
    const int g = lane >> 2, t = lane & 3, head = sg.kv;
    const int32_t *table = cc.table + (size_t)sg.b * cc.pages_per_seq;
    // the page of this lane's position of a tile (past the end: of the last position), then its row
    int off = 0;
    auto page_of = [&](int tile) {
      const int pos = min(tile * TILE + lane % TILE, len - 1), at = p.page_shift >= 0 ? pos >> p.page_shift : pos / cc.page_size;
      off = pos - at * cc.page_size;
      return table[at];
    };
    // row of this lane's position; valid: bit i is set where position i counts.  A page that is none of the pool's is read as page 0.
    auto row_of = [&](int tile, int page, uint32_t &valid) {
      const bool ok = (unsigned)page < (unsigned)cc.num_pages;
      if (!ok) set_status(p.a.status, ST_BOUNDS, 63, sg.b, page);
      valid = __ballot_sync(0xffffffffu, ok && tile * TILE + lane % TILE < len) & FULL;
      return ((ok ? page : 0) * cc.G + head) * cc.page_size + off;
    };
    uint32_t valid;
    int tile = sg.t0, page = page_of(tile);
    load_queries(p, sg, g, t);
    int row = row_of(tile, page, valid);
    Keys k[NG];
    Values v[NG];
#pragma unroll
    for (int u = 0; u < NG; u++) load_keys(cc, row, 16 * u, g, t, k[u]);
    if constexpr (V_AHEAD) {
#pragma unroll
      for (int u = 0; u < NG; u++) load_values(cc, row, 16 * u, g, t, v[u]);
    }
    page = page_of(min(tile + 1, sg.t1 - 1));
    begin(p, g, t);
    for (; tile < sg.t1; tile++) {
      const uint32_t live = valid;
      const int row_here = row;
      row = row_of(min(tile + 1, sg.t1 - 1), page, valid);      // the last tile is asked for once more
      page = page_of(min(tile + 2, sg.t1 - 1));
      // ---- scores
      float s[NG][NB][4], vs[NG][2], ks[NG][2];
#pragma unroll
      for (int u = 0; u < NG; u++) {
#pragma unroll
        for (int n = 0; n < NB; n++) s[u][n][0] = s[u][n][1] = s[u][n][2] = s[u][n][3] = 0.0f;
#pragma unroll
        for (int j = 0; j < KP; j++) {
          const uint4 k0 = k[u].x[0][j], k1 = k[u].x[1][j];
          const uint32_t x[4] = {k0.x, k0.y, k0.z, k0.w}, y[4] = {k1.x, k1.y, k1.z, k1.w};
          if constexpr (Q8) {
#pragma unroll
            for (int w = 0; w < 4; w++) {
              uint32_t a0, a1, a2, a3;
              da_to_f16<FMT>(x[w], a0, a2);
              da_to_f16<FMT>(y[w], a1, a3);
#pragma unroll
              for (int n = 0; n < NB; n++) da_mma<true>(s[u][n], a0, a1, a2, a3, q[n][4 * j + w][0], q[n][4 * j + w][1]);
            }
          } else {
#pragma unroll
            for (int w = 0; w < 4; w += 2)
#pragma unroll
              for (int n = 0; n < NB; n++) da_mma<false>(s[u][n], x[w], y[w], x[w + 1], y[w + 1], q[n][2 * j + w / 2][0], q[n][2 * j + w / 2][1]);
          }
        }
#pragma unroll
        for (int i = 0; i < 2; i++) vs[u][i] = Q8 ? k[u].vs[i] : 1.0f, ks[u][i] = Q8 ? k[u].ks[i] : 1.0f;
      }
#pragma unroll
      for (int u = 0; u < NG; u++) {
        if constexpr (V_AHEAD) load_keys(cc, row, 16 * u, g, t, k[u]);
        else load_values(cc, row_here, 16 * u, g, t, v[u]);
      }
      // ---- probabilities: positions g and g + 8 of a group (elements 0, 1 and 2, 3) of two heads
      if constexpr (SPLIT) {                             // the other part of the same head and position is two lanes away
#pragma unroll
        for (int u = 0; u < NG; u++)
#pragma unroll
          for (int n = 0; n < NB; n++)
#pragma unroll
            for (int e = 0; e < 4; e++) {
              const float o = __shfl_xor_sync(0xffffffffu, s[u][n][e], 2);
              s[u][n][e] = t < 2 ? fmaf(o, 4.8828125e-4f, s[u][n][e]) : fmaf(s[u][n][e], 4.8828125e-4f, o);
            }
      }
#pragma unroll
      for (int u = 0; u < NG; u++)
#pragma unroll
        for (int n = 0; n < NB; n++)
#pragma unroll
          for (int e = 0; e < 4; e++) s[u][n][e] *= Q8 ? ks[u][e >> 1] * qf[n][e & 1] : qf[n][e & 1];
      if (live != FULL) {
#pragma unroll
        for (int u = 0; u < NG; u++)
#pragma unroll
          for (int i = 0; i < 2; i++)
            if (!((live >> (16 * u + g + 8 * i)) & 1)) {
              vs[u][i] = 0.0f;                           // what stands there may be no number
#pragma unroll
              for (int n = 0; n < NB; n++) s[u][n][2 * i] = s[u][n][2 * i + 1] = -INFINITY;
            }
      }
      uint32_t b[NG][NB][2];                             // as the MMA takes them
      uint32_t rest[Q8 ? 1 : NG][Q8 ? 1 : NB][2];        // bf16: what that leaves of them
      float sum[NB][2];
      // A second pass, after a reference or a power has changed, is rare past the first tiles.  (One copy of this code: with two, heads of 256 took 65 us
      // instead of 56, 16 sequences of 4096, 8 KV heads in e4m3.)
#pragma unroll 1
      for (int pass = 0;; pass++) {
        bool over = false;
#pragma unroll
        for (int n = 0; n < NB; n++) {
          sum[n][0] = sum[n][1] = 0.0f;
#pragma unroll
          for (int u = 0; u < NG; u++)
#pragma unroll
            for (int i = 0; i < 2; i++) {
              float w[2];
#pragma unroll
              for (int e = 0; e < 2; e++) {
                w[e] = da_ex2(s[u][n][2 * i + e] - r[n][e]);
                over |= w[e] > 256.0f;
                sum[n][e] += w[e];
                if constexpr (Q8) {
                  w[e] *= vs[u][i] * up[n][e];
                  over |= w[e] > 32768.0f;
                }
              }
              if constexpr (Q8) {
                b[u][n][i] = part_of(w[0], w[1], SPLIT ? t >> 1 : 0);
              } else {
                b[u][n][i] = pack_bf16(w[0], w[1]);
                rest[u][n][i] = pack_bf16(w[0] - __uint_as_float(b[u][n][i] << 16), w[1] - __uint_as_float(b[u][n][i] & 0xffff0000u));
              }
            }
        }
        if (!__any_sync(0xffffffffu, over && pass == 0)) break;
#pragma unroll
        for (int n = 0; n < NB; n++)
#pragma unroll
          for (int e = 0; e < 2; e++) {
            float m = r[n][e];
#pragma unroll
            for (int u = 0; u < NG; u++) m = fmaxf(m, fmaxf(s[u][n][e], s[u][n][e + 2]));
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
            // 8 bits: whole powers of two, so that both changes are exact (2^-127: 0).  bf16: the maximum itself, whose probability then is 1 and loses nothing
            float f;
            if constexpr (Q8) m = ceilf(m), f = power_of_two(-(int)fminf(m - r[n][e], 127.0f));
            else f = da_ex2(r[n][e] - m);
            r[n][e] = m;
            l[n][e] *= f;
            if constexpr (Q8) {
              float top = 7.52316384526264e-37f;         // 2^-120, the least scale
#pragma unroll
              for (int u = 0; u < NG; u++) top = fmaxf(top, fmaxf(da_ex2(s[u][n][e] - m) * vs[u][0], da_ex2(s[u][n][e + 2] - m) * vs[u][1]));
#pragma unroll
              for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
              f *= inverse_power(up[n][e]);
              top = fminf(fmaxf(top, 64.0f * f), 1.329227995784916e36f);      // 2^120
              up[n][e] = power_of_two(6 + 127 - (int)(__float_as_uint(top) >> 23));
              f *= up[n][e];
            }
#pragma unroll
            for (int i = 0; i < STEPS; i++) o[n][i][e] *= f, o[n][i][e + 2] *= f;
          }
      }
#pragma unroll
      for (int n = 0; n < NB; n++) {
        l[n][0] += sum[n][0], l[n][1] += sum[n][1];
#pragma unroll
        for (int u = 0; u < NG; u++)
#pragma unroll
          for (int i = 0; i < 2; i++) {
            if constexpr (!Q8) rest[u][n][i] = da_transpose(rest[u][n][i]);
            b[u][n][i] = da_transpose(b[u][n][i]);       // [positions g][heads 2t, 2t + 1] -> [head g][positions 2t, 2t + 1]
          }
      }
      // ---- output
      if (live != FULL) {                                // a page that is none: zero times whatever stands in page 0 is to be zero
#pragma unroll
        for (int u = 0; u < NG; u++)
#pragma unroll
          for (int i = 0; i < 4; i++)
            if (!((live >> (16 * u + 2 * t + (i & 1) + 4 * (i & 2))) & 1))
#pragma unroll
              for (int j = 0; j < VP * VB / 4; j++) v[u].x[i][j] = 0;
      }
#pragma unroll
      for (int u = 0; u < NG; u++) {
#pragma unroll
        for (int j = 0; j < VP * VB / 4; j++) {
          const uint32_t v0 = v[u].x[0][j], v1 = v[u].x[1][j], v2 = v[u].x[2][j], v3 = v[u].x[3][j];
          if constexpr (Q8) {                            // four dimensions: two contractions' rows g and g + 8
            uint32_t lo[2], hi[2], lo8[2], hi8[2];       // [positions 2t, 2t + 1 | 2t + 8, 2t + 9] of dimensions 0, 1 / 2, 3
            da_to_f16<FMT>(__byte_perm(v0, v1, 0x5140), lo[0], hi[0]);
            da_to_f16<FMT>(__byte_perm(v0, v1, 0x7362), lo8[0], hi8[0]);
            da_to_f16<FMT>(__byte_perm(v2, v3, 0x5140), lo[1], hi[1]);
            da_to_f16<FMT>(__byte_perm(v2, v3, 0x7362), lo8[1], hi8[1]);
#pragma unroll
            for (int n = 0; n < NB; n++) {
              da_mma<true>(o[n][2 * j], lo[0], hi[0], lo[1], hi[1], b[u][n][0], b[u][n][1]);
              da_mma<true>(o[n][2 * j + 1], lo8[0], hi8[0], lo8[1], hi8[1], b[u][n][0], b[u][n][1]);
            }
          } else {
            const uint32_t a0 = __byte_perm(v0, v1, 0x5410), a1 = __byte_perm(v0, v1, 0x7632), a2 = __byte_perm(v2, v3, 0x5410), a3 = __byte_perm(v2, v3, 0x7632);
#pragma unroll
            for (int n = 0; n < NB; n++) {
              da_mma<false>(o[n][j], a0, a1, a2, a3, b[u][n][0], b[u][n][1]);
              da_mma<false>(o[n][j], a0, a1, a2, a3, rest[u][n][0], rest[u][n][1]);
            }
          }
        }
      }
#pragma unroll
      for (int u = 0; u < NG; u++) {
        if constexpr (V_AHEAD) load_values(cc, row, 16 * u, g, t, v[u]);
        else load_keys(cc, row, 16 * u, g, t, k[u]);
      }
    }
#pragma unroll
    for (int n = 0; n < NB; n++)
#pragma unroll
      for (int e = 0; e < 2; e++) {
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], d);
        if constexpr (Q8) {
#pragma unroll
          for (int i = 0; i < STEPS; i++) {
            if constexpr (SPLIT) {
              o[n][i][e] = fmaf(__shfl_xor_sync(0xffffffffu, o[n][i][e], 2), 4.8828125e-4f, o[n][i][e]);      // what t < 2 hold is used
              o[n][i][e + 2] = fmaf(__shfl_xor_sync(0xffffffffu, o[n][i][e + 2], 2), 4.8828125e-4f, o[n][i][e + 2]);
            }
            o[n][i][e] *= inverse_power(up[n][e]), o[n][i][e + 2] *= inverse_power(up[n][e]);
          }
        }
      }
  }

  template <typename F, typename G> __device__ __forceinline__ void each(int, int lane, F f, G stat) {
    const int g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int n = 0; n < NB; n++)
#pragma unroll
      for (int e = 0; e < 2; e++) {
        const int h = PER_BLOCK * n + 2 * t + e;
        if (SPLIT && t >= 2) continue;
#pragma unroll
        for (int j = 0; j < VP; j++)
#pragma unroll
          for (int i = 0; i < EP; i += 4) {
            const int at = (j * EP + i) / 2;
            f(h, j * 8 * EP + g * EP + i, make_float4(o[n][at][e], o[n][at][e + 2], o[n][at + 1][e], o[n][at + 1][e + 2]));
          }
        if (g == 0) stat(h, r[n][e], l[n][e]);
      }
  }
};

template <int FMT, int HD, bool SPLIT> static cudaError_t mma_by_heads(const DaArgs &p, const DecodePlan &plan, int ctas, cudaStream_t s) {
  constexpr int EB = kv_is_8bit(FMT) ? 1 : 2, NG = HD * EB <= 128 ? 2 : 1;
  if constexpr (HD < 256)
    if (plan.columns == 16) return launch<MmaBody<FMT, HD, 16, SPLIT, NG>>(p, ctas, s);
  if constexpr (HD * EB == 128 && EB == 1)
    if (plan.groups == 1) return launch<MmaBody<FMT, HD, 8, SPLIT, 1>>(p, ctas, s);
  return launch<MmaBody<FMT, HD, 8, SPLIT, NG>>(p, ctas, s);
}
template <int FMT, bool SPLIT> static cudaError_t mma_by_hd(const DaArgs &p, const DecodePlan &plan, int ctas, cudaStream_t s) {
  return p.a.cache.hd == 64 ? mma_by_heads<FMT, 64, SPLIT>(p, plan, ctas, s) : p.a.cache.hd == 128 ? mma_by_heads<FMT, 128, SPLIT>(p, plan, ctas, s)
                                                                                                  : mma_by_heads<FMT, 256, SPLIT>(p, plan, ctas, s);
}

cudaError_t launch_decode_mma(const DaArgs &p, int fmt, const DecodePlan &plan, int ctas, cudaStream_t s) {
  if (fmt == KV_BF16) return mma_by_hd<KV_BF16, false>(p, plan, ctas, s);
  if (fmt == KV_E4M3) return p.q_f32 ? mma_by_hd<KV_E4M3, true>(p, plan, ctas, s) : mma_by_hd<KV_E4M3, false>(p, plan, ctas, s);
  return p.q_f32 ? mma_by_hd<KV_INT8, true>(p, plan, ctas, s) : mma_by_hd<KV_INT8, false>(p, plan, ctas, s);
}

}  // namespace spec
