// Attention of one new token per sequence over the paged cache: host-side interface.
#pragma once
#include "kv_cache.cuh"

namespace spec {

struct DecodeAttn {
  const void *q;                // [batch][H][hd], tokens q_ts elements apart
  long long q_ts;
  KvCache cache;
  const int32_t *len;           // [batch]
  void *out;                    // [batch][H][hd]
  float *lse;                   // [batch][H] or null
  int batch, H;
  float scale;
  void *workspace;
  int32_t *status;
};
size_t decode_attn_workspace_bytes();
constexpr int DECODE_MAX_BATCH = 8192;
// cudaErrorNotSupported: more tiles of positions than an int counts
// How a call is taken apart: `heads` query heads a warp takes together, `chunks` of them a KV head; the body's columns (tensor cores, else room for as many heads),
// groups of 16 positions a tile (0: plain FMAs) and warps
struct DecodePlan { int chunks, heads, columns, groups, warps; };
// positions: that a sequence's row of the page table holds
DecodePlan decode_attn_plan(int q_f32, int fmt, int batch, int H, int G, int hd, int ctas, long long positions = 1ll << 31);
cudaError_t launch_decode_attn(const DecodeAttn &a, int dtype, int fmt, cudaStream_t s);

}  // namespace spec
