// Internal declarations of the decoder block's operators (cts_block.h): the
// cache, the attention over it, norms and rotary positions.
#pragma once

#include "cts.h"
#include "cts_internal.h"

namespace cts {

constexpr int kMxBlock = 32;      // elements that share a scale

// The cache's arrays, and where a token's bytes lie in them.
struct KvCache {
  uint8_t *kc, *ks, *vc, *vs;
  int n_pages, page_shift, heads, d;
  __host__ __device__ int64_t slots() const { return static_cast<int64_t>(n_pages) << page_shift; }
};

hipError_t launch_kv_write(const KvCache& c, int T, const void* k, int64_t ldk, const void* v, int64_t ldv,
                           const int64_t* slots, int dtype, hipStream_t s);
hipError_t launch_kv_read(const KvCache& c, int T, const int64_t* slots, void* k, int64_t ldk, void* v, int64_t ldv,
                          int dtype, hipStream_t s);

struct AttnParams {
  KvCache c;
  const void* q; int64_t ldq;
  void* out; int64_t ldo;
  const int32_t *table, *kv_len, *q_start;
  int T, B, heads, group;           // group: query heads of a key/value head
  int max_pages, max_q, max_kv, window, dtype;
  float scale_log2e;
  // the plan: 16-row tiles of a sequence, tokens of a piece, pieces
  int subs, chunk, pieces;
  int part_rows;                    // rows of a tile that partials are kept for
  float* part;                      // [B][subs][kv heads][pieces][part_rows][d], then [..][part_rows][2]
};

// Chooses subs, chunk, pieces and part_rows, and gives the workspace's bytes
// (not falling with any size).
size_t plan_attention(AttnParams* p);
hipError_t launch_attention(const AttnParams& p, hipStream_t s);

struct NormParams {
  int T, d;
  const void *x, *y, *post, *gate, *weight;
  void *h, *n;
  int64_t ldx, ldy, ldg, ldh, ldn;
  float scale, eps;
};
constexpr int kNormMaxD = 32768;
hipError_t launch_block_norm(const NormParams& p, int dtype, hipStream_t s);

constexpr int kRotaryMaxAxes = 4;
struct RotaryParams {
  int T, heads[2], d, rot, n_pos, axes, interleaved;
  const void* in[2]; int64_t ldi[2];
  void* out[2]; int64_t ldo[2];
  const float *cos, *sin;
  const int32_t* pos;
  int end[kRotaryMaxAxes];          // pairs of the axes up to this one
};
hipError_t launch_rotary(const RotaryParams& p, int dtype, hipStream_t s);

}  // namespace cts
