// Device helpers of the attention kernels (attention.hip, attention_tile.hip, attention_tree.hip).
#pragma once

#include "block_internal.h"

namespace cts {
namespace {

constexpr int kRowTile = 16;       // query rows of a tile
constexpr int kUnit = 32;          // tokens of a step
constexpr int kSmallRows = 64;     // rows of a sequence that the 16-row tiles are for
constexpr int kWaves = 8;          // waves of a workgroup that share a tile's steps
constexpr int kRuns = 512;         // runs of steps, at most: two workgroups for every compute unit
constexpr int kFewTiles = 64;      // tiles (x heads) up to which each tile is cut into runs of its own
constexpr int kJoinThreads = 256;
constexpr int kPromptRows = 128;   // query rows of a workgroup for prompts
constexpr int64_t kPromptGroups = 512;  // workgroups that few prompts are split into: two for every compute unit
constexpr int64_t kPromptSteps = 8;     // steps of 8192 / d tokens of a piece, at least
// The sums follow the running maximum only once it has grown by 2^8: until then
// weights are up to 2^8 instead of 1, which costs no precision in floats (nor in
// bf16), and the sums are seldom rescaled.  The weight that a row's maximum came
// from stays 1, so its length is 0 only where it has seen nothing.
constexpr float kSlack = 8.0f;

__device__ __forceinline__ uint32_t fp4_pair(uint32_t w, float unit, int byte) {
  switch (byte) {
    case 0: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 0));
    case 1: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 1));
    case 2: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 2));
    default: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 3));
  }
}

// v as computed here and not before: in a branch that is seldom taken, what is
// computed from it stays there (the compiler otherwise works both sides out every
// time and selects; masks alone are a third of a step's vector instructions).
__device__ __forceinline__ int rare(int v) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("" : "+v"(v));
#endif
  return v;
}
// Whether byte i of w is past the scales that are written (at most 252): 255, a NaN
// block, or 253 and 254, which put some magnitudes past the largest float.
__device__ __forceinline__ bool past_scales(uint32_t w, int i) { return ((w >> (8 * i)) & 0xffu) > 252u; }
// the float 2^(s - 127) of byte i of w (255: as the conversion's NaN scale)
__device__ __forceinline__ float unit_of(uint32_t w, int i) {
  return __uint_as_float((i < 3 ? w << (23 - 8 * i) : w >> 1) & 0x7f800000u);
}

__device__ __forceinline__ float max_over_groups(float v) {       // over the lanes of the same n
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum_over_groups(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ bf16x8 frag(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  typedef uint32_t u32x4_ __attribute__((ext_vector_type(4)));
  const u32x4_ v = {a, b, c, d};
  return __builtin_bit_cast(bf16x8, v);
}

// l + both halves of a pair of bf16 weights.  A row's length is the sum of its weights as
// they are multiplied: where one token has most of the weight, the weight's rounding
// then cancels.
__device__ __forceinline__ float add_pair(uint32_t w, float l) {
  typedef short short2_ __attribute__((ext_vector_type(2)));
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(short2_, w), __builtin_bit_cast(short2_, 0x3f803f80u), l, false);
}

// Inclusive sum over the wave's lanes.
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);      // from 1, 2, 4, 8 lanes below in a row of 16
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);      // the last lane of rows 0 and 2 to the next row
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);      // lane 31 to the upper half
  return v;
}

// eight floats as NS bf16 parts whose sum is the float (to 8, 16 or 24 bits)
template <int NS> __device__ __forceinline__ void split(const float* f, bf16x8* out) {
  float r[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = f[i];
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = f32_to_bf16_pair(r[2 * i], r[2 * i + 1]);
      r[2 * i] -= __uint_as_float(w[i] << 16);
      r[2 * i + 1] -= __uint_as_float(w[i] & 0xffff0000u);
    }
    out[s] = frag(w[0], w[1], w[2], w[3]);
  }
}

struct Tile {                      // what a 16-row tile of a sequence covers
  int b, q0, rows, row0;           // the sequence, its first query row, its rows (query x head of the group), the tile's first
  int first_pos;                   // position of the sequence's first query
  int lo, hi;                      // tokens that some row of the tile sees, [lo, hi); lo a multiple of a step
  int steps;                       // steps of kUnit tokens (one where nothing is seen); 0: no such rows
};

// Whether whole tiles take the sequences by their lengths: with up to two workgroups for every
// compute unit, where lengths can differ enough for their order to matter.
__host__ __device__ inline bool by_length(const AttnParams& p) {
  const int tiles = p.B * p.subs * p.c.heads;
  return tiles > 256 && tiles <= 512 && p.B <= 128 && p.max_kv >= 1024;
}

struct Queries { int q0, n; };     // a sequence's query rows
__device__ __forceinline__ Queries queries_of(const AttnParams& p, int b) {
  if (!p.q_start) return {b, 1};
  const int q0 = min(max(p.q_start[b], 0), p.T);
  return {q0, min(max(p.q_start[b + 1], q0), p.T) - q0};
}

__device__ __forceinline__ Tile tile_of(const AttnParams& p, int b, int sub) {
  Tile t;
  const Queries q = queries_of(p, b);
  const int len = min(max(p.kv_len[b], 0), p.max_kv);
  t.b = b;
  t.q0 = q.q0;
  t.rows = min(q.n, p.max_q) * p.group;
  t.row0 = sub * kRowTile;
  t.first_pos = len - q.n;
  const int j0 = t.row0 / p.group, j1 = (min(t.rows, t.row0 + kRowTile) - 1) / p.group;
  t.hi = max(0, t.first_pos + j1 + 1);
  t.lo = p.window ? max(0, t.first_pos + j0 - p.window + 1) & ~(kUnit - 1) : 0;
  t.steps = t.row0 < t.rows ? max(1, (t.hi - t.lo + kUnit - 1) / kUnit) : 0;
  return t;
}

// The tiles of the sequences with few rows: tile `index` is sub-tile index %
// subs of sequence index / subs (steps 0 for the others).
__device__ __forceinline__ Tile small_tile(const AttnParams& p, int index) {
  const int b = p.subs == 1 ? index : index / p.subs;
  Tile t = tile_of(p, b, index - b * p.subs);
  if (t.rows > kSmallRows) t.steps = 0;
  return t;
}

__device__ __forceinline__ Tile uniform(Tile t) {      // what every lane holds alike, in scalar registers
  return {__builtin_amdgcn_readfirstlane(t.b),  __builtin_amdgcn_readfirstlane(t.q0),
          __builtin_amdgcn_readfirstlane(t.rows), __builtin_amdgcn_readfirstlane(t.row0),
          __builtin_amdgcn_readfirstlane(t.first_pos), __builtin_amdgcn_readfirstlane(t.lo),
          __builtin_amdgcn_readfirstlane(t.hi), __builtin_amdgcn_readfirstlane(t.steps)};
}

// N (4 or 8) elements
template <int N> __device__ __forceinline__ void store_out(float* o, const float* f) {
#pragma unroll
  for (int i = 0; i < N; i += 4) *reinterpret_cast<float4*>(o + i) = make_float4(f[i], f[i + 1], f[i + 2], f[i + 3]);
}
template <int N> __device__ __forceinline__ void store_out(bf16_t* o, const float* f) {
  const uint32_t a = f32_to_bf16_pair(f[0], f[1]), b = f32_to_bf16_pair(f[2], f[3]);
  if constexpr (N == 8)
    *reinterpret_cast<uint4*>(o) = make_uint4(a, b, f32_to_bf16_pair(f[4], f[5]), f32_to_bf16_pair(f[6], f[7]));
  else
    *reinterpret_cast<uint2*>(o) = make_uint2(a, b);
}

template <typename TQ> __device__ __forceinline__ void load_q(const TQ* q, float* f);
template <> __device__ __forceinline__ void load_q<float>(const float* q, float* f) {
  const float4 a = reinterpret_cast<const float4*>(q)[0], b = reinterpret_cast<const float4*>(q)[1];
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
  f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
template <> __device__ __forceinline__ void load_q<bf16_t>(const bf16_t* q, float* f) {
  const uint4 v = *reinterpret_cast<const uint4*>(q);
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}

}  // namespace
}  // namespace cts
