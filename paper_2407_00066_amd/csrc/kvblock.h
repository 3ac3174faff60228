// The cache's layout and its 4-bit blocks in device code (kvcache.hip, kvappend.hip).
#pragma once

#include <algorithm>

#include "block_internal.h"

namespace cts {
namespace {

constexpr int kThreads = 256;

template <typename TI> __device__ __forceinline__ void load8(const TI* p, float* f);
template <> __device__ __forceinline__ void load8<float>(const float* p, float* f) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
  f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
template <> __device__ __forceinline__ void load8<bf16_t>(const bf16_t* p, float* f) {
  const uint4 v = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}

// Where 8 elements (eighth e of a head row) of a slot lie: code and scale bytes.
// Only a page's start needs 64 bits: a page is less than 2^30 bytes.
struct At { uint64_t code, scale; };
__device__ __forceinline__ At place(const KvCache& c, int64_t slot, uint32_t head, uint32_t e, bool value) {
  const uint32_t page = static_cast<uint32_t>(slot >> c.page_shift), half = c.d >> 1, nb = c.d >> 5;
  const uint32_t o = static_cast<uint32_t>(slot) & ((1u << c.page_shift) - 1);
  const uint32_t head_codes = half << c.page_shift, head_scales = nb << c.page_shift;
  uint32_t code = head * head_codes, scale = head * head_scales;
  if (value) {
    code += (o >> 2) * (4 * half) + e * 16 + (o & 3) * 4;
    scale += (o >> 2) * (4 * nb) + (e >> 2) * 4 + (o & 3);
  } else {
    code += o * half + e * 4;
    scale += o * nb + (e >> 2);
  }
  return {static_cast<uint64_t>(page) * (c.heads * head_codes) + code,
          static_cast<uint64_t>(page) * (c.heads * head_scales) + scale};
}

// A workgroup takes `tokens` consecutive tokens; piece i of theirs is eighth
// i % ne of a token's row.
constexpr int kPieces = 2;                       // of a thread at a time (8191 tokens of 8 x 128 written: 1, 2, 4 pieces 11, 9.2, 10 us)
struct Work { Divider ne; int tokens; };

// A block's scale from `top`, the largest magnitude of each of its four threads, which go together: as an integer it
// orders like the value, NaN above all.
struct BlockScale { int s; bool finite; };
__device__ __forceinline__ BlockScale block_scale(uint32_t top) {
  top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 1)));
  top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 2)));
  const bool finite = top < 0x7f800000u;
  // a mantissa from 1.75 on would round past 6: the next power of two then
  return {finite ? min(252, max(1, static_cast<int>((top + (1u << 21)) >> 23) - 2)) : 255, finite};
}
__device__ __forceinline__ uint32_t codes8(const float* f, BlockScale b) {
  uint32_t q = 0;
  if (b.finite) {
    const float unit = __uint_as_float(static_cast<uint32_t>(b.s) << 23);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, f[0], f[1], unit, 0);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, f[2], f[3], unit, 1);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, f[4], f[5], unit, 2);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, f[6], f[7], unit, 3);
  }
  return q;
}

// Eight elements, eighth e of a head row, quantised into a slot.
__device__ __forceinline__ void store8(const KvCache& c, int64_t slot, int head, int e, bool value, const float* f) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(f[i]) & 0x7fffffffu);
  const BlockScale b = block_scale(top);
  const uint32_t q = codes8(f, b);
  const At at = place(c, slot, head, e, value);
  *reinterpret_cast<uint32_t*>((value ? c.vc : c.kc) + at.code) = q;
  if ((e & 3) == 0) (value ? c.vs : c.ks)[at.scale] = static_cast<uint8_t>(b.s);
}

// Workgroup w's keys or values of the rows from `rows` on, `ld` apart, into their slots.
template <typename TI>
__device__ __forceinline__ void write_rows(const KvCache& c, const Work& work, int T, uint32_t w, const TI* __restrict__ rows,
                                           int64_t ld, const int64_t* __restrict__ slots, bool value) {
  const int64_t t0 = static_cast<int64_t>(w) * work.tokens;
  const int ne = work.ne.d, per = c.d >> 3, shift = 31 - __builtin_clz(per);
  const int n = static_cast<int>(min(static_cast<int64_t>(work.tokens), T - t0)) * ne;
  const TI* const src = rows + t0 * ld;
  for (int i0 = threadIdx.x; i0 < n; i0 += kThreads * kPieces) {
    float f[kPieces][8];
    int64_t slot[kPieces];
    int piece[kPieces];
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      const int i = i0 + j * kThreads;           // four threads of a block of 32 go together: 4 | ne and 4 | n
      slot[j] = -1;
      if (i >= n) continue;
      const int t = work.ne(i);
      piece[j] = i - t * ne;
      slot[j] = slots[t0 + t];
      load8(src + static_cast<uint64_t>(static_cast<uint32_t>(t)) * static_cast<uint32_t>(ld) + piece[j] * 8, f[j]);
    }
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      if (slot[j] < 0 || slot[j] >= c.slots()) continue;
      // (store8 written out: its loop over elements in a function of its own costs 15 registers more a pass, and 8191 tokens
      // of 8 x 128 written and 8704 read 18.7 us instead of 17.9)
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(f[j][i]) & 0x7fffffffu);
      const BlockScale b = block_scale(top);
      const uint32_t q = codes8(f[j], b);
      const int head = piece[j] >> shift, e = piece[j] & (per - 1);
      const At at = place(c, slot[j], head, e, value);
      *reinterpret_cast<uint32_t*>((value ? c.vc : c.kc) + at.code) = q;
      if ((e & 3) == 0) (value ? c.vs : c.ks)[at.scale] = static_cast<uint8_t>(b.s);
    }
  }
}

// Enough workgroups for every compute unit first, then kPieces pieces a thread.
Work work_of(const KvCache& c, int T, int elements = 8) {
  const int64_t ne = static_cast<int64_t>(c.heads) * c.d / elements;
  const int64_t spread = (T + 1023) / 1024, full = (kThreads * kPieces + ne - 1) / ne;
  return {Divider(static_cast<uint32_t>(ne)), static_cast<int>(std::max<int64_t>(1, std::min(spread, full)))};
}
int64_t groups_of(const Work& w, int T) { return (T + static_cast<int64_t>(w.tokens) - 1) / w.tokens; }

}  // namespace
}  // namespace cts
