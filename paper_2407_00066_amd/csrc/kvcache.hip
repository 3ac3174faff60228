// The cache's writes and reads (cts_kv_write, cts_kv_read): 32 elements along
// the head dimension share a power of two, each element is a 4-bit float
// (1 sign, 2 exponent, 1 mantissa bit).
//
// Bound by memory: a bf16 token's head row of d elements is 2 d bytes one way and
// 0.53 d the other.  A thread takes 8 elements (one or two 16-byte accesses on the
// dense side, 4 bytes on the packed side), four threads a block of 32, and a few
// such pieces of other tokens, whose loads go out together; gfx950 converts two elements
// an instruction and scales them on the way.  8191 tokens of 8 heads of 128 in bf16: written
// in 9.2 us (4.6 TB/s), 20011 read back in float in 30 us (6.2 TB/s).
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

template <typename TI>
__global__ __launch_bounds__(kThreads) void kv_write_kernel(KvCache c, Work work, int T, const TI* __restrict__ k,
                                                            int64_t ldk, const TI* __restrict__ v, int64_t ldv,
                                                            const int64_t* __restrict__ slots) {
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * work.tokens;
  const int ne = work.ne.d, per = c.d >> 3, shift = 31 - __builtin_clz(per);
  const int n = static_cast<int>(min(static_cast<int64_t>(work.tokens), T - t0)) * ne;
  const bool value = blockIdx.y;
  const TI* const src = value ? v + t0 * ldv : k + t0 * ldk;
  const int64_t ld = value ? ldv : ldk;
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
      // the largest magnitude as an integer: it orders like the value, NaN above all
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(f[j][i]) & 0x7fffffffu);
      top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 1)));
      top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 2)));
      const bool finite = top < 0x7f800000u;
      // a mantissa from 1.75 on would round past 6: the next power of two then
      const int s = finite ? min(252, max(1, static_cast<int>((top + (1u << 21)) >> 23) - 2)) : 255;
      uint32_t q = 0;
      if (finite) {
        const float unit = __uint_as_float(static_cast<uint32_t>(s) << 23);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, f[j][0], f[j][1], unit, 0);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, f[j][2], f[j][3], unit, 1);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, f[j][4], f[j][5], unit, 2);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, f[j][6], f[j][7], unit, 3);
      }
      const int head = piece[j] >> shift, e = piece[j] & (per - 1);
      const At at = place(c, slot[j], head, e, value);
      *reinterpret_cast<uint32_t*>((value ? c.vc : c.kc) + at.code) = q;
      if ((e & 3) == 0) (value ? c.vs : c.ks)[at.scale] = static_cast<uint8_t>(s);
    }
  }
}

// Read back: a thread writes 16 bytes, so that a wave's stores are whole lines: 8 elements
// of bf16 (an eighth), 4 of float (half of one).
template <typename TO, bool NT>
__global__ __launch_bounds__(kThreads) void kv_read_kernel(KvCache c, Work work, int T, const int64_t* __restrict__ slots,
                                                           TO* __restrict__ k, int64_t ldk, TO* __restrict__ v,
                                                           int64_t ldv) {
  constexpr int E = 16 / sizeof(TO), H = 8 / E;  // elements of a thread, threads of an eighth
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * work.tokens;
  const int ne = work.ne.d, per = c.d >> 3, shift = 31 - __builtin_clz(per);
  const int n = static_cast<int>(min(static_cast<int64_t>(work.tokens), T - t0)) * ne;
  const bool value = blockIdx.y;
  TO* const dst = value ? v + t0 * ldv : k + t0 * ldk;
  const int64_t ld = value ? ldv : ldk;
  for (int i0 = threadIdx.x; i0 < n; i0 += kThreads * kPieces) {
    int64_t slot[kPieces];
    int t[kPieces], piece[kPieces];
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      const int i = min(i0 + j * kThreads, n - 1);
      t[j] = work.ne(i);
      piece[j] = i - t[j] * ne;
      slot[j] = slots[t0 + t[j]];
    }
    uint32_t q[kPieces], s[kPieces];
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      q[j] = s[j] = 0;
      if (slot[j] < 0 || slot[j] >= c.slots()) continue;
      const int e = piece[j] / H;
      const At at = place(c, slot[j], e >> shift, e & (per - 1), value);
      const uint8_t* const code = (value ? c.vc : c.kc) + at.code;
      if constexpr (H == 1) q[j] = *reinterpret_cast<const uint32_t*>(code);
      else q[j] = reinterpret_cast<const uint16_t*>(code)[piece[j] & 1];
      s[j] = (value ? c.vs : c.ks)[at.scale];
    }
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      if (i0 + j * kThreads >= n) break;
      const float unit = __uint_as_float(s[j] << 23);
      TO* const to = dst + static_cast<uint64_t>(static_cast<uint32_t>(t[j])) * static_cast<uint32_t>(ld) + piece[j] * E;
      const uint32_t w0 = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q[j], unit, 0));
      const uint32_t w1 = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q[j], unit, 1));
      if constexpr (H == 1) {
        const uint32_t w2 = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q[j], unit, 2));
        const uint32_t w3 = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q[j], unit, 3));
        store16<NT>(to, w0, w1, w2, w3);
      } else {
        store16<NT>(to, w0 << 16, w0 & 0xffff0000u, w1 << 16, w1 & 0xffff0000u);
      }
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
dim3 grid_of(const Work& w, int T) { return dim3(static_cast<uint32_t>(groups_of(w, T)), 2); }

}  // namespace

bool kv_fits(const KvCache& c, int T, int elements) { return groups_of(work_of(c, T, elements), T) <= max_groups(kThreads); }

hipError_t launch_kv_write(const KvCache& c, int T, const void* k, int64_t ldk, const void* v, int64_t ldv,
                           const int64_t* slots, int dtype, hipStream_t s) {
  const Work w = work_of(c, T);
  if (dtype == CTS_F32)
    kv_write_kernel<float><<<grid_of(w, T), kThreads, 0, s>>>(c, w, T, static_cast<const float*>(k), ldk,
                                                              static_cast<const float*>(v), ldv, slots);
  else
    kv_write_kernel<bf16_t><<<grid_of(w, T), kThreads, 0, s>>>(c, w, T, static_cast<const bf16_t*>(k), ldk,
                                                               static_cast<const bf16_t*>(v), ldv, slots);
  return hipGetLastError();
}

template <typename TO>
static void read_launch(const KvCache& c, int T, const int64_t* slots, void* k, int64_t ldk, void* v, int64_t ldv,
                        hipStream_t s) {
  const Work w = work_of(c, T, 16 / sizeof(TO));
  TO *ko = static_cast<TO*>(k), *vo = static_cast<TO*>(v);
  if (2 * sizeof(TO) * T * c.heads * c.d >= kStreamBytes)
    kv_read_kernel<TO, true><<<grid_of(w, T), kThreads, 0, s>>>(c, w, T, slots, ko, ldk, vo, ldv);
  else
    kv_read_kernel<TO, false><<<grid_of(w, T), kThreads, 0, s>>>(c, w, T, slots, ko, ldk, vo, ldv);
}

hipError_t launch_kv_read(const KvCache& c, int T, const int64_t* slots, void* k, int64_t ldk, void* v, int64_t ldv,
                          int dtype, hipStream_t s) {
  if (dtype == CTS_F32) read_launch<float>(c, T, slots, k, ldk, v, ldv, s);
  else read_launch<bf16_t>(c, T, slots, k, ldk, v, ldv, s);
  return hipGetLastError();
}

}  // namespace cts
