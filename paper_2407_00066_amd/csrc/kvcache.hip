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
#include "kvblock.h"

namespace cts {
namespace {

template <typename TI>
__global__ __launch_bounds__(kThreads) void kv_write_kernel(KvCache c, Work work, int T, const TI* __restrict__ k,
                                                            int64_t ldk, const TI* __restrict__ v, int64_t ldv,
                                                            const int64_t* __restrict__ slots) {
  const bool value = blockIdx.y;
  write_rows<TI>(c, work, T, blockIdx.x, value ? v : k, value ? ldv : ldk, slots, value);
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
