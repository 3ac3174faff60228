// The cache's writes and reads (cts_kv_write, cts_kv_read): 32 elements along
// the head dimension share a power of two, each element is a 4-bit float
// (1 sign, 2 exponent, 1 mantissa bit).
//
// Bound by memory: a bf16 token's head row of d elements is 2 d bytes one way and
// 0.53 d the other.  A thread takes 8 elements (one or two 16-byte accesses on the
// dense side, 4 bytes on the packed side), four threads a block of 32; gfx950
// converts two elements an instruction and scales them on the way.
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

// 8 elements as pairs of bf16
template <typename TO> __device__ __forceinline__ void store8(TO* p, const uint32_t* w);
template <> __device__ __forceinline__ void store8<bf16_t>(bf16_t* p, const uint32_t* w) {
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
template <> __device__ __forceinline__ void store8<float>(float* p, const uint32_t* w) {
  float f[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
  reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}

// Where 8 elements (eighth e of a head row) of a slot lie: code and scale bytes.
struct At { int64_t code, scale; };
__device__ __forceinline__ At place(const KvCache& c, int64_t slot, int head, int e, bool value) {
  const int64_t page = slot >> c.page_shift;
  const int o = static_cast<int>(slot & ((1 << c.page_shift) - 1));
  const int64_t row = (page * c.heads + head) << c.page_shift;      // the (page, head)'s first token
  const int ne = c.d >> 3, nb = c.d >> 5;
  if (!value) return {(row + o) * (c.d >> 1) + e * 4, (row + o) * nb + (e >> 2)};
  return {row * (c.d >> 1) + ((o >> 2) * ne + e) * 16 + (o & 3) * 4, row * nb + ((o >> 2) * nb + (e >> 2)) * 4 + (o & 3)};
}

template <typename TI>
__global__ __launch_bounds__(kThreads) void kv_write_kernel(KvCache c, int T, const TI* __restrict__ k, int64_t ldk,
                                                            const TI* __restrict__ v, int64_t ldv,
                                                            const int64_t* __restrict__ slots) {
  const int ne = c.heads * (c.d >> 3);                               // eighths of a token's keys
  const int64_t id = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  const int64_t t = id / ne;
  if (t >= T) return;                                                // four threads of a block leave together: 4 | ne
  const int64_t slot = slots[t];
  if (slot < 0 || slot >= c.slots()) return;
  const bool value = blockIdx.y;
  const int e_all = static_cast<int>(id - t * ne);
  float f[8];
  load8(value ? v + t * ldv + e_all * 8 : k + t * ldk + e_all * 8, f);
  // the largest magnitude as an integer: it orders like the value, NaN above all
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(f[i]) & 0x7fffffffu);
  top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 1)));
  top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 2)));
  const bool finite = top < 0x7f800000u;
  // a mantissa from 1.75 on would round past 6: the next power of two then
  const int s = finite ? min(252, max(1, static_cast<int>((top + (1u << 21)) >> 23) - 2)) : 255;
  uint32_t q = 0;
  if (finite) {
    const float unit = __uint_as_float(static_cast<uint32_t>(s) << 23);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, f[0], f[1], unit, 0);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, f[2], f[3], unit, 1);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, f[4], f[5], unit, 2);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, f[6], f[7], unit, 3);
  }
  const int head = e_all / (c.d >> 3), e = e_all - head * (c.d >> 3);
  const At at = place(c, slot, head, e, value);
  *reinterpret_cast<uint32_t*>((value ? c.vc : c.kc) + at.code) = q;
  if ((e & 3) == 0) (value ? c.vs : c.ks)[at.scale] = static_cast<uint8_t>(s);
}

template <typename TO>
__global__ __launch_bounds__(kThreads) void kv_read_kernel(KvCache c, int T, const int64_t* __restrict__ slots,
                                                           TO* __restrict__ k, int64_t ldk, TO* __restrict__ v,
                                                           int64_t ldv) {
  const int ne = c.heads * (c.d >> 3);
  const int64_t id = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  const int64_t t = id / ne;
  if (t >= T) return;
  const bool value = blockIdx.y;
  const int e_all = static_cast<int>(id - t * ne);
  const int64_t slot = slots[t];
  uint32_t w[4] = {0, 0, 0, 0};
  if (slot >= 0 && slot < c.slots()) {
    const int head = e_all / (c.d >> 3), e = e_all - head * (c.d >> 3);
    const At at = place(c, slot, head, e, value);
    const uint32_t q = *reinterpret_cast<const uint32_t*>((value ? c.vc : c.kc) + at.code);
    const float unit = __uint_as_float(static_cast<uint32_t>((value ? c.vs : c.ks)[at.scale]) << 23);
    w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, unit, 0));
    w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, unit, 1));
    w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, unit, 2));
    w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, unit, 3));
  }
  store8(value ? v + t * ldv + e_all * 8 : k + t * ldk + e_all * 8, w);
}

dim3 grid_of(const KvCache& c, int T) {
  const int64_t n = static_cast<int64_t>(T) * c.heads * (c.d >> 3);
  return dim3(static_cast<uint32_t>((n + kThreads - 1) / kThreads), 2);
}

}  // namespace

hipError_t launch_kv_write(const KvCache& c, int T, const void* k, int64_t ldk, const void* v, int64_t ldv,
                           const int64_t* slots, int dtype, hipStream_t s) {
  if (dtype == CTS_F32)
    kv_write_kernel<float><<<grid_of(c, T), kThreads, 0, s>>>(c, T, static_cast<const float*>(k), ldk,
                                                              static_cast<const float*>(v), ldv, slots);
  else
    kv_write_kernel<bf16_t><<<grid_of(c, T), kThreads, 0, s>>>(c, T, static_cast<const bf16_t*>(k), ldk,
                                                               static_cast<const bf16_t*>(v), ldv, slots);
  return hipGetLastError();
}

hipError_t launch_kv_read(const KvCache& c, int T, const int64_t* slots, void* k, int64_t ldk, void* v, int64_t ldv,
                          int dtype, hipStream_t s) {
  if (dtype == CTS_F32)
    kv_read_kernel<float><<<grid_of(c, T), kThreads, 0, s>>>(c, T, slots, static_cast<float*>(k), ldk,
                                                             static_cast<float*>(v), ldv);
  else
    kv_read_kernel<bf16_t><<<grid_of(c, T), kThreads, 0, s>>>(c, T, slots, static_cast<bf16_t*>(k), ldk,
                                                              static_cast<bf16_t*>(v), ldv);
  return hipGetLastError();
}

}  // namespace cts
