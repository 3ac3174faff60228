// Rows of elements in device code: 16-byte accesses, and the turning of a row's heads
// by their positions (rownorm.hip, kvappend.hip).
#pragma once

#include "block_internal.h"

namespace cts {
namespace {

template <typename T> struct Elem;
template <> struct Elem<float> {
  static constexpr int N = 4;                       // elements of 16 bytes
  __device__ static __forceinline__ float get(const float* p) { return *p; }
  __device__ static __forceinline__ void put(float* p, float v) { *p = v; }
  __device__ static __forceinline__ void get16(const float* p, float* f) {
    const float4 v = *reinterpret_cast<const float4*>(p);
    f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
  }
  template <bool NT> __device__ static __forceinline__ void put16(float* p, const float* f) {
    store16<NT>(p, __float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
};
template <> struct Elem<bf16_t> {
  static constexpr int N = 8;
  __device__ static __forceinline__ float get(const bf16_t* p) { return bf16_to_f32(p->bits); }
  __device__ static __forceinline__ void put(bf16_t* p, float v) { p->bits = f32_to_bf16(v); }
  __device__ static __forceinline__ void get16(const bf16_t* p, float* f) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  template <bool NT> __device__ static __forceinline__ void put16(bf16_t* p, const float* f) {
    store16<NT>(p, f32_to_bf16_pair(f[0], f[1]), f32_to_bf16_pair(f[2], f[3]), f32_to_bf16_pair(f[4], f[5]),
                f32_to_bf16_pair(f[6], f[7]));
  }
};

// V consecutive elements: one 16-byte access, or one element
template <typename T, int V> __device__ __forceinline__ void get(const T* p, float* f) {
  if constexpr (V == 1) f[0] = Elem<T>::get(p);
  else Elem<T>::get16(p, f);
}
template <typename T, int V, bool NT> __device__ __forceinline__ void put(T* p, const float* f) {
  if constexpr (V == 1) Elem<T>::put(p, f[0]);
  else Elem<T>::template put16<NT>(p, f);
}

// A pair turned by its angle; the same two instructions each wherever it is computed, so
// that the calls that turn rows agree by bits.
__device__ __forceinline__ void turn(float& lo, float& hi, float c, float s) {
  const float x1 = lo, x2 = hi;
  lo = __builtin_fmaf(x1, c, -(x2 * s));
  hi = __builtin_fmaf(x2, c, x1 * s);
}

// Cosines and sines of token t's pairs j0 .. j0 + N - 1 (N 4 or 8, j0 a multiple of N): 16 or 32 bytes of each
// table for every axis that the pairs lie in, nearly always one or two (2003 tokens of 24 heads of 128 in
// fp32, 64 elements turned on three axes: with a load for every pair 20.3 us, so 13.6).
// pos0: the token's position on the first axis, which the caller asks for before its rows.
// The launch's arrays are read at indexes that the compiler knows, here and in turn_heads: at others it holds them all in
// registers and finds an entry by comparing, 470 selects a thread (64 and 2000 tokens of 32 + 8 heads of 128
// in bf16: 4.6 and 20.4 us, so 3.0 and 9.4).
template <int N>
__device__ __forceinline__ void angles(const RotaryParams& p, int64_t t, int pos0, int j0, float* c, float* s) {
  if (p.axes == 1) {
    const int row = min(max(pos0, 0), p.n_pos - 1);
    const int64_t at = static_cast<int64_t>(row) * (p.rot / 2) + j0;
#pragma unroll
    for (int j = 0; j < N; j += 4) {
      get<float, 4>(p.cos + at + j, c + j);
      get<float, 4>(p.sin + at + j, s + j);
    }
    return;
  }
  static_assert(kRotaryMaxAxes == 4);
  const int e0 = p.end[0], e1 = p.end[1], e2 = p.end[2], e3 = p.end[3];
  auto end_of = [=](int a) { return a == 0 ? e0 : a == 1 ? e1 : a == 2 ? e2 : e3; };
  int axis = 0;
  while (axis + 1 < p.axes && j0 >= end_of(axis)) ++axis;
  for (int from = 0;;) {                          // pairs from here on are of this axis or a later one
    const int row = min(max(p.pos[static_cast<int64_t>(axis) * p.T + t], 0), p.n_pos - 1);
    const int64_t at = static_cast<int64_t>(row) * (p.rot / 2) + j0;
    float cv[N], sv[N];
#pragma unroll
    for (int j = 0; j < N; j += 4) {
      get<float, 4>(p.cos + at + j, cv + j);
      get<float, 4>(p.sin + at + j, sv + j);
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
      c[j] = j >= from ? cv[j] : c[j];
      s[j] = j >= from ? sv[j] : s[j];
    }
    from = end_of(axis) - j0;
    if (from >= N || ++axis >= p.axes) return;
  }
}

// Thread `i` of the tokens from t0 on: it turns 8 pairs of a head (with halves, 8 elements of
// each half; interleaved, 16 consecutive ones) or copies 8 elements past rot, for HEADS
// heads that share the pairs' angles: their cosines and sines are loaded once for all of them.
template <typename T, int HEADS, bool NT>
__device__ __forceinline__ void turn_heads(const RotaryParams& p, int64_t t0, int i) {
  constexpr int N = Elem<T>::N;
  const int64_t t = t0 + p.per_token(i);
  const int in_token = i - p.per_token(i) * p.per_token.d;
  const int group = p.per_head(in_token), piece = in_token - group * p.per_head.d;
  const int heads = p.heads[0] + p.heads[1], groups = (heads + HEADS - 1) / HEADS;
  const int pieces = p.rot / 16, half = p.rot / 2;
  const bool turns = piece < pieces;
  const int j0 = piece * 8;                       // the first pair
  const int at0 = !turns ? p.rot + (piece - pieces) * 8 : p.interleaved ? 2 * j0 : j0;
  const int at1 = p.interleaved ? 2 * j0 + 8 : j0 + half;
  const int pos0 = p.pos[t];
  float a[HEADS][16];
  T* o[HEADS];
#pragma unroll
  for (int k = 0; k < HEADS; ++k) {
    const int all = group + k * groups;
    o[k] = nullptr;
    if (all >= heads) continue;
    const bool key = all >= p.heads[0];
    const int64_t head = key ? all - p.heads[0] : all;
    const T* x = static_cast<const T*>(key ? p.in[1] : p.in[0]) + t * (key ? p.ldi[1] : p.ldi[0]) + head * p.d;
    o[k] = static_cast<T*>(key ? p.out[1] : p.out[0]) + t * (key ? p.ldo[1] : p.ldo[0]) + head * p.d;
#pragma unroll
    for (int e = 0; e < 8; e += N) get<T, N>(x + at0 + e, a[k] + e);
    if (turns)
#pragma unroll
      for (int e = 0; e < 8; e += N) get<T, N>(x + at1 + e, a[k] + 8 + e);
  }
  if (turns) {
    float c[8] = {}, s[8] = {};
    angles<8>(p, t, pos0, j0, c, s);
#pragma unroll
    for (int k = 0; k < HEADS; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if constexpr (HEADS <= 2) {                 // (four heads: selects cost more than both branches' code)
          float& lo = p.interleaved ? a[k][2 * j] : a[k][j];
          float& hi = p.interleaved ? a[k][2 * j + 1] : a[k][8 + j];
          turn(lo, hi, c[j], s[j]);
        } else if (p.interleaved) {
          turn(a[k][2 * j], a[k][2 * j + 1], c[j], s[j]);
        } else {
          turn(a[k][j], a[k][8 + j], c[j], s[j]);
        }
      }
  }
#pragma unroll
  for (int k = 0; k < HEADS; ++k) {
    if (!o[k]) continue;
#pragma unroll
    for (int e = 0; e < 8; e += N) put<T, N, NT>(o[k] + at0 + e, a[k] + e);
    if (turns)
#pragma unroll
      for (int e = 0; e < 8; e += N) put<T, N, NT>(o[k] + at1 + e, a[k] + 8 + e);
  }
}

// The threads of a head and of a token that turn_heads takes.
template <int HEADS> void set_threads(RotaryParams* p) {
  const int per = p->rot / 16 + (p->d - p->rot) / 8, groups = (p->heads[0] + p->heads[1] + HEADS - 1) / HEADS;
  p->per_head = Divider(per);
  p->per_token = Divider(per * groups);
}

}  // namespace
}  // namespace cts
