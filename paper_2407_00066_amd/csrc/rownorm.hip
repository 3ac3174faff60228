// The norms around a block (cts_block_norm) and rotary positions (cts_rotary): both read
// each element once and write it once, and are bound by memory (4096 x 4096 in bf16 with
// norms on both sides: 22 us, 6.0 TB/s; 6007 tokens of 40 heads of 128 turned: 29 us,
// 4.3 TB/s), by their launch for a few tokens (3.3 us in a graph).
#include <algorithm>

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

// V elements at `at`, zeros past the row's end (d is a multiple of V): the address is
// clamped instead of the load skipped, so that all of a row's loads go out together.
template <typename T, int V> __device__ __forceinline__ void get_or_zero(const T* p, uint32_t at, uint32_t d, float* f) {
  get<T, V>(p + min(at, d - V), f);
  if (at >= d)
#pragma unroll
    for (int j = 0; j < V; ++j) f[j] = 0.0f;
}

// Sum over the row's THREADS threads, in a fixed order.
template <int THREADS> __device__ __forceinline__ float row_sum(float v, float* lds) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o);
  if constexpr (THREADS > 64) {
    __syncthreads();                                // the last sum's readers are done
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0f;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) v += lds[w];
  }
  return v;
}

// THREADS threads hold a row in registers, at most 32 elements each, so that
// x and y are read once whatever is computed from them.
template <typename T, int THREADS, int V, int NV, bool NT>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void block_norm_kernel(NormParams p) {
  __shared__ float lds[THREADS / 64];
  constexpr int kRows = THREADS < 256 ? 256 / THREADS : 1;
  const uint32_t tid = threadIdx.x % THREADS;
  // (the row's number in a scalar register: its addresses are scalars and one offset)
  const int64_t t = static_cast<int64_t>(blockIdx.x) * kRows + __builtin_amdgcn_readfirstlane(threadIdx.x / THREADS);
  if (t >= p.T) return;                             // whole waves, and no barrier where rows are a wave's
  const uint32_t d = p.d;
  const T* x = static_cast<const T*>(p.x) + t * p.ldx;
  float a[NV][V];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const uint32_t at = (i * THREADS + tid) * V;
    get_or_zero<T, V>(x, at, d, a[i]);
  }
  if (p.y) {
    const T* y = static_cast<const T*>(p.y) + t * p.ldy;
    const T* gate = p.gate ? static_cast<const T*>(p.gate) + t * p.ldg : nullptr;
    const T* post = static_cast<const T*>(p.post);
    T* const h = static_cast<T*>(p.h) + t * p.ldh;
    float u[NV][V];
    float sq = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const uint32_t at = (i * THREADS + tid) * V;
      get_or_zero<T, V>(y, at, d, u[i]);
#pragma unroll
      for (int j = 0; j < V; ++j) sq += u[i][j] * u[i][j];
    }
    float rs = 1.0f;
    if (post) rs = rsqrtf(row_sum<THREADS>(sq, lds) / p.d + p.eps);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const uint32_t at = (i * THREADS + tid) * V;
      float w[V];
      if (post) {
        get_or_zero<T, V>(post, at, d, w);
#pragma unroll
        for (int j = 0; j < V; ++j) u[i][j] *= rs * w[j];
      }
      if (gate) {
        get_or_zero<T, V>(gate, at, d, w);
#pragma unroll
        for (int j = 0; j < V; ++j) u[i][j] *= w[j];
      }
#pragma unroll
      for (int j = 0; j < V; ++j) a[i][j] += p.scale * u[i][j];
      if (at < d) put<T, V, NT>(h + at, a[i]);
    }
  }
  const T* const weight = static_cast<const T*>(p.weight);
  T* const n = static_cast<T*>(p.n) + t * p.ldn;
  float sq = 0.0f;
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < V; ++j) sq += a[i][j] * a[i][j];
  const float rs = rsqrtf(row_sum<THREADS>(sq, lds) / p.d + p.eps);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const uint32_t at = (i * THREADS + tid) * V;
    float w[V];
    get_or_zero<T, V>(weight, at, d, w);
#pragma unroll
    for (int j = 0; j < V; ++j) w[j] *= rs * a[i][j];
    if (at < d) put<T, V, NT>(n + at, w);
  }
}

template <typename T, int THREADS, int V, bool NT> void norm_launch(const NormParams& p, hipStream_t s) {
  constexpr int kRows = THREADS < 256 ? 256 / THREADS : 1;
  constexpr int kBlock = THREADS < 256 ? 256 : THREADS;
  const int nv = (p.d + THREADS * V - 1) / (THREADS * V);
  const uint32_t grid = static_cast<uint32_t>((p.T + kRows - 1) / kRows);
  constexpr int kMost = 32 / V;
  if constexpr (THREADS == 64) {                    // (wider rows have more than 8 elements a thread)
    if (nv <= kMost / 4) {
      block_norm_kernel<T, THREADS, V, kMost / 4, NT><<<grid, kBlock, 0, s>>>(p);
      return;
    }
  }
  if (nv <= kMost / 2) block_norm_kernel<T, THREADS, V, kMost / 2, NT><<<grid, kBlock, 0, s>>>(p);
  else block_norm_kernel<T, THREADS, V, kMost, NT><<<grid, kBlock, 0, s>>>(p);
}

template <typename T, int THREADS, int V> void norm_launch(const NormParams& p, hipStream_t s) {
  if constexpr (V > 1) {
    if ((p.y ? 2 : 1) * sizeof(T) * p.T * p.d >= kStreamBytes) return norm_launch<T, THREADS, V, true>(p, s);
  }
  norm_launch<T, THREADS, V, false>(p, s);
}

template <typename T, int V> void norm_rows(const NormParams& p, hipStream_t s) {
  if (p.d <= 64 * 32) norm_launch<T, 64, V>(p, s);
  else if (p.d <= 256 * 32) norm_launch<T, 256, V>(p, s);
  else norm_launch<T, 1024, V>(p, s);
}

template <typename T> bool vectors(const NormParams& p) {
  uintptr_t bits = static_cast<uintptr_t>(p.d) | static_cast<uintptr_t>(p.ldx | p.ldy | p.ldg | p.ldh | p.ldn);
  bits *= sizeof(T);
  for (const void* q : {p.x, p.y, p.post, p.gate, p.weight, static_cast<const void*>(p.h), static_cast<const void*>(p.n)})
    bits |= reinterpret_cast<uintptr_t>(q);
  return (bits & 15) == 0;
}

template <typename T> void norm_typed(NormParams p, hipStream_t s) {
  constexpr int kMost = static_cast<int>(max_groups(1024));     // rows of a launch, whatever threads a row has
  for (int left = p.T; left > 0; left -= kMost) {
    p.T = std::min(left, kMost);
    if (vectors<T>(p)) norm_rows<T, Elem<T>::N>(p, s);
    else norm_rows<T, 1>(p, s);
    if (left <= kMost) break;
    p.x = static_cast<const T*>(p.x) + p.ldx * kMost;
    p.n = static_cast<T*>(p.n) + p.ldn * kMost;
    if (p.y) {
      p.y = static_cast<const T*>(p.y) + p.ldy * kMost;
      p.h = static_cast<T*>(p.h) + p.ldh * kMost;
      if (p.gate) p.gate = static_cast<const T*>(p.gate) + p.ldg * kMost;
    }
  }
}

// ------------------------------------------------------------------- rotary
constexpr int kRotThreads = 256;

// A thread turns 8 pairs of a head (with halves, 8 elements of each half; interleaved, 16
// consecutive ones) or copies 8 elements past rot, for HEADS heads that share the
// pairs' angles: their cosines and sines are loaded once for all of them.
template <typename T, int HEADS, bool NT>
__global__ __launch_bounds__(kRotThreads) void rotary_kernel(RotaryParams p, int64_t t0, int n) {
  constexpr int N = Elem<T>::N;
  const int i = blockIdx.x * kRotThreads + threadIdx.x;
  if (i >= n) return;
  const int64_t t = t0 + p.per_token(i);
  const int in_token = i - p.per_token(i) * p.per_token.d;
  const int group = p.per_head(in_token), piece = in_token - group * p.per_head.d;
  const int heads = p.heads[0] + p.heads[1], groups = (heads + HEADS - 1) / HEADS;
  const int pieces = p.rot / 16, half = p.rot / 2;
  const bool turns = piece < pieces;
  const int j0 = piece * 8;                       // the first pair
  const int at0 = !turns ? p.rot + (piece - pieces) * 8 : p.interleaved ? 2 * j0 : j0;
  const int at1 = p.interleaved ? 2 * j0 + 8 : j0 + half;
  float a[HEADS][16];
  T* o[HEADS];
#pragma unroll
  for (int k = 0; k < HEADS; ++k) {
    const int all = group + k * groups;
    o[k] = nullptr;
    if (all >= heads) continue;
    const int which = all >= p.heads[0], head = which ? all - p.heads[0] : all;
    const T* x = static_cast<const T*>(p.in[which]) + t * p.ldi[which] + static_cast<int64_t>(head) * p.d;
    o[k] = static_cast<T*>(p.out[which]) + t * p.ldo[which] + static_cast<int64_t>(head) * p.d;
#pragma unroll
    for (int e = 0; e < 8; e += N) get<T, N>(x + at0 + e, a[k] + e);
    if (turns)
#pragma unroll
      for (int e = 0; e < 8; e += N) get<T, N>(x + at1 + e, a[k] + 8 + e);
  }
  if (turns) {
    float c[8], s[8];
    int axis = 0;
    while (axis + 1 < p.axes && j0 >= p.end[axis]) ++axis;
    auto row = [&](int ax) {
      return static_cast<int64_t>(min(max(p.pos[static_cast<int64_t>(ax) * p.T + t], 0), p.n_pos - 1)) * half + j0;
    };
    if (j0 + 8 <= p.end[axis]) {                  // one axis: 32 bytes of each table
      const int64_t at = row(axis);
#pragma unroll
      for (int j = 0; j < 8; j += 4) {
        get<float, 4>(p.cos + at + j, c + j);
        get<float, 4>(p.sin + at + j, s + j);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        while (axis + 1 < p.axes && j0 + j >= p.end[axis]) ++axis;
        const int64_t at = row(axis) + j;
        c[j] = p.cos[at];
        s[j] = p.sin[at];
      }
    }
#pragma unroll
    for (int k = 0; k < HEADS; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float& lo = p.interleaved ? a[k][2 * j] : a[k][j];
        float& hi = p.interleaved ? a[k][2 * j + 1] : a[k][8 + j];
        const float x1 = lo, x2 = hi;
        lo = x1 * c[j] - x2 * s[j];
        hi = x2 * c[j] + x1 * s[j];
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

template <typename T, int HEADS, bool NT> void rotary_launch(RotaryParams p, hipStream_t s) {
  const int per = p.rot / 16 + (p.d - p.rot) / 8, groups = (p.heads[0] + p.heads[1] + HEADS - 1) / HEADS;
  p.per_head = Divider(per);
  p.per_token = Divider(per * groups);
  // thread numbers stay below 2^31: more tokens than that take several launches
  const int64_t most = 0x7fffff00 / p.per_token.d;
  for (int64_t t0 = 0; t0 < p.T; t0 += most) {
    const int n = static_cast<int>(std::min<int64_t>(most, p.T - t0) * p.per_token.d);
    rotary_kernel<T, HEADS, NT><<<(n + kRotThreads - 1) / kRotThreads, kRotThreads, 0, s>>>(p, t0, n);
  }
}

template <typename T> void rotary_typed(const RotaryParams& p, hipStream_t s) {
  // Angles shared by four heads where that leaves workgroups enough (6007 tokens of 40
  // heads of 128 with 1, 2, 4 heads a thread: 47, 41, 37 us, before streaming stores);
  // such outputs are of 32 MB and more.
  const int64_t n = static_cast<int64_t>(p.T) * (p.heads[0] + p.heads[1]) * (p.d / 16);
  constexpr int64_t kShared = kRotThreads * 4 * 1024;
  static_assert(kShared * 16 * sizeof(T) >= kStreamBytes);
  if (n < kShared) rotary_launch<T, 1, false>(p, s);
  else rotary_launch<T, 4, true>(p, s);
}

}  // namespace

hipError_t launch_block_norm(const NormParams& p, int dtype, hipStream_t s) {
  if (dtype == CTS_F32) norm_typed<float>(p, s);
  else norm_typed<bf16_t>(p, s);
  return hipGetLastError();
}

hipError_t launch_rotary(const RotaryParams& p, int dtype, hipStream_t s) {
  if (dtype == CTS_F32) rotary_typed<float>(p, s);
  else rotary_typed<bf16_t>(p, s);
  return hipGetLastError();
}

}  // namespace cts
