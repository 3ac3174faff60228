// The norms around a block (cts_block_norm) and rotary positions (cts_rotary):
// both read each element once and write it once, and are bound by memory (by
// their launch for a few tokens).
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
  __device__ static __forceinline__ void put16(float* p, const float* f) {
    *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
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
  __device__ static __forceinline__ void put16(bf16_t* p, const float* f) {
    *reinterpret_cast<uint4*>(p) = make_uint4(f32_to_bf16_pair(f[0], f[1]), f32_to_bf16_pair(f[2], f[3]),
                                              f32_to_bf16_pair(f[4], f[5]), f32_to_bf16_pair(f[6], f[7]));
  }
};

// V consecutive elements: one 16-byte access, or one element
template <typename T, int V> __device__ __forceinline__ void get(const T* p, float* f) {
  if constexpr (V == 1) f[0] = Elem<T>::get(p);
  else Elem<T>::get16(p, f);
}
template <typename T, int V> __device__ __forceinline__ void put(T* p, const float* f) {
  if constexpr (V == 1) Elem<T>::put(p, f[0]);
  else Elem<T>::put16(p, f);
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
template <typename T, int THREADS, int V, int NV>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void block_norm_kernel(NormParams p) {
  __shared__ float lds[THREADS / 64];
  constexpr int kRows = THREADS < 256 ? 256 / THREADS : 1;
  const int tid = threadIdx.x % THREADS;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / THREADS;
  if (t >= p.T) return;                             // whole waves, and no barrier where rows are a wave's
  const T* x = static_cast<const T*>(p.x) + t * p.ldx;
  float a[NV][V];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int at = (i * THREADS + tid) * V;
#pragma unroll
    for (int j = 0; j < V; ++j) a[i][j] = 0.0f;
    if (at < p.d) get<T, V>(x + at, a[i]);
  }
  if (p.y) {
    const T* y = static_cast<const T*>(p.y) + t * p.ldy;
    const T* gate = p.gate ? static_cast<const T*>(p.gate) + t * p.ldg : nullptr;
    const T* post = static_cast<const T*>(p.post);
    float u[NV][V];
    float sq = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int at = (i * THREADS + tid) * V;
#pragma unroll
      for (int j = 0; j < V; ++j) u[i][j] = 0.0f;
      if (at < p.d) get<T, V>(y + at, u[i]);
#pragma unroll
      for (int j = 0; j < V; ++j) sq += u[i][j] * u[i][j];
    }
    float rs = 1.0f;
    if (post) rs = rsqrtf(row_sum<THREADS>(sq, lds) / p.d + p.eps);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int at = (i * THREADS + tid) * V;
      if (at >= p.d) continue;
      float w[V];
      if (post) {
        get<T, V>(post + at, w);
#pragma unroll
        for (int j = 0; j < V; ++j) u[i][j] *= rs * w[j];
      }
      if (gate) {
        get<T, V>(gate + at, w);
#pragma unroll
        for (int j = 0; j < V; ++j) u[i][j] *= w[j];
      }
#pragma unroll
      for (int j = 0; j < V; ++j) a[i][j] += p.scale * u[i][j];
      put<T, V>(static_cast<T*>(p.h) + t * p.ldh + at, a[i]);
    }
  }
  float sq = 0.0f;
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < V; ++j) sq += a[i][j] * a[i][j];
  const float rs = rsqrtf(row_sum<THREADS>(sq, lds) / p.d + p.eps);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int at = (i * THREADS + tid) * V;
    if (at >= p.d) continue;
    float w[V];
    get<T, V>(static_cast<const T*>(p.weight) + at, w);
#pragma unroll
    for (int j = 0; j < V; ++j) w[j] *= rs * a[i][j];
    put<T, V>(static_cast<T*>(p.n) + t * p.ldn + at, w);
  }
}

template <typename T, int THREADS, int V> void norm_launch(const NormParams& p, hipStream_t s) {
  constexpr int kRows = THREADS < 256 ? 256 / THREADS : 1;
  constexpr int kBlock = THREADS < 256 ? 256 : THREADS;
  const int nv = (p.d + THREADS * V - 1) / (THREADS * V);
  const uint32_t grid = static_cast<uint32_t>((p.T + kRows - 1) / kRows);
  constexpr int kMost = 32 / V;
  if (nv <= kMost / 4) block_norm_kernel<T, THREADS, V, kMost / 4><<<grid, kBlock, 0, s>>>(p);
  else if (nv <= kMost / 2) block_norm_kernel<T, THREADS, V, kMost / 2><<<grid, kBlock, 0, s>>>(p);
  else block_norm_kernel<T, THREADS, V, kMost><<<grid, kBlock, 0, s>>>(p);
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

template <typename T> void norm_typed(const NormParams& p, hipStream_t s) {
  if (vectors<T>(p)) norm_rows<T, Elem<T>::N>(p, s);
  else norm_rows<T, 1>(p, s);
}

// ------------------------------------------------------------------- rotary
constexpr int kRotThreads = 256;

// A thread turns 8 pairs of one head: with halves, 8 elements of each half; interleaved,
// 16 consecutive ones.  Then the elements past rot are copied, 8 a thread.
template <typename T>
__global__ __launch_bounds__(kRotThreads) void rotary_kernel(RotaryParams p) {
  constexpr int N = Elem<T>::N;
  const int pieces = p.rot / 16, tail = (p.d - p.rot) / 8, per = pieces + tail;
  const int heads = p.heads[0] + p.heads[1];
  const int64_t id = static_cast<int64_t>(blockIdx.x) * kRotThreads + threadIdx.x;
  const int64_t hid = id / per;
  const int piece = static_cast<int>(id - hid * per);
  const int64_t t = hid / heads;
  if (t >= p.T) return;
  int head = static_cast<int>(hid - t * heads);
  const int which = head >= p.heads[0];
  if (which) head -= p.heads[0];
  const T* x = static_cast<const T*>(p.in[which]) + t * p.ldi[which] + static_cast<int64_t>(head) * p.d;
  T* o = static_cast<T*>(p.out[which]) + t * p.ldo[which] + static_cast<int64_t>(head) * p.d;
  float a[16];
  if (piece >= pieces) {
    const int at = p.rot + (piece - pieces) * 8;
#pragma unroll
    for (int i = 0; i < 8; i += N) get<T, N>(x + at + i, a + i);
#pragma unroll
    for (int i = 0; i < 8; i += N) put<T, N>(o + at + i, a + i);
    return;
  }
  const int half = p.rot / 2, j0 = piece * 8;
  float c[8], s[8];
  int axis = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    while (axis + 1 < p.axes && j0 + j >= p.end[axis]) ++axis;
    const int pos = min(max(p.pos[static_cast<int64_t>(axis) * p.T + t], 0), p.n_pos - 1);
    c[j] = p.cos[static_cast<int64_t>(pos) * half + j0 + j];
    s[j] = p.sin[static_cast<int64_t>(pos) * half + j0 + j];
  }
  const int at0 = p.interleaved ? 2 * j0 : j0, at1 = p.interleaved ? 2 * j0 + 8 : j0 + half;
#pragma unroll
  for (int i = 0; i < 8; i += N) get<T, N>(x + at0 + i, a + i);
#pragma unroll
  for (int i = 0; i < 8; i += N) get<T, N>(x + at1 + i, a + 8 + i);
  if (p.interleaved) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float x1 = a[2 * j], x2 = a[2 * j + 1];
      a[2 * j] = x1 * c[j] - x2 * s[j];
      a[2 * j + 1] = x2 * c[j] + x1 * s[j];
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float x1 = a[j], x2 = a[8 + j];
      a[j] = x1 * c[j] - x2 * s[j];
      a[8 + j] = x2 * c[j] + x1 * s[j];
    }
  }
#pragma unroll
  for (int i = 0; i < 8; i += N) put<T, N>(o + at0 + i, a + i);
#pragma unroll
  for (int i = 0; i < 8; i += N) put<T, N>(o + at1 + i, a + 8 + i);
}

}  // namespace

hipError_t launch_block_norm(const NormParams& p, int dtype, hipStream_t s) {
  if (dtype == CTS_F32) norm_typed<float>(p, s);
  else norm_typed<bf16_t>(p, s);
  return hipGetLastError();
}

hipError_t launch_rotary(const RotaryParams& p, int dtype, hipStream_t s) {
  const int64_t n = static_cast<int64_t>(p.T) * (p.heads[0] + p.heads[1]) * (p.rot / 16 + (p.d - p.rot) / 8);
  const uint32_t grid = static_cast<uint32_t>((n + kRotThreads - 1) / kRotThreads);
  if (dtype == CTS_F32) rotary_kernel<float><<<grid, kRotThreads, 0, s>>>(p);
  else rotary_kernel<bf16_t><<<grid, kRotThreads, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace cts
