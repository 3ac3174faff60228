// The norms around a block (cts_block_norm) and rotary positions (cts_rotary): both read
// each element once and write it once, and are bound by memory (4096 x 4096 in bf16 with
// norms on both sides: 22 us, 6.0 TB/s; 6007 tokens of 40 heads of 128 turned on
// three axes: 23.4 us, 5.3 TB/s), by their launch for a few tokens (3.0 to 3.5 us in a graph).
#include <algorithm>

#include "block_internal.h"
#include "rows.h"

namespace cts {
namespace {

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

template <typename T, int HEADS, bool NT>
__global__ __launch_bounds__(kRotThreads) void rotary_kernel(RotaryParams p, int64_t t0, int n) {
  const int i = blockIdx.x * kRotThreads + threadIdx.x;
  if (i < n) turn_heads<T, HEADS, NT>(p, t0, i);
}

template <typename T, int HEADS, bool NT> void rotary_launch(RotaryParams p, hipStream_t s) {
  set_threads<HEADS>(&p);
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
