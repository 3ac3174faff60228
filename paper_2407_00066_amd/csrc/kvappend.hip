// New tokens into the cache with their positions turned on the way (cts_kv_append), and the
// accepted ones of a step's drafts moved up behind their sequence (cts_kv_keep).
//
// Append is rotary and the cache's write in one launch, on the same formulas and with
// the same roundings: a key is turned in float, rounded to its type and then
// quantised.  Bound by memory like those two; a key is read once from memory
// instead of twice, and its turned row is not written.  Workgroups take keys, values or queries.
// A thread has 8 elements of a key: the 8 that they are turned with are another thread's, and
// read again from the nearest cache instead of exchanged, so that any rot will do.
#include "kvblock.h"
#include "rows.h"

namespace cts {
namespace {

struct Append {
  KvCache c;
  Work work;
  RotaryParams r;                                // [0] the queries, [1] the keys (out may be null)
  const void* v; int64_t ldv;
  const int64_t* slots;
  uint32_t kv_groups;                            // workgroups of keys and values, in turn; then come those of queries
  int q_threads;
};

// f[8], eighth e of a key of token t, turned; at: the key's row.
template <typename T> __device__ __forceinline__ void turn8(const RotaryParams& p, int64_t t, int e, const T* at, float* f) {
  const int half = p.rot / 2, first = 8 * e;
  if (first >= p.rot) return;
  float c[8], s[8];
  if (p.interleaved) {
    angles<4>(p, t, first / 2, c, s);
#pragma unroll
    for (int j = 0; j < 4; ++j) turn(f[2 * j], f[2 * j + 1], c[j], s[j]);
  } else {
    const bool low = first < half;
    const int j0 = low ? first : first - half;
    float g[8];
    load8(at + (low ? first + half : j0), g);
    angles<8>(p, t, j0, c, s);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float lo = low ? f[j] : g[j], hi = low ? g[j] : f[j];
      turn(lo, hi, c[j], s[j]);
      f[j] = low ? lo : hi;
    }
  }
}

// as the type holds them
__device__ __forceinline__ void round8(float*, float*) {}
__device__ __forceinline__ void round8(bf16_t*, float* f) {
#pragma unroll
  for (int j = 0; j < 8; j += 2) {
    const uint32_t w = f32_to_bf16_pair(f[j], f[j + 1]);
    f[j] = __uint_as_float(w << 16);
    f[j + 1] = __uint_as_float(w & 0xffff0000u);
  }
}

template <typename T, int HEADS, bool NT>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(Append p) {
  if (blockIdx.x >= p.kv_groups) {
    const int i = static_cast<int>(blockIdx.x - p.kv_groups) * kThreads + threadIdx.x;
    if (i < p.q_threads) turn_heads<T, HEADS, NT>(p.r, 0, i);
    return;
  }
  const int64_t t0 = static_cast<int64_t>(blockIdx.x >> 1) * p.work.tokens;
  const int ne = p.work.ne.d, per = p.c.d >> 3, shift = 31 - __builtin_clz(per);
  const int n = static_cast<int>(min(static_cast<int64_t>(p.work.tokens), p.r.T - t0)) * ne;
  const bool value = blockIdx.x & 1;
  const T* const src = static_cast<const T*>(value ? p.v : p.r.in[1]);
  const int64_t ld = value ? p.ldv : p.r.ldi[1];
  // A head's threads are neighbours in one wave, whose loads are all done before it stores:
  // turned keys may be written over the keys themselves.
  for (int i0 = threadIdx.x; i0 < n; i0 += kThreads * kPieces) {
    float f[kPieces][8];
    int64_t slot[kPieces];
    int piece[kPieces];
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      const int i = i0 + j * kThreads;           // four threads of a block of 32 go together: 4 | ne and 4 | n
      slot[j] = -1;
      if (i >= n) continue;
      const int64_t t = t0 + p.work.ne(i);
      piece[j] = i - static_cast<int>(p.work.ne(i)) * ne;
      slot[j] = p.slots[t];
      const T* const row = src + t * ld;
      load8(row + piece[j] * 8, f[j]);
      if (!value) {
        const int e = piece[j] & (per - 1);
        turn8(p.r, t, e, row + (piece[j] - e) * 8, f[j]);
        round8(static_cast<T*>(nullptr), f[j]);
      }
    }
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      const int i = i0 + j * kThreads;
      if (i >= n) continue;
      if (!value && p.r.out[1]) {
        T* const o = static_cast<T*>(p.r.out[1]) + (t0 + p.work.ne(i)) * p.r.ldo[1] + piece[j] * 8;
#pragma unroll
        for (int x = 0; x < 8; x += Elem<T>::N) put<T, Elem<T>::N, NT>(o + x, f[j] + x);
      }
      if (slot[j] < 0 || slot[j] >= p.c.slots()) continue;
      store8(p.c, slot[j], piece[j] >> shift, piece[j] & (per - 1), value, f[j]);
    }
  }
}

// Workgroups of a call's queries; more than this many threads are not counted in 31 bits.
constexpr int64_t kMostQuery = 0x7fffff00;
int64_t query_threads(const RotaryParams& r) { return static_cast<int64_t>(r.T) * (r.heads[0] ? r.per_token.d : 0); }

template <typename T, int HEADS, bool NT> hipError_t append_launch(Append p, hipStream_t s) {
  if (p.r.heads[0]) set_threads<HEADS>(&p.r);
  p.q_threads = static_cast<int>(query_threads(p.r));
  const uint32_t q_groups = static_cast<uint32_t>((static_cast<int64_t>(p.q_threads) + kThreads - 1) / kThreads);
  kv_append_kernel<T, HEADS, NT><<<p.kv_groups + q_groups, kThreads, 0, s>>>(p);
  return hipGetLastError();
}

template <typename T> hipError_t append_typed(const Append& p, hipStream_t s) {
  // (the rule of rotary)
  constexpr int64_t kShared = kThreads * 4 * 1024;
  if (static_cast<int64_t>(p.r.T) * p.r.heads[0] * (p.r.d / 16) < kShared) return append_launch<T, 1, false>(p, s);
  return append_launch<T, 4, true>(p, s);
}

// ------------------------------------------------------------------- keep
// A workgroup takes one block of 32 elements of one head of a sequence: all of its accepted
// tokens are read before any is written, so that no order and no repetition of them matters.
constexpr int kKeepThreads = 128, kKeepParts = 8;

struct alignas(16) Kept { uint32_t k[4], v[4]; };

__global__ __launch_bounds__(kKeepThreads) void kv_keep_kernel(KvCache c, int max_pages, const int32_t* __restrict__ table,
                                                               const int32_t* __restrict__ kv_len,
                                                               const int32_t* __restrict__ q_start,
                                                               const int32_t* __restrict__ path,
                                                               const int32_t* __restrict__ n_path, int max_path) {
  __shared__ Kept kept[kKeepMaxPath];
  __shared__ uint8_t scales[kKeepMaxPath][2];
  __shared__ int64_t to[kKeepMaxPath];           // the slot that an accepted draft takes, -1: none
  const int blocks = c.d >> 5, blk = blockIdx.x % blocks, h = blockIdx.x / blocks % c.heads;
  const int64_t b = blockIdx.x / blocks / c.heads;
  const int64_t room = static_cast<int64_t>(max_pages) << c.page_shift;
  const int64_t len = min(static_cast<int64_t>(max(kv_len[b], 0)), room);
  const int64_t n = max(static_cast<int64_t>(q_start[b + 1]) - q_start[b], static_cast<int64_t>(0)), past = len - n;
  const int m = min(max(n_path[b], 0), max_path);
  auto slot_of = [&](int64_t pos) -> int64_t {
    if (pos < 0 || pos >= len) return -1;
    const int32_t page = table[b * max_pages + (pos >> c.page_shift)];
    if (page < 0 || page >= c.n_pages) return -1;
    return static_cast<int64_t>(page) << c.page_shift | (pos & ((1 << c.page_shift) - 1));
  };
  const int part = threadIdx.x % kKeepParts;     // 0: keys; 1 .. 4: an eighth of the values; 5, 6: their scales
  const bool value = part != 0 && part != 5;
  const int e = 4 * blk + (part >= 1 && part <= 4 ? part - 1 : 0);
  for (int i = threadIdx.x / kKeepParts; i < m; i += kKeepThreads / kKeepParts) {
    const int32_t from_draft = path[b * max_path + i];
    const int64_t from = from_draft >= 0 && from_draft < n ? slot_of(past + from_draft) : -1;
    const int64_t dest = from < 0 || from_draft == i ? -1 : slot_of(past + i);
    if (part == 7) {
      to[i] = dest;
    } else if (dest >= 0) {
      const At at = place(c, from, h, e, value);
      if (part == 0) *reinterpret_cast<uint4*>(kept[i].k) = *reinterpret_cast<const uint4*>(c.kc + at.code);
      else if (part <= 4) kept[i].v[part - 1] = *reinterpret_cast<const uint32_t*>(c.vc + at.code);
      else scales[i][part - 5] = (value ? c.vs : c.ks)[at.scale];
    }
  }
  __syncthreads();
  for (int i = threadIdx.x / kKeepParts; i < m; i += kKeepThreads / kKeepParts) {
    if (part == 7 || to[i] < 0) continue;
    const At at = place(c, to[i], h, e, value);
    if (part == 0) *reinterpret_cast<uint4*>(c.kc + at.code) = *reinterpret_cast<const uint4*>(kept[i].k);
    else if (part <= 4) *reinterpret_cast<uint32_t*>(c.vc + at.code) = kept[i].v[part - 1];
    else (value ? c.vs : c.ks)[at.scale] = scales[i][part - 5];
  }
}

}  // namespace

bool append_fits(const KvCache& c, const RotaryParams& r) {
  RotaryParams one = r;
  if (r.heads[0]) set_threads<1>(&one);
  const int64_t q = query_threads(one);
  return q <= kMostQuery && 2 * groups_of(work_of(c, r.T), r.T) + (q + kThreads - 1) / kThreads <= max_groups(kThreads);
}

hipError_t launch_kv_append(const KvCache& c, const RotaryParams& r, const void* v, int64_t ldv, const int64_t* slots,
                            int dtype, hipStream_t s) {
  Append p{c, work_of(c, r.T), r, v, ldv, slots, 0, 0};
  p.kv_groups = static_cast<uint32_t>(2 * groups_of(p.work, r.T));
  p.r.heads[1] = 0;                              // (the keys' workgroups take them)
  return dtype == CTS_F32 ? append_typed<float>(p, s) : append_typed<bf16_t>(p, s);
}

bool keep_fits(const KvCache& c, int B) { return static_cast<int64_t>(B) * c.heads * (c.d >> 5) <= max_groups(kKeepThreads); }

hipError_t launch_kv_keep(const KvCache& c, int B, int max_pages, const int32_t* table, const int32_t* kv_len,
                          const int32_t* q_start, const int32_t* path, const int32_t* n_path, int max_path, hipStream_t s) {
  kv_keep_kernel<<<static_cast<uint32_t>(B) * c.heads * (c.d >> 5), kKeepThreads, 0, s>>>(c, max_pages, table, kv_len, q_start,
                                                                                      path, n_path, max_path);
  return hipGetLastError();
}

}  // namespace cts
