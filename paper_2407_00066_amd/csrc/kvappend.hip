// New tokens into the cache with their positions turned on the way (cts_kv_append), and the
// accepted ones of a step's drafts moved up behind their sequence (cts_kv_keep).
//
// Append is rotary and the cache's write in one launch, on the same formulas and with
// the same roundings: a key is turned in float, rounded to its type and then
// quantised.  Bound by memory like those two; a key is read once from memory
// instead of twice, and its turned row is not written.  Workgroups take keys, values or queries.
// A thread has 8 elements of a key: the 8 that they are turned with are another thread's, and
// read again from the nearest cache instead of exchanged, so that any rot will do.  8191 tokens of 32 + 8 heads of
// 128 in bf16: 39 us, 4.6 TB/s, where the caches hold none of them (rotary and write 33.8 + 9.7), 32 where they hold what
// fits; 33 tokens: 3.1 us (3.0 + 2.7), the chain of position, angles and rows.  (Calls in a graph.)
#include "kvblock.h"
#include "rows.h"

namespace cts {
namespace {

struct Append {
  KvCache c;
  Work work;                                     // of the values
  RotaryParams r;                                // [0] the queries, [1] the keys (out may be null)
  Divider per_token;                             // threads of a token's keys
  const void* v; int64_t ldv;
  const int64_t* slots;
  uint32_t key_groups, value_groups;             // workgroups of keys and of values; then come those of queries
  int key_threads, query_threads;
};

// f[8], eighth e of a key, turned; g: the eighth that it is turned with (halves).
template <int N> __device__ __forceinline__ void turn8(const RotaryParams& p, int e, const float* c, const float* s,
                                                       float* f, const float* g) {
  if constexpr (N == 4) {
#pragma unroll
    for (int j = 0; j < 4; ++j) turn(f[2 * j], f[2 * j + 1], c[j], s[j]);
  } else {
    const bool low = 8 * e < p.rot / 2;
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

// Thread i of the keys: eighth e of HEADS heads of a token, which share its angles.  A head's threads are
// neighbours in one wave, whose loads are all done before it stores: turned keys may be written over the keys.
template <typename T, int HEADS, bool NT> __device__ __forceinline__ void append_keys(const Append& p, int i) {
  const int per = p.c.d >> 3, shift = 31 - __builtin_clz(per), groups = (p.c.heads + HEADS - 1) / HEADS;
  const int64_t t = p.per_token(i);
  const int in_token = i - static_cast<int>(t) * p.per_token.d, group = in_token >> shift, e = in_token & (per - 1);
  const int64_t slot = p.slots[t];
  const int pos0 = p.r.pos[t];
  const T* const row = static_cast<const T*>(p.r.in[1]) + t * p.r.ldi[1];
  const int half = p.r.rot / 2, first = 8 * e;
  const bool turns = first < p.r.rot, pairs = turns && !p.r.interleaved;
  float f[HEADS][8], g[HEADS][8];
#pragma unroll
  for (int k = 0; k < HEADS; ++k) {
    const int head = min(group + k * groups, p.c.heads - 1);
    load8(row + head * p.c.d + first, f[k]);
    if (pairs) load8(row + head * p.c.d + (first < half ? first + half : first - half), g[k]);
  }
  if (turns) {
    float c[8] = {}, s[8] = {};
    if (p.r.interleaved) {
      angles<4>(p.r, t, pos0, first / 2, c, s);
#pragma unroll
      for (int k = 0; k < HEADS; ++k) turn8<4>(p.r, e, c, s, f[k], g[k]);
    } else {
      angles<8>(p.r, t, pos0, first < half ? first : first - half, c, s);
#pragma unroll
      for (int k = 0; k < HEADS; ++k) turn8<8>(p.r, e, c, s, f[k], g[k]);
    }
  }
#pragma unroll
  for (int k = 0; k < HEADS; ++k) {
    const int head = group + k * groups;
    if (head >= p.c.heads) continue;
    round8(static_cast<T*>(nullptr), f[k]);
    if (p.r.out[1]) {
      T* const o = static_cast<T*>(p.r.out[1]) + t * p.r.ldo[1] + head * p.c.d + first;
#pragma unroll
      for (int x = 0; x < 8; x += Elem<T>::N) put<T, Elem<T>::N, NT>(o + x, f[k] + x);
    }
    if (slot >= 0 && slot < p.c.slots()) store8(p.c, slot, head, e, false, f[k]);
  }
}

template <typename T, int HEADS, bool NT>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(Append p) {
  uint32_t w = blockIdx.x;
  if (w < p.key_groups) {
    const int i = static_cast<int>(w) * kThreads + threadIdx.x;
    if (i < p.key_threads) append_keys<T, HEADS, NT>(p, i);
    return;
  }
  w -= p.key_groups;
  if (w < p.value_groups) {
    write_rows<T>(p.c, p.work, p.r.T, w, static_cast<const T*>(p.v), p.ldv, p.slots, true);
    return;
  }
  const int i = static_cast<int>(w - p.value_groups) * kThreads + threadIdx.x;
  if (i < p.query_threads) turn_heads<T, HEADS, NT>(p.r, 0, i);
}

// Threads are counted in 31 bits.
constexpr int64_t kMostThreads = 0x7fffff00;
int64_t key_threads(const KvCache& c, int T, int heads) { return static_cast<int64_t>(T) * ((c.heads + heads - 1) / heads) * (c.d >> 3); }
int64_t query_threads(const RotaryParams& r) { return static_cast<int64_t>(r.T) * (r.heads[0] ? r.per_token.d : 0); }
int64_t groups_for(int64_t threads) { return (threads + kThreads - 1) / kThreads; }

template <typename T, int HEADS, bool NT> hipError_t append_launch(Append p, hipStream_t s) {
  if (p.r.heads[0]) set_threads<HEADS>(&p.r);
  p.query_threads = static_cast<int>(query_threads(p.r));
  p.key_threads = static_cast<int>(key_threads(p.c, p.r.T, HEADS));
  p.per_token = Divider(static_cast<uint32_t>(p.key_threads / p.r.T));
  p.key_groups = static_cast<uint32_t>(groups_for(p.key_threads));
  p.value_groups = static_cast<uint32_t>(groups_of(p.work, p.r.T));
  const uint32_t all = p.key_groups + p.value_groups + static_cast<uint32_t>(groups_for(p.query_threads));
  kv_append_kernel<T, HEADS, NT><<<all, kThreads, 0, s>>>(p);
  return hipGetLastError();
}

template <typename T> hipError_t append_typed(const Append& p, hipStream_t s) {
  // Two heads share their angles where that leaves workgroups enough, and large outputs are stored past the caches.
  // 32 + 8 heads of 128 in bf16, 1, 2 and 4 heads a thread with streaming stores: 200 tokens 3.4 / 4.0 / 5.2 us, 800 5.4 /
  // 5.7 / 7.0, 1600 9.2 / 8.2 / 9.1, 4000 18.2 / 18.5 / 18.6, 16 000 74.8 / 75.4 / 80.2 (with ordinary stores, 2 heads:
  // 1600 9.0, 4000 20.2, 16 000 78.3); 64 + 8 heads, 1600 13.1 / 11.9 / 12.5; 20 + 4 on three axes 9.4 / 8.2 / 8.4. In
  // fp32 a thread's 16-byte stores lie 32 or 64 bytes apart, which streaming stores do not gather, and one head's rows
  // are as long as two in bf16.  One head with ordinary stores, so, two with streaming ones: 1600 tokens of 32 + 8 heads
  // of 128 14.1 / 18.4 us, interleaved 17.3 / 34.3, 16 000 131 / 173 and 152 / 354, of 64 + 8 219 / 308, of 8 + 1 heads
  // of 64 15.1 / 20.9; of 20 + 4 on three axes, half of a head turned, 1600 12.1 / 13.3, 4000 28.0 / 27.4.
  if constexpr (sizeof(T) == 2) {
    const int64_t n = static_cast<int64_t>(p.r.T) * (p.r.heads[0] * (p.r.d / 16) + p.c.heads * (p.r.d / 8));
    if (n >= 512 * kThreads)
      return sizeof(T) * p.r.T * p.r.heads[0] * p.r.d < kStreamBytes ? append_launch<T, 2, false>(p, s) : append_launch<T, 2, true>(p, s);
  }
  return append_launch<T, 1, false>(p, s);
}

// ------------------------------------------------------------------- keep
// A workgroup takes one block of 32 elements of one head of a sequence: all of its accepted
// tokens are read before any is written, so that no order and no repetition of them matters.
// Codes and scales move as bytes, eight threads a token, without a barrier between heads.  64 sequences
// of up to 33 drafts, 8 heads of 128: 5.2 us, one sequence 3.6 (calls in a graph): launch and the chain of path, page and
// codes.
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
  const int64_t q = query_threads(one), k = key_threads(c, r.T, 1);
  return q <= kMostThreads && k <= kMostThreads &&
         groups_for(q) + groups_for(k) + groups_of(work_of(c, r.T), r.T) <= max_groups(kThreads);
}

hipError_t launch_kv_append(const KvCache& c, const RotaryParams& r, const void* v, int64_t ldv, const int64_t* slots,
                            int dtype, hipStream_t s) {
  Append p{};
  p.c = c; p.work = work_of(c, r.T); p.r = r; p.v = v; p.ldv = ldv; p.slots = slots;
  p.r.heads[1] = 0;                              // (their workgroups take them)
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
