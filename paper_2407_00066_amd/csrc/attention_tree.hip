// Attention of drafted tokens (cts_kv_tree_attention): a sequence's last n cached tokens are
// drafts, its query rows; all see the tokens before the drafts, and of the drafts
// those that their mask names.  The same one-pass softmax and the same transposed products as
// attention.hip, on 16 x 16 tiles (the lanes' parts of them are described there), a row
// being query x head of one key/value head's group.
//
// A workgroup takes RG groups of 16 rows of a sequence for one head: each step of 32 tokens is
// loaded and converted once for all of them.  Its waves take the steps in turn and join in
// shared memory.  Masks stand there too, a query's bits between a word of ones and one of
// zeros: what lies before the drafts is seen, what lies behind them is not, and 32 tokens' bits
// are one shift wherever the drafts begin.
//
// In bf16 a weight is rounded to bf16 for the product with the values, and a row's length is the sum of the
// rounded ones: one matrix instruction instead of the two or three that more parts of it would take, for an
// error (2-norm) of 0.0021 to 0.0023 where the output's own rounding alone is 0.0017.
//
// 32 + 8 heads of 128 in bf16: 200 requests of 30 to 2000 tokens with 1 to 6 drafts 59.5 us, 3.8 TB/s of codes and
// scales; 64, 31 and 50 drafts after 65 472, 39 970 and 131 022 tokens 228 us, 861 TFLOP/s, bound by vector
// instructions beside the matrix instructions: a step of 64 rows is 64 products (1024 cycles) and 267 others
// (2300 cycles in all with two waves a SIMD, as the waves time it).  16 rows a walk, which convert the codes four
// times as often: 427 us.  One tree of 7 over 709 tokens: 8.5 us, the chain of lengths, pages, codes and the
// waves' join.
#include <algorithm>

#include "attention_common.h"
#include "ldsdma.h"

namespace cts {
namespace {

constexpr int kMaskWords = kTreeMaxQ / 32 + 2;     // of a query, in shared memory

struct TreeTile {
  int b, q0, drafts, rows, row0;   // the sequence, its first query row, the drafts that count, its rows, the tile's first
  int past;                        // position of the first draft
  int lo, hi;                      // tokens that are walked, [lo, hi); lo a multiple of a step
  int steps;                       // of kUnit tokens (one where there are none); 0: no such rows
};

__device__ __forceinline__ TreeTile tree_tile(const TreeParams& p, int b, int sub) {
  TreeTile t;
  const Queries q = queries_of(p, b);
  const int len = min(max(p.kv_len[b], 0), p.max_kv);
  t.b = b;
  t.q0 = q.q0;
  t.drafts = min(q.n, p.max_q);
  t.rows = t.drafts * p.group;
  t.row0 = sub * p.tile_rows;
  t.past = len - q.n;
  t.hi = max(0, t.past + t.drafts);
  // (no row's position lies before the drafts)
  t.lo = p.window ? max(0, t.past - p.window + 1) & ~(kUnit - 1) : 0;
  t.steps = t.row0 < t.rows ? max(1, (t.hi - t.lo + kUnit - 1) / kUnit) : 0;
  return t;
}

__device__ __forceinline__ TreeTile uniform(TreeTile t) {
  return {__builtin_amdgcn_readfirstlane(t.b),    __builtin_amdgcn_readfirstlane(t.q0),
          __builtin_amdgcn_readfirstlane(t.drafts), __builtin_amdgcn_readfirstlane(t.rows),
          __builtin_amdgcn_readfirstlane(t.row0), __builtin_amdgcn_readfirstlane(t.past),
          __builtin_amdgcn_readfirstlane(t.lo),   __builtin_amdgcn_readfirstlane(t.hi),
          __builtin_amdgcn_readfirstlane(t.steps)};
}

__device__ __forceinline__ TreeTile of_lane(const TreeTile& t, int lane) {
  return {__builtin_amdgcn_readlane(t.b, lane),      __builtin_amdgcn_readlane(t.q0, lane),
          __builtin_amdgcn_readlane(t.drafts, lane), __builtin_amdgcn_readlane(t.rows, lane),
          __builtin_amdgcn_readlane(t.row0, lane),   __builtin_amdgcn_readlane(t.past, lane),
          __builtin_amdgcn_readlane(t.lo, lane),     __builtin_amdgcn_readlane(t.hi, lane),
          __builtin_amdgcn_readlane(t.steps, lane)};
}

// Kinds of instructions to the scheduler.
constexpr int kValu = 0x2, kMatrix = 0x8, kLdsRead = 0x100;

// The maximum of a row that has seen nothing: finite, so that no step asks whether there is one (scores below it weigh
// nothing).
constexpr float kNoMax = -3.0e38f;

// What a wave holds of 16 rows (attention.hip).
template <int D> struct Sums {
  static constexpr int NC = D > 128 ? 2 : 1;
  static constexpr int NB = D == 64 ? 4 : 8;
  f32x4 o[NC][NB];
  float m, l;
  static __device__ __forceinline__ int element(int g, int c, int i) {
    const int r = 4 * g + i;
    return D == 64 ? 8 * (r & 7) + 4 * (r >> 3) : 8 * (r + 16 * c);
  }
};

// Groups of 16 rows that a workgroup can take: what registers hold.
constexpr int most_groups(int d, bool f32) { return d == 256 ? (f32 ? 1 : 2) : f32 ? 2 : 4; }

// Parts of a query or weight in bf16, 16-byte pieces of its rows' queries that a lane multiplies, and whether
// they stay in shared memory: more than 6 of them a lane leave too little room for the sums.
template <int D, typename TQ, int RG> struct Query {
  static constexpr int NS = sizeof(TQ) == 4 ? 3 : 1, KS = D / 32, N = RG * KS * NS;
  static constexpr bool kShared = N > 6;
};

// A step's codes and scales, loaded straight into shared memory where the lane that loads
// 16 bytes is, as a rule, the one that converts them: a wave's own, SLOTS steps
// under way, no registers held and no barrier.
template <int D> struct Step {
  static constexpr int kPieces = D == 64 ? 1 : D / 64;       // loads of 16 bytes a lane for the keys, as many for the values
  static constexpr int kScales = D == 256 ? 2 : 1;           // loads of 4 bytes a lane for the scales
  static constexpr int kLoads = 2 * kPieces + kScales;
  static constexpr int kBytes = 2 * kPieces * 1024 + kScales * 256;
  // (three: 200 small trees 63 -> 72 us, 64 x 8 drafts after 4000 tokens 68 -> 76; four: one workgroup a compute
  // unit, 239 -> 370 over long documents)
  static constexpr int kSlots = 2;
};

// Shared memory.  Queries and masks stand in arrays of their own: the compiler waits for all loads
// under way before it reads from the array that they go to, and not before others.
template <int D, int WAVES> union Codes {
  char ring[WAVES][Step<D>::kSlots][Step<D>::kBytes];
  struct {
    float sums[WAVES][kRowTile][D + 4];
    float2 ml[WAVES][4 * kRowTile];
  } done;
};

__device__ __forceinline__ uint32_t lds_at(const void* p) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) void*)p));
}
// Each lane's 16 or 4 bytes at `base` (the same for the whole wave) + off, to lds + 16 or 4 x lane.
__device__ __forceinline__ void load_lds16(const uint8_t* base, uint32_t off, char* lds) {
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_global_load_lds((__attribute__((address_space(1))) void*)(base + off),
                                   (__attribute__((address_space(3))) void*)lds, 16, 0, 0);
#endif
}
__device__ __forceinline__ void load_lds4(const uint8_t* at, char* lds) {
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_global_load_lds((__attribute__((address_space(1))) void*)at,
                                   (__attribute__((address_space(3))) void*)lds, 4, 0, 0);
#endif
}

// The bytes of w that are past 252, as their highest bits.
__device__ __forceinline__ uint32_t over_252(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x03030303u) & w & 0x80808080u; }

// A step's keys and their scales of both groups of 16 tokens, from shared memory: reads and their wait in
// one piece of assembly (as plain reads they would wait for the next step's loads too).
// at: the step; k: KS words of each group, ks: scales of the lane's elements.
template <int D> __device__ __forceinline__ void read_keys(uint32_t at, int lane, uint32_t (*k)[D / 32], uint32_t* ks) {
#if defined(__HIP_DEVICE_COMPILE__)
  const int n = lane & 15, g = lane >> 4;
  if constexpr (D == 64) {
    uint64_t a, b;
    asm volatile("ds_read_b64 %0, %4\n\tds_read_b64 %1, %4 offset:512\n\tds_read_u8 %2, %5 offset:2048\n\t"
                 "ds_read_u8 %3, %5 offset:2080\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(a), "=&v"(b), "=&v"(ks[0]), "=&v"(ks[1]) : "v"(at + n * 32 + g * 8), "v"(at + n * 2 + (g >> 1)) : "memory");
    k[0][0] = static_cast<uint32_t>(a); k[0][1] = static_cast<uint32_t>(a >> 32);
    k[1][0] = static_cast<uint32_t>(b); k[1][1] = static_cast<uint32_t>(b >> 32);
  } else if constexpr (D == 128) {
    u32x4 a, b;
    asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %4 offset:1024\n\tds_read_u8 %2, %5 offset:4096\n\t"
                 "ds_read_u8 %3, %5 offset:4160\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(a), "=&v"(b), "=&v"(ks[0]), "=&v"(ks[1]) : "v"(at + lane * 16), "v"(at + n * 4 + g) : "memory");
#pragma unroll
    for (int i = 0; i < 4; ++i) { k[0][i] = a[i]; k[1][i] = b[i]; }
  } else {
    u32x4 a, b, c, d;
    asm volatile("ds_read_b128 %0, %6\n\tds_read_b128 %1, %6 offset:1024\n\tds_read_b128 %2, %6 offset:2048\n\t"
                 "ds_read_b128 %3, %6 offset:3072\n\tds_read_u16 %4, %7 offset:8192\n\tds_read_u16 %5, %7 offset:8320\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(a), "=&v"(b), "=&v"(c), "=&v"(d), "=&v"(ks[0]), "=&v"(ks[1])
                 : "v"(at + lane * 16), "v"(at + n * 8 + 2 * g) : "memory");
#pragma unroll
    for (int i = 0; i < 4; ++i) { k[0][i] = a[i]; k[0][4 + i] = b[i]; k[1][i] = c[i]; k[1][4 + i] = d[i]; }
  }
#endif
}

// The step's values: v, 8 elements of 4 tokens a piece, and their tokens' scales.
template <int D> __device__ __forceinline__ void read_values(uint32_t at, int lane, uint32_t (*v)[D > 128 ? 2 : 1][4],
                                                             uint32_t (*vs)[D > 128 ? 2 : 1]) {
#if defined(__HIP_DEVICE_COMPILE__)
  const int n = lane & 15, g = lane >> 4;
  if constexpr (D <= 128) {
    // (heads of 64: lanes n and n + 8 read the same piece)
    constexpr int kAt = D == 64 ? 1024 : 2048, kStep = D == 64 ? 512 : 1024, kScale = D == 64 ? 2048 + 64 : 4096 + 128;
    const uint32_t from = at + (D == 64 ? (g * 8 + (n & 7)) * 16 : lane * 16);
    const uint32_t scale = at + (D == 64 ? (g * 2 + ((n & 7) >> 2)) * 4 : (g * 4 + (n >> 2)) * 4);
    u32x4 a, b;
    asm volatile("ds_read_b128 %0, %4 offset:%6\n\tds_read_b128 %1, %4 offset:%7\n\tds_read_b32 %2, %5 offset:%8\n\t"
                 "ds_read_b32 %3, %5 offset:%9\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(a), "=&v"(b), "=&v"(vs[0][0]), "=&v"(vs[1][0])
                 : "v"(from), "v"(scale), "n"(kAt), "n"(kAt + kStep), "n"(kScale), "n"(kScale + D / 2) : "memory");
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[0][0][i] = a[i]; v[1][0][i] = b[i]; }
  } else {
    u32x4 a, b, c, d;
    asm volatile("ds_read_b128 %0, %8 offset:4096\n\tds_read_b128 %1, %8 offset:5120\n\tds_read_b128 %2, %8 offset:6144\n\t"
                 "ds_read_b128 %3, %8 offset:7168\n\tds_read_b32 %4, %9 offset:8448\n\tds_read_b32 %5, %9 offset:8464\n\t"
                 "ds_read_b32 %6, %9 offset:8576\n\tds_read_b32 %7, %9 offset:8592\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(a), "=&v"(b), "=&v"(c), "=&v"(d), "=&v"(vs[0][0]), "=&v"(vs[0][1]), "=&v"(vs[1][0]), "=&v"(vs[1][1])
                 : "v"(at + lane * 16), "v"(at + (g * 8 + (n >> 2)) * 4) : "memory");
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[0][0][i] = a[i]; v[0][1][i] = b[i]; v[1][0][i] = c[i]; v[1][1][i] = d[i]; }
  }
#endif
}

// Page number of the lane's group of 16 tokens in the steps s0, s0 + stride, ..: two
// groups a step, a lane one.
__device__ __forceinline__ int look_up(const TreeParams& p, int b, int lo, int s0, int stride) {
  const int lane = threadIdx.x & 63;
  const int64_t tok = lo + static_cast<int64_t>(s0 + (lane >> 1) * stride) * kUnit + 16 * (lane & 1);
  return p.table[static_cast<int64_t>(b) * p.max_pages + min(tok >> p.c.page_shift, static_cast<int64_t>(p.max_pages - 1))];
}

// Word w of the mask of the tile's query q as it is loaded (from the last draft's words on: the last one that counts),
// and as it stands in shared memory: drafts that do not count are 0.
__device__ __forceinline__ uint32_t load_mask(const TreeParams& p, const TreeTile& t, int first, int q, int w) {
  return p.mask[static_cast<int64_t>(t.q0 + first + q) * p.mask_words + min(max(w, 0), (t.drafts - 1) >> 5)];
}
__device__ __forceinline__ uint32_t mask_word(const TreeTile& t, int w, uint32_t bits) {
  const int left = t.drafts - 32 * w;
  return w < 0 ? ~0u : left <= 0 ? 0u : left < 32 ? bits & ((1u << left) - 1) : bits;
}

// 32 bytes from `at` and from 1, 2 and 3 times STRIDE further on, added element by element to f (in one piece with
// their wait: plain reads would wait for the stores under way).
template <int STRIDE> __device__ __forceinline__ void add_four(uint32_t at, float* f) {
#if defined(__HIP_DEVICE_COMPILE__)
  f32x4 v[8];
  asm volatile("ds_read_b128 %0, %8\n\tds_read_b128 %1, %8 offset:16\n\tds_read_b128 %2, %8 offset:%9\n\t"
               "ds_read_b128 %3, %8 offset:%10\n\tds_read_b128 %4, %8 offset:%11\n\tds_read_b128 %5, %8 offset:%12\n\t"
               "ds_read_b128 %6, %8 offset:%13\n\tds_read_b128 %7, %8 offset:%14\n\ts_waitcnt lgkmcnt(0)"
               : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]), "=&v"(v[4]), "=&v"(v[5]), "=&v"(v[6]), "=&v"(v[7])
               : "v"(at), "n"(STRIDE), "n"(STRIDE + 16), "n"(2 * STRIDE), "n"(2 * STRIDE + 16), "n"(3 * STRIDE), "n"(3 * STRIDE + 16)
               : "memory");
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      f[i] += v[2 * w][i];
      f[4 + i] += v[2 * w + 1][i];
    }
#endif
}

// `count` of the tile's steps from s0, `stride` apart, for key/value head h, by
// wave `wave`; pages: look_up of the first 32.  The workgroup meets once, for masks and queries.
// SHARED: tiles may have more than 16 rows.
template <int D, typename TQ, int RG, int stride, bool SHARED>
__device__ __forceinline__ void attend(const TreeParams& p, const TreeTile& t, int h, int wave, int s0, int count, int pages,
                                       Codes<D, stride>& codes, bf16x8 (*queries)[64], uint32_t (*masks)[kMaskWords], int2* seers, Sums<D>* st) {
  using Q = Query<D, TQ, RG>;
  using S = Step<D>;
  constexpr int NS = Q::NS, KS = Q::KS;          // (KS: steps of the first product; words of keys a lane holds)
  constexpr int NC = Sums<D>::NC, NB = Sums<D>::NB;
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const bool any = count > 0 && t.hi > t.lo;

  // Of each group of 16 tokens a lane loads the 16 bytes that it converts: of keys token n,
  // elements (D / 4) g on; of values quad g, eighth n (+ 16).  Heads of 64 have half as many bytes:
  // a lane loads for both groups at once, and they are dealt out when they are read.
  uint32_t k_at[S::kPieces], v_at[S::kPieces];
  uint32_t s_at;
  if constexpr (D == 64) {
    k_at[0] = v_at[0] = (lane & 31) * 16;
    s_at = (lane & 7) * 4;
  } else {
#pragma unroll
    for (int c = 0; c < D / 128; ++c) {
      k_at[c] = n * (D / 2) + g * (D / 8) + 16 * c;
      v_at[c] = (g * (D / 8) + n + 16 * c) * 16;
    }
    s_at = (lane & (D / 8 - 1)) * 4;
  }
  char (*const ring)[S::kBytes] = codes.ring[wave];
  const int page_mask = (1 << p.c.page_shift) - 1;
  uint32_t bad = 0;                                // which groups of the last steps asked for lie outside the cache, two bits a step
  int slot_in = 0, slot = 0;
  auto ask = [&](int it) {                         // for step `it`, of which `pages` has the pages
    int64_t base[2];
    bad <<= 2;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int page = __builtin_amdgcn_readlane(pages, 2 * (it & 31) + i);
      const int tok = t.lo + (s0 + it * stride) * kUnit + 16 * i;
      const bool outside = static_cast<uint32_t>(page) >= static_cast<uint32_t>(p.c.n_pages);
      bad |= outside ? 1u << i : 0u;
      base[i] = ((static_cast<int64_t>(outside ? 0 : page) * p.c.heads + h) << p.c.page_shift) + (tok & page_mask);
    }
    char* to = ring[slot_in];
    slot_in = slot_in + 1 == S::kSlots ? 0 : slot_in + 1;
    if constexpr (D == 64) {
      // (lanes 32 on: the second group)
      const int64_t from = lane < 32 ? base[0] : base[1];
      load_lds16(p.c.kc + from * 32, k_at[0], to);
      load_lds16(p.c.vc + from * 32, v_at[0], to + 1024);
      const int which = lane >> 3 & 3;             // (lanes 32 on load the same once more)
      const int64_t of = which & 1 ? base[1] : base[0];
      load_lds4((which & 2 ? p.c.vs : p.c.ks) + of * 2 + s_at, to + 2048);
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int c = 0; c < D / 128; ++c) {
          load_lds16(p.c.kc + base[i] * (D / 2), k_at[c], to);
          to += 1024;
        }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int c = 0; c < D / 128; ++c) {
          load_lds16(p.c.vc + base[i] * (D / 2), v_at[c], to);
          to += 1024;
        }
      if constexpr (D == 128) {
        const int which = lane >> 4;
        const int64_t of = which & 1 ? base[1] : base[0];
        load_lds4((which & 2 ? p.c.vs : p.c.ks) + of * 4 + s_at, to);
      } else {
        const int64_t of = lane & 32 ? base[1] : base[0];
        load_lds4(p.c.ks + of * 8 + s_at, to);
        load_lds4(p.c.vs + of * 8 + s_at, to + 256);
      }
    }
  };
  // All that is needed is asked for before any of it is waited for: the masks' first words, the queries, then the codes.
  const int q_first = p.by_group(t.row0), q_last = p.by_group(min(t.rows, t.row0 + RG * kRowTile) - 1);
  const int words = (q_last - q_first + 1) * kMaskWords;
  uint32_t word = 0;
  if (static_cast<int>(threadIdx.x) < words) word = load_mask(p, t, q_first, threadIdx.x / kMaskWords, static_cast<int>(threadIdx.x % kMaskWords) - 1);
  bf16x8 qf[Q::kShared ? 1 : RG][KS][NS];
  constexpr int kMine = Q::kShared ? (RG * KS + stride - 1) / stride : RG * KS;      // the waves share out what they share
  uint4 raw[kMine][sizeof(TQ) / 2];
  auto row_of = [&](int k) { return t.row0 + kRowTile * min((Q::kShared ? wave + k * stride : k) / KS, RG - 1) + n; };
#pragma unroll
  for (int k = 0; k < kMine; ++k) {
    const int s = (Q::kShared ? wave + k * stride : k) % KS;
    const int row = min(row_of(k), t.rows - 1), query = p.by_group(row);               // (rows that are not there: 0 later)
    const TQ* const q = static_cast<const TQ*>(p.q) + (t.q0 + query) * p.ldq +
                        static_cast<int64_t>(h * p.group + row - query * p.group) * D + (D / 4) * g + 8 * s;
#pragma unroll
    for (int e = 0; e < static_cast<int>(sizeof(TQ) / 2); ++e) raw[k][e] = reinterpret_cast<const uint4*>(q)[e];
  }
  // of row `lane`: its query's place among the tile's, and the first token before the drafts that it sees
  int2 seer = make_int2(0, 0);
  {
    const int row = min(t.row0 + lane, t.rows - 1), query = p.by_group(row);
    seer.x = query - q_first;
    if (p.window) seer.y = min(max(p.positions[t.q0 + query], t.past) - p.window + 1, t.past);
  }
  if (any)
#pragma unroll
    for (int i = 0; i < S::kSlots - 1; ++i) ask(min(i, count - 1));
  for (int k = threadIdx.x; k < words; k += 64 * stride) {
    if (k >= 64 * stride) word = load_mask(p, t, q_first, k / kMaskWords, k % kMaskWords - 1);
    masks[k / kMaskWords][k % kMaskWords] = mask_word(t, k % kMaskWords - 1, word);
  }
  if (threadIdx.x < RG * kRowTile) seers[threadIdx.x] = seer;           // (the first wave's)
#pragma unroll
  for (int k = 0; k < kMine; ++k) {
    if (row_of(k) >= t.rows)
#pragma unroll
      for (int e = 0; e < static_cast<int>(sizeof(TQ) / 2); ++e) raw[k][e] = make_uint4(0, 0, 0, 0);
    bf16x8 part[NS];
    if constexpr (NS == 1) part[0] = __builtin_bit_cast(bf16x8, raw[k][0]);
    else split<NS>(reinterpret_cast<const float*>(&raw[k][0]), part);
#pragma unroll
    for (int z = 0; z < NS; ++z) {
      if constexpr (Q::kShared) {
        if (wave + k * stride < RG * KS) queries[(wave + k * stride) * NS + z][lane] = part[z];
      } else {
        qf[k / KS][k % KS][z] = part[z];
      }
    }
  }
#pragma unroll
  for (int r = 0; r < RG; ++r) {
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < NB; ++e) st[r].o[c][e] = f32x4{0, 0, 0, 0};
    st[r].m = kNoMax;
    st[r].l = 0.0f;
  }
  // tokens from here on every row sees, as far as windows go
  int all_lo = 0;
  if (p.window) {
    all_lo = max(0, seer.y);
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) all_lo = max(all_lo, __shfl_xor(all_lo, x));
    all_lo = __builtin_amdgcn_readfirstlane(all_lo);
  }
  lds_barrier();                                                        // masks and queries are there
  if (!any) return;

  pages = rare(pages);                             // here: waited for inside the loop, the loads under way would be too
  const uint32_t ring_at = __builtin_amdgcn_readfirstlane(lds_at(ring));
  // Of two waves of a SIMD the older goes first, and the younger of two equal pieces ended a third later, alone for that
  // time: it goes first every other step (long documents: ends at 177 and 240 us, so at 221 and 232; always: 242 and 179).
  // (Not where every tile has 16 rows, for whose short steps it costs more than it gives: 8 x 16 drafts after 2000 tokens
  // 18.7 us, with it 19.5.)
  const bool younger = SHARED && p.cut && blockIdx.x >= 256;
  for (int it = 0; it < count; ++it) {
    if (younger) {
      if (it & 1) __builtin_amdgcn_s_setprio(1);
      else __builtin_amdgcn_s_setprio(0);
    }
    const int at = t.lo + (s0 + it * stride) * kUnit;
    // the next step's codes are asked for (past the end: the last step's again); this one's have to be there
    const int next = min(it + S::kSlots - 1, count - 1);
    if ((next & 31) == 0 && next != 0) pages = rare(look_up(p, t.b, t.lo, s0 + next * stride, stride));
    ask(next);
    wait_vmcnt<(S::kSlots - 1) * S::kLoads>();
    const uint32_t from = ring_at + slot * S::kBytes;
    slot = slot + 1 == S::kSlots ? 0 : slot + 1;
    const uint32_t bad_now = bad >> (2 * (S::kSlots - 1));

    // scores of the lane's rows against tokens at + 16 i + 4 g + j
    f32x4 x[RG][2];
    {
      uint32_t k[2][KS], ks[2];
      bf16x8 b[2][Q::kShared ? RG * NS : 1];         // the rows' pieces that are multiplied, and the next ones
      if constexpr (Q::kShared)
#pragma unroll
        for (int e = 0; e < RG * NS; ++e) b[0][e] = queries[(e / NS * KS) * NS + e % NS][lane];
      read_keys<D>(from, lane, k, ks);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (bad_now >> i & 1) ks[i] = ~0u;
#pragma unroll
        for (int r = 0; r < RG; ++r) x[r][i] = f32x4{0, 0, 0, 0};
      }
#pragma unroll
      for (int y = 0; y < KS; ++y) {
        if constexpr (Q::kShared)
          if (y + 1 < KS)
#pragma unroll
            for (int e = 0; e < RG * NS; ++e) b[(y + 1) & 1][e] = queries[(e / NS * KS + y + 1) * NS + e % NS][lane];
        bf16x8 a[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float unit = unit_of(ks[i], D == 256 ? y / 4 : 0);
          a[i] = frag(fp4_pair(k[i][y], unit, 0), fp4_pair(k[i][y], unit, 1), fp4_pair(k[i][y], unit, 2), fp4_pair(k[i][y], unit, 3));
        }
#pragma unroll
        for (int r = 0; r < RG; ++r)
#pragma unroll
          for (int z = 0; z < NS; ++z)
#pragma unroll
            for (int i = 0; i < 2; ++i) x[r][i] = mfma(a[i], Q::kShared ? b[y & 1][Q::kShared ? r * NS + z : 0] : qf[Q::kShared ? 0 : r][y][z], x[r][i]);
      }
      // The next keys are converted behind the products of these.
      if constexpr (RG >= 2) {
        __builtin_amdgcn_sched_group_barrier(kValu, 10, 0);
#pragma unroll
        for (int y = 0; y < KS; ++y) {
          if (Q::kShared && y + 1 < KS) __builtin_amdgcn_sched_group_barrier(kLdsRead, RG * NS, 0);
#pragma unroll
          for (int j = 0; j < 2 * RG * NS; ++j) {
            __builtin_amdgcn_sched_group_barrier(kMatrix, 1, 0);
            __builtin_amdgcn_sched_group_barrier(kValu, RG * NS >= 4 ? 1 : 2, 0);
          }
        }
      }
    }
    uint32_t v[2][NC][4], vs[2][NC];
    read_values<D>(from, lane, v, vs);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int c = 0; c < NC; ++c)
        if (bad_now >> i & 1) vs[i][c] = ~0u;

    const bool masked = at + kUnit > t.past || at < all_lo;              // the same for the whole wave
    // which of tokens at + 4 g .. a row sees (bit 16 i + j)
    auto seen_by = [&](int r) -> uint32_t {
      const int begin = rare(max(at - t.past, -kUnit));
      const int2 seer = seers[kRowTile * r + n];
      const uint32_t* const w = &masks[seer.x][(begin >> 5) + 1];
      uint32_t bits = static_cast<uint32_t>((static_cast<uint64_t>(w[1]) << 32 | w[0]) >> (begin & 31));
      const int hide = seer.y - at;                                      // tokens that a window hides
      if (hide > 0) bits &= hide < 32 ? ~0u << hide : 0u;
      return bits >> (4 * g);
    };
    if (masked) {
#pragma unroll
      for (int r = 0; r < RG; ++r) {
        const uint32_t bits = seen_by(r);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t keep = static_cast<uint32_t>(static_cast<int32_t>(bits << (31 - 16 * i - j)) >> 31);
            x[r][i][j] = __uint_as_float((__float_as_uint(x[r][i][j]) & keep) | (0xff800000u & ~keep));
          }
      }
    }
    // The maxima are looked at lane by lane, and across lanes only where one has grown past the slack.
    auto top_of = [&](int r) {
      float top = x[r][0][0];
#pragma unroll
      for (int i = 1; i < 8; ++i) top = fmaxf(top, x[r][i >> 2][i & 3]);
      return top * p.scale_log2e;
    };
    bool grown = false;
#pragma unroll
    for (int r = 0; r < RG; ++r) grown |= top_of(r) > st[r].m + kSlack;
    if (__any(grown)) {
#pragma unroll
      for (int r = 0; r < RG; ++r) {
        // (only the rows that have grown follow, so that no row's bits depend on another's)
        const float all = max_over_groups(top_of(r));
        const float m_new = all > st[r].m + kSlack ? all : st[r].m;
        const float fade = __builtin_amdgcn_exp2f(st[r].m - m_new);
        st[r].l *= fade;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int e = 0; e < NB; ++e) st[r].o[c][e] *= fade;
        st[r].m = m_new;
      }
    }
    bf16x8 pf[RG][NS];
#pragma unroll
    for (int r = 0; r < RG; ++r) {
      float w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        w[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r][i >> 2][i & 3], p.scale_log2e, -st[r].m));
        if (NS == 3) st[r].l += w[i];
      }
      split<NS>(w, pf[r]);
      if (NS == 1) {
        // (a row's length is the sum of its weights as they are rounded for the product)
        const uint4 y = __builtin_bit_cast(uint4, pf[r][0]);
        st[r].l = add_pair(y.x, add_pair(y.y, add_pair(y.z, add_pair(y.w, st[r].l))));
      }
    }

#pragma unroll
    for (int c = 0; c < NC; ++c) {
      if (masked) {
        // A weight of zero does not hide a NaN or infinite value: blocks that can hold one are
        // taken out of the product, and the rows that do see one are made NaN.
        if (__any((over_252(vs[0][c]) | over_252(vs[1][c])) != 0)) {
          uint32_t hit[4] = {0, 0, 0, 0};
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (past_scales(vs[i][c], j)) hit[2 * i + j / 2] |= 0x3f80u << (16 * (j & 1));
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (past_scales(vs[i][c], j)) {
                vs[i][c] ^= 0x80u << (8 * j);                            // 255 -> 127
                v[i][c][j] = 0;
              }
#pragma unroll
          for (int r = 0; r < RG; ++r) {
            const uint32_t bits = seen_by(r);
            float in[8];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
              for (int j = 0; j < 4; ++j) in[4 * i + j] = bits >> (16 * i + j) & 1 ? 1.0f : 0.0f;
            bf16x8 who[1];
            split<1>(in, who);
            const f32x4 count = mfma(frag(hit[0], hit[1], hit[2], hit[3]), who[0], f32x4{0, 0, 0, 0});
#pragma unroll
            for (int e = 0; e < NB; ++e)
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (count[i] > 0.0f) st[r].o[c][e][i] = NAN;
          }
        }
      }
#pragma unroll
      for (int e = 0; e < NB / 2; ++e) {
        uint32_t y[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            y[i][j] = fp4_pair(D == 64 ? v[i][c][j] >> (16 * (n >> 3)) : v[i][c][j], unit_of(vs[i][c], j), e);
        const bf16x8 even = frag(__builtin_amdgcn_perm(y[0][1], y[0][0], 0x05040100u), __builtin_amdgcn_perm(y[0][3], y[0][2], 0x05040100u),
                                 __builtin_amdgcn_perm(y[1][1], y[1][0], 0x05040100u), __builtin_amdgcn_perm(y[1][3], y[1][2], 0x05040100u));
        const bf16x8 odd = frag(__builtin_amdgcn_perm(y[0][1], y[0][0], 0x07060302u), __builtin_amdgcn_perm(y[0][3], y[0][2], 0x07060302u),
                                __builtin_amdgcn_perm(y[1][1], y[1][0], 0x07060302u), __builtin_amdgcn_perm(y[1][3], y[1][2], 0x07060302u));
#pragma unroll
        for (int r = 0; r < RG; ++r)
#pragma unroll
          for (int z = 0; z < NS; ++z) {
            st[r].o[c][2 * e] = mfma(even, pf[r][z], st[r].o[c][2 * e]);
            st[r].o[c][2 * e + 1] = mfma(odd, pf[r][z], st[r].o[c][2 * e + 1]);
          }
      }
      // (the same of values: 24 instructions for 2 RG products)
      if constexpr (RG >= 2) {
        __builtin_amdgcn_sched_group_barrier(kValu, 28, 0);
#pragma unroll
        for (int j = 0; j < NB * RG * NS; ++j) {
          __builtin_amdgcn_sched_group_barrier(kMatrix, 1, 0);
          __builtin_amdgcn_sched_group_barrier(kValu, RG * NS >= 4 ? 3 : RG * NS == 3 ? 4 : 6, 0);
        }
      }
    }
  }
#pragma unroll
  for (int r = 0; r < RG; ++r) st[r].l = sum_over_groups(st[r].l);
  wait_vmcnt<0>();                                                      // the last loads, whatever they bring
}

// What a workgroup takes: some steps of a tile for one head, and where their sums go if that is not all of them.
struct Piece {
  TreeTile t;
  int h, begin, end, slot;
};

// Work is counted in units of about 150 cycles: a step takes 2 and one for every group of rows. Where bounds
// allow more of it than 31 bits count, a tile's units are taken 2^unit_shift at a time, rounded up.
__device__ __forceinline__ int unit_of(const TreeTile& t, int tile_rows) {
  return 2 + (min(t.rows - t.row0, tile_rows) + kRowTile - 1) / kRowTile;
}

__device__ __forceinline__ TreeTile tile_at(const TreeParams& p, int i) {
  const int b = p.subs == 1 ? i : i / p.subs;
  return tree_tile(p, b, i - b * p.subs);
}

// What comes before and after a piece's steps, in units.
constexpr int kAround = 100;

// Piece w of the batch; false: there are not so many.  Tiles are cut along their tokens into equal pieces.  With
// few tiles there are no more pieces than workgroups that run at a time, since a second round would take as
// long as the first; otherwise a piece is at most a workgroup's share of the work, and what more pieces
// would take.  Up to 64 tiles (of a head) are taken by the length of their pieces, to an eighth: the
// longest first, one to a compute unit, then the shortest beside them, then the others as workgroups end.
__device__ __forceinline__ bool find_piece(const TreeParams& p, int w, Piece* out) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, tiles = p.B * p.subs;
  int4* const info = reinterpret_cast<int4*>(p.info);
  auto units_of = [&](const TreeTile& t) { return (t.steps * unit_of(t, p.tile_rows) + (1 << p.unit_shift) - 1) >> p.unit_shift; };
  TreeTile t0{};                                     // the first 64 are kept
  int total = 0, some = 0;                           // units, tiles that have any
  for (int base = 0; base < tiles; base += 64) {
    const int i = base + lane;
    TreeTile t{};
    if (i < tiles) t = tile_at(p, i);
    if (i < tiles && t.steps == 0 && i % static_cast<int>(gridDim.x) == w && wave == 0)
      for (int h = 0; h < p.c.heads; ++h) info[static_cast<int64_t>(i) * p.c.heads + h] = make_int4(0, 0, 0, 0);
    if (base == 0) t0 = t;
    total += __builtin_amdgcn_readlane(wave_scan(units_of(t)), 63);
    some += __builtin_popcountll(__ballot(t.steps > 0));
  }
  total *= p.c.heads;
  some *= p.c.heads;
  if (total == 0) return false;
  const bool few = some <= (tiles <= 64 ? p.resident : p.resident / 2);
  int len;
  if (few) len = (total - 1) / (p.resident - (tiles <= 64 ? some / 2 : some)) + 1;
  else len = total / p.resident + total / p.resident / 8 + (some * (kAround * 5 / 8) / p.resident >> p.unit_shift);
  len = max(len, p.least);
  auto pieces_of = [&](const TreeTile& t) {
    const int units = units_of(t);
    return units <= len ? (units > 0 ? 1 : 0) : static_cast<int>(static_cast<float>(units) * __builtin_amdgcn_rcpf(static_cast<float>(len))) + 1;
  };
  int at = 0, base = 0, of = 0, mine = 0;            // the tile, and the piece's number among its heads' pieces
  TreeTile t = t0;
  if (tiles <= 64) {
    int n;
    for (;; len += len / 8) {
      mine = pieces_of(t);
      n = __builtin_amdgcn_readlane(wave_scan(mine), 63) * p.c.heads;
      if (!few || n <= p.resident) break;
    }
    if (w >= n) return false;
    const int beside = p.resident - 256;             // (workgroups that have a place beside another)
    of = w < 256 ? w : w < 256 + beside ? n - 1 - (w - 256) : w - beside;
    const int bucket = mine ? min(7, static_cast<int>(static_cast<float>(units_of(t)) *
                                                      __builtin_amdgcn_rcpf(static_cast<float>(mine * len)) * 8.0f)) : -1;
    int before = 0;                                  // pieces that come first
#pragma unroll
    for (int k = 7, all = 0; k >= 0; --k) {
      const int v = bucket == k ? mine : 0, to = wave_scan(v);
      if (bucket == k) before = all + to - v;
      all += __builtin_amdgcn_readlane(to, 63);
    }
    at = __builtin_ctzll(__ballot(before * p.c.heads <= of && of < (before + mine) * p.c.heads));
    out->slot = of;
    of -= __builtin_amdgcn_readlane(before, at) * p.c.heads;
  } else {
    uint64_t here = 0;
    for (int before = 0; base < tiles; base += 64) {
      if (base) {
        t = TreeTile{};
        if (base + lane < tiles) t = tile_at(p, base + lane);
      }
      mine = pieces_of(t);
      const int n = mine * p.c.heads, to = wave_scan(n);
      here = __ballot(before + to > w);
      if (here) {
        at = __builtin_ctzll(here);
        of = w - before - __builtin_amdgcn_readlane(to - n, at);
        break;
      }
      before += __builtin_amdgcn_readlane(to, 63);
    }
    if (!here) return false;
    out->slot = w;
  }
  out->t = of_lane(t, at);
  mine = __builtin_amdgcn_readlane(mine, at);
  out->h = mine == 1 ? of : of / mine;
  // (a multiple of its waves' number: they end together)
  const int piece = of - out->h * mine;
  const int each = mine == 1 ? out->t.steps : ((out->t.steps - 1) / mine + p.waves) & -p.waves;
  out->begin = piece * each;
  out->end = min(out->t.steps, out->begin + each);
  if (piece == 0 && threadIdx.x == 0)
    info[static_cast<int64_t>(base + at) * p.c.heads + out->h] =
        make_int4((out->t.steps - 1) / each + 1, out->slot, out->t.q0,
                  out->t.row0 << 8 | min(p.tile_rows, out->t.rows - out->t.row0));
  return out->begin < out->end;                      // (equal pieces may be fewer)
}

// The tile (of a head) whose work is the rank-th most, to an eighth of the most there can be; of up to kOrdered tiles.
// With more workgroups than compute units the longest go first: they would end last.
constexpr int kOrdered = 256;
__device__ __forceinline__ TreeTile tile_of_rank(const TreeParams& p, int rank) {
  constexpr int kEach = kOrdered / 64;
  const int lane = threadIdx.x & 63, tiles = p.B * p.subs;
  const float scale = 8.0f / static_cast<float>(p.most_units);
  TreeTile t[kEach]{};
  int bucket[kEach];
#pragma unroll
  for (int c = 0; c < kEach; ++c)
    if (64 * c + lane < tiles) t[c] = tile_at(p, 64 * c + lane);
#pragma unroll
  for (int c = 0; c < kEach; ++c)
    bucket[c] = 64 * c + lane < tiles ? min(7, static_cast<int>(static_cast<float>(t[c].steps * unit_of(t[c], p.tile_rows)) * scale)) : -1;
  for (int k = 7; k >= 0; --k)
#pragma unroll
    for (int c = 0; c < kEach; ++c) {
      const uint64_t here = __ballot(bucket[c] == k);
      const int n = __builtin_popcountll(here);
      if (rank < n) {
        const int below = __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(here >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(here), 0));
        return of_lane(t[c], __builtin_ctzll(__ballot(bucket[c] == k && below == rank)));
      }
      rank -= n;
    }
  return TreeTile{};                                 // (every tile is in a bucket)
}

template <int D, typename TQ>
__device__ __forceinline__ TQ* out_at(const TreeParams& p, int q0, int h, int row) {
  const int query = p.by_group(row);
  return static_cast<TQ*>(p.out) + (q0 + query) * p.ldo + static_cast<int64_t>(h * p.group + row - query * p.group) * D;
}

// The steps of a piece for RG groups of rows, and what comes of them: results, or a cut tile's sums.
template <int D, typename TQ, int RG, int WAVES, bool SHARED>
__device__ __forceinline__ void take(const TreeParams& p, const Piece& me, int pages, Codes<D, WAVES>& codes,
                                     bf16x8 (*queries)[64], uint32_t (*masks)[kMaskWords], int2* seers) {
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const TreeTile& t = me.t;
  Sums<D> st[RG];
  const int first = me.begin + wave, count = first < me.end ? (me.end - first + WAVES - 1) / WAVES : 0;
  attend<D, TQ, RG, WAVES, SHARED>(p, t, me.h, wave, first, count, pages, codes, queries, masks, seers, st);
  // Each wave brings its sums to the maximum of all, and to their length where the result is whole; then
  // they only have to be added.
  const bool whole = me.end - me.begin == t.steps;
  lds_barrier();                                     // the codes are read
  if (g == 0)
#pragma unroll
    for (int r = 0; r < RG; ++r) codes.done.ml[wave][kRowTile * r + n] = make_float2(st[r].m, st[r].l);
  lds_barrier();
  float M[RG], L[RG];
#pragma unroll
  for (int r = 0; r < RG; ++r) {
    float2 ml[WAVES];
    M[r] = kNoMax;
    L[r] = 0.0f;
#pragma unroll
    for (int v = 0; v < WAVES; ++v) {
      ml[v] = codes.done.ml[v][kRowTile * r + n];
      M[r] = fmaxf(M[r], ml[v].x);
    }
#pragma unroll
    for (int v = 0; v < WAVES; ++v) L[r] += __builtin_amdgcn_exp2f(ml[v].x - M[r]) * ml[v].y;
    const float by = __builtin_amdgcn_exp2f(st[r].m - M[r]) * (!whole ? 1.0f : L[r] == 0.0f ? 0.0f : 1.0f / L[r]);
#pragma unroll
    for (int c = 0; c < Sums<D>::NC; ++c)
#pragma unroll
      for (int e = 0; e < Sums<D>::NB; ++e) st[r].o[c][e] *= by;
    if (!whole && wave == 0 && g == 0 && t.row0 + kRowTile * r + n < t.rows)
      *reinterpret_cast<float2*>(p.part_ml + 2 * (static_cast<int64_t>(me.slot) * p.tile_rows + kRowTile * r + n)) = make_float2(M[r], L[r]);
  }
#pragma unroll 1
  for (int r = 0; r < RG; ++r) {
    if (r) lds_barrier();                            // the last sums are read
#pragma unroll
    for (int x = 0; x < RG; ++x) {
      if (x != r) continue;
#pragma unroll
      for (int c = 0; c < Sums<D>::NC; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float f[Sums<D>::NB];
#pragma unroll
          for (int e = 0; e < Sums<D>::NB; ++e) f[e] = st[x].o[c][e][i];
          store_out<Sums<D>::NB>(codes.done.sums[wave][n] + Sums<D>::element(g, c, i), f);
        }
    }
    lds_barrier();
    const int row0 = t.row0 + kRowTile * r;
    for (int k = threadIdx.x; k < min(kRowTile, t.rows - row0) * (D / 8); k += 64 * WAVES) {
      const int at = k / (D / 8), e = (k % (D / 8)) * 8;
      float f[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      constexpr int kWave = sizeof(codes.done.sums[0]);
      const uint32_t from = lds_at(&codes.done.sums[0][at][e]);
#pragma unroll
      for (int v = 0; v < WAVES; v += 4) add_four<kWave>(from + v * kWave, f);
      if (whole) store_out<8>(out_at<D, TQ>(p, t.q0, me.h, row0 + at) + e, f);
      else store_out<8>(p.part + (static_cast<int64_t>(me.slot) * p.tile_rows + kRowTile * r + at) * D + e, f);
    }
  }
}

// Waves of a workgroup: eight where there are few, four, of which a compute unit takes more, where there are
// many; shared memory holds the codes of eight waves of heads of 256, and queries in 32 bits beside those of four.
// One tree over 709 tokens, eight waves or four: 8.8 / 9.5 us, eight in fp32 13.8 / 16.3; 200 small trees 93 / 63, 64
// uneven ones 60 / 57.
constexpr int waves_in(int d, int bytes, bool few) { return d == 256 ? (bytes == 4 ? 4 : 8) : few ? 8 : 4; }
// Waves of a SIMD that the registers are for.
constexpr int waves_of(int d, int bytes, int rg, int waves) {
  return d == 256 ? (bytes == 4 ? 1 : 2) : bytes == 4 ? 2 : rg == 1 ? 4 : rg == 2 && waves == 4 ? 3 : 2;
}

template <int D, typename TQ, int RG, int WAVES>
__global__ __launch_bounds__(64 * WAVES, waves_of(D, sizeof(TQ), RG, WAVES)) void tree_kernel(TreeParams p) {
  __shared__ __attribute__((aligned(16))) Codes<D, WAVES> codes;
  __shared__ __attribute__((aligned(16))) bf16x8 queries[Query<D, TQ, RG>::kShared ? Query<D, TQ, RG>::N : 1][64];
  __shared__ uint32_t masks[RG * kRowTile][kMaskWords];
  __shared__ int2 seers[RG * kRowTile];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), w = blockIdx.x;
  Piece me;
  int pages = 0;
  if (p.cut) {
    if (!find_piece(p, w, &me)) return;
    pages = look_up(p, me.t.b, me.t.lo, me.begin + wave, WAVES);
  } else {
    const int index = w / p.c.heads;
    me.h = w - index * p.c.heads;
    if (p.ordered) {
      me.t = tile_of_rank(p, index);
    } else {
      const int b = p.subs == 1 ? index : index / p.subs;
      // the first pages are on their way while the tile's length is
      if (!p.window) pages = look_up(p, b, 0, wave, WAVES);
      me.t = uniform(tree_tile(p, b, index - b * p.subs));
    }
    if (me.t.steps == 0) return;
    if (p.ordered || p.window) pages = look_up(p, me.t.b, me.t.lo, wave, WAVES);
    me.begin = me.slot = 0;
    me.end = me.t.steps;
  }
  // (groups of rows that the tile does not have are left out)
  const int rows = me.t.rows - me.t.row0;
  if (RG == 1 || rows <= kRowTile) {
    take<D, TQ, 1, WAVES, (RG > 1)>(p, me, pages, codes, queries, masks, seers);
  } else if constexpr (RG >= 2) {
    if (RG == 2 || rows <= 2 * kRowTile) {
      take<D, TQ, 2, WAVES, (RG > 1)>(p, me, pages, codes, queries, masks, seers);
    } else if constexpr (RG == 4) {
      if (rows <= 3 * kRowTile) take<D, TQ, 3, WAVES, (RG > 1)>(p, me, pages, codes, queries, masks, seers);
      else take<D, TQ, 4, WAVES, (RG > 1)>(p, me, pages, codes, queries, masks, seers);
    }
  }
}

// Joins the pieces of tile blockIdx.x (tile x head) for join_rows rows, in their order: kRows rows at a time, whose
// threads take eight elements of every kGroups-th piece.
template <int D, typename TQ>
__global__ __launch_bounds__(kJoinThreads) void tree_join_kernel(TreeParams p) {
  constexpr int kPer = D / 8, kRows = 4, kGroups = kJoinThreads / (kRows * kPer);
  __shared__ float4 part[kGroups][kRows][kPer][2];
  __shared__ float len[kGroups][kRows];
  const int4 info = reinterpret_cast<const int4*>(p.info)[blockIdx.x];
  const int n = info.x, rows = info.w & 255;
  if (n < 2) return;
  auto row_of = [&](int k, int r) { return static_cast<int64_t>(info.y + k) * p.tile_rows + r; };
  const int e = threadIdx.x % kPer, rr = threadIdx.x / kPer % kRows, group = threadIdx.x / (kPer * kRows);
  for (int r0 = blockIdx.y * p.join_rows; r0 < min(rows, static_cast<int>(blockIdx.y + 1) * p.join_rows); r0 += kRows) {
    const int r = r0 + rr;
    float L = 0.0f, f[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (r < rows) {
      float M = kNoMax;                              // (the row's threads look at a piece each)
      for (int k = e; k < n; k += kPer) M = fmaxf(M, p.part_ml[2 * row_of(k, r)]);
#pragma unroll
      for (int x = 1; x < kPer; x <<= 1) M = fmaxf(M, __shfl_xor(M, x));
#pragma unroll 4
      for (int k = group; k < n; k += kGroups) {
        const int64_t at = row_of(k, r);
        const float2 ml = *reinterpret_cast<const float2*>(p.part_ml + 2 * at);
        const float4* o = reinterpret_cast<const float4*>(p.part + at * D + 8 * e);
        const float4 x = o[0], y = o[1];
        const float a = __builtin_amdgcn_exp2f(ml.x - M);
        L += a * ml.y;
        f[0] += a * x.x; f[1] += a * x.y; f[2] += a * x.z; f[3] += a * x.w;
        f[4] += a * y.x; f[5] += a * y.y; f[6] += a * y.z; f[7] += a * y.w;
      }
    }
    part[group][rr][e][0] = make_float4(f[0], f[1], f[2], f[3]);
    part[group][rr][e][1] = make_float4(f[4], f[5], f[6], f[7]);
    if (e == 0) len[group][rr] = L;
    lds_barrier();
    if (group == 0 && r < rows) {
#pragma unroll
      for (int k = 1; k < kGroups; ++k) {
        L += len[k][rr];
        const float4 x = part[k][rr][e][0], y = part[k][rr][e][1];
        f[0] += x.x; f[1] += x.y; f[2] += x.z; f[3] += x.w;
        f[4] += y.x; f[5] += y.y; f[6] += y.z; f[7] += y.w;
      }
      const float inv = L == 0.0f ? 0.0f : 1.0f / L;
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] *= inv;
      store_out<8>(out_at<D, TQ>(p, info.z, blockIdx.x % p.c.heads, (info.w >> 8) + r) + 8 * e, f);
    }
    lds_barrier();
  }
}

template <int D, typename TQ, int RG> void launch_tiles(const TreeParams& p, hipStream_t s) {
  constexpr int kFew = waves_in(D, sizeof(TQ), true), kMany = waves_in(D, sizeof(TQ), false);
  if (p.waves == kMany) tree_kernel<D, TQ, RG, kMany><<<static_cast<uint32_t>(p.groups), 64 * kMany, 0, s>>>(p);
  else tree_kernel<D, TQ, RG, kFew><<<static_cast<uint32_t>(p.groups), 64 * kFew, 0, s>>>(p);
  if (p.cut)
    tree_join_kernel<D, TQ><<<dim3(static_cast<uint32_t>(p.B * p.subs * p.c.heads), p.tile_rows / p.join_rows), kJoinThreads, 0, s>>>(p);
}

// Steps of all tiles up to which tiles of fewer rows are taken (32 + 8 heads of 128, us with tiles of 64 rows / with this: 16
// sequences of 16 drafts after 2000 tokens 28.1 / 22.5, 200 drafts after 1500 25.9 / 17.8, 8 x 16 in fp32 28.3 / 23.6;
// above it rows have to share their steps: 64 x 8 after 900 20.9 / 24.0, 64 uneven trees 57 / 63, wide trees 58 / 75,
// long documents 239 / 427).
constexpr int64_t kLittleWork = 16384;

// Tiles (of a head) up to which they are cut: every piece is found by a look at all of them, so that finding them
// takes the square of their number.  6 drafts each after 500 tokens, after 50 to 4000, and after 500 with one sequence of
// 16 000, bounds of 16 384, 32 + 8 heads of 128, us cut / whole: 512 sequences 127 / 78, 200 / 158, 135 / 163; 1024 309 /
// 146, 384 / 251, 305 / 205; 2048 839 / 301, 990 / 490, 848 / 297; 8192 9800 / 1290, 9500 / 1840, 9760 / 1140; 4 + 1 heads,
// 1024 56 / 25, 76 / 61, 66 / 129; 2048 137 / 42, 169 / 89, 144 / 139; 4096 423 / 76, 440 / 142, 429 / 159.
constexpr int64_t kCutTiles = 2048;

template <int D, typename TQ> hipError_t launch(const TreeParams& p, hipStream_t s) {
  constexpr int kMost = most_groups(D, sizeof(TQ) == 4);
  switch (p.tile_rows / kRowTile) {
    case 1: launch_tiles<D, TQ, 1>(p, s); break;
    case 2: if constexpr (kMost >= 2) launch_tiles<D, TQ, 2>(p, s); break;
    default: if constexpr (kMost >= 4) launch_tiles<D, TQ, 4>(p, s); break;
  }
  return hipGetLastError();
}

}  // namespace

// The plan for tiles of `groups` groups of rows over `steps` steps at most; the workspace's bytes.
static size_t plan_groups(TreeParams* p, int groups, int64_t steps) {
  const int bytes_of = p->dtype == CTS_F32 ? 4 : 2;
  const int64_t rows = static_cast<int64_t>(p->max_q) * p->group;
  p->tile_rows = groups * kRowTile;
  p->subs = static_cast<int>((rows + p->tile_rows - 1) / p->tile_rows);
  const int64_t of_head = static_cast<int64_t>(p->B) * p->subs;
  // (more than a launch takes are refused if these tiles are chosen, and only need a workspace that does not fall)
  const int64_t tiles = std::min(of_head * p->c.heads, max_groups(64 * kWaves));
  // Cut and whole, us: 12 sequences of up to 6000 tokens for one head of 256 24.6 / 56, 8 wide trees 58 / 93, 64 drafts
  // after 8000 tokens 29 / 73, long documents 239 / 1013; with 512 tiles of up to 128 steps finding the pieces and joining
  // them costs more than uneven ends: 51.6 / 45.
  p->cut = steps > 64 && of_head <= kCutTiles && (tiles < 512 || steps > std::min<int64_t>(256, tiles / 4));
  // (64 trees after 40 to 4000 tokens: 64 us in the batch's order, so 57)
  p->ordered = !p->cut && tiles > 256 && of_head <= kOrdered;
  // (64 drafts after 8000 tokens, four rows of a tile a workgroup or 16: 29.4 / 32.3 us; 12 sequences with a head of 256
  // 24.6 / 28.7)
  p->join_rows = tiles <= 256 ? 4 : kRowTile;
  p->waves = waves_in(p->c.d, bytes_of, !p->cut && tiles < 256);
  p->resident = 256 * std::max(1, 4 * waves_of(p->c.d, bytes_of, groups, p->waves) / p->waves);
  const int64_t least = 8 * p->waves;                // (two steps a wave)
  p->most_units = static_cast<int>(steps) * (2 + groups);
  // few tiles are cut into p->resident pieces at most, others into as many more than they are
  auto pieces_of = [&](int64_t n) { return std::min(n + p->resident, n * (6 * steps / least + 2)); };
  p->groups = p->cut ? pieces_of(tiles) : tiles;
  // all tiles' units, each rounded up, stay below 2^31 (where some are not counted one by one there are
  // more tiles or longer ones than pieces_of's second bound is for; pieces of 8 and more keep to the first)
  p->unit_shift = 0;
  while ((tiles * steps * (2 + groups) >> p->unit_shift) + tiles > 0x50000000) ++p->unit_shift;
  p->least = static_cast<int>(std::max<int64_t>(8, least >> p->unit_shift));
  // (of more tiles than are cut, as for the most that are: a workspace serves every smaller batch)
  if (steps <= 64) return 16;
  const int64_t most = steps > 256 ? kCutTiles * p->c.heads : 4 * steps;
  const int64_t n = p->cut ? tiles : std::min<int64_t>(tiles, std::max<int64_t>(511, most));
  return static_cast<size_t>(pieces_of(n)) * p->tile_rows * (p->c.d + 2) * sizeof(float) + static_cast<size_t>(n) * 16 + 16;
}

bool plan_tree(TreeParams* p, size_t* bytes) {
  p->by_group = Divider(static_cast<uint32_t>(p->group));
  const int64_t rows = static_cast<int64_t>(p->max_q) * p->group;
  auto steps_of = [](int64_t span) { return std::max<int64_t>(1, (span + kUnit - 1) / kUnit); };
  const int64_t all_steps = steps_of(p->max_kv);
  int64_t steps = all_steps;
  if (p->window) steps = steps_of(std::min<int64_t>(p->max_kv, static_cast<int64_t>(p->window) + p->max_q + kUnit));
  // Rows share a walk over the tokens where there is work for every compute unit; where there is not, tiles of
  // fewer rows end sooner.
  const int most = most_groups(p->c.d, p->dtype == CTS_F32);
  int groups = 0;
  *bytes = 0;
  for (int g = 1; g <= most && (g == 1 || rows > g / 2 * kRowTile); g *= 2) {
    *bytes = std::max(*bytes, plan_groups(p, g, all_steps));         // (whichever is taken, with any window)
    const int64_t tiles = static_cast<int64_t>(p->B) * p->subs * p->c.heads;
    const bool little = tiles <= kLittleWork && tiles * steps <= kLittleWork;
    if (!groups && (little || rows <= p->tile_rows || 2 * g > most)) groups = g;
  }
  plan_groups(p, groups, steps);
  return static_cast<int64_t>(p->B) * p->subs * p->c.heads + p->resident <= max_groups(64 * kWaves);
}

void place_tree(TreeParams* p, void* workspace) {
  const size_t slots = static_cast<size_t>(p->groups) * p->tile_rows;
  p->part = static_cast<float*>(workspace);
  p->part_ml = p->part + slots * p->c.d;
  p->info = reinterpret_cast<int32_t*>(p->part_ml + slots * 2);
}

hipError_t launch_tree(const TreeParams& p, hipStream_t s) {
  const bool f32 = p.dtype == CTS_F32;
  switch (p.c.d) {
    case 64: return f32 ? launch<64, float>(p, s) : launch<64, bf16_t>(p, s);
    case 128: return f32 ? launch<128, float>(p, s) : launch<128, bf16_t>(p, s);
    default: return f32 ? launch<256, float>(p, s) : launch<256, bf16_t>(p, s);
  }
}

}  // namespace cts
