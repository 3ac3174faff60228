// Internal declarations of the decoder block's operators (cts_block.h): the
// cache, the attention over it, norms and rotary positions.
#pragma once

#include "cts.h"
#include "cts_internal.h"

namespace cts {

// n / d for n < 2^31 by a multiplication (a division by a number that only the
// launch knows takes the GPU tens of instructions, a 64-bit one over a hundred).
struct Divider {
  uint32_t d, mul, shift;
  Divider() = default;
  explicit Divider(uint32_t by) : d(by), mul(0), shift(0) {
    while ((1ull << shift) < by) ++shift;
    mul = static_cast<uint32_t>((((1ull << shift) - by) << 32) / by + 1);
  }
  __device__ __forceinline__ uint32_t operator()(uint32_t n) const { return (__umulhi(n, mul) + n) >> shift; }
};

// A launch has fewer than 2^32 threads along an axis: one with more runs what the low 32 bits
// count, and reports success.
constexpr int64_t max_groups(int threads) { return 0xffffffffll / threads; }

// 16 bytes.  NT: stored past the caches.  Outputs of kStreamBytes and more are: ordinary
// stores of that much hold up the loads beside them, and the next kernel loses
// nothing (norm of T x 4096, bf16, ordinary / NT, alone and with a matrix product of n
// after it: T = 256 4.4 / 4.1 us and 29.3 / 29.5, 1024 8.2 / 6.7 and 50 / 48, 4096
// 29 / 21 and 136 / 134, 16384 98 / 93 and 491 / 498).
template <bool NT> __device__ __forceinline__ void store16(void* p, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  typedef uint32_t word4 __attribute__((ext_vector_type(4)));
  const word4 v = {a, b, c, d};
  if constexpr (NT) __builtin_nontemporal_store(v, static_cast<word4*>(p));
  else *static_cast<word4*>(p) = v;
}
constexpr uint64_t kStreamBytes = uint64_t{4} << 20;

// The cache's arrays, and where a token's bytes lie in them.
struct KvCache {
  uint8_t *kc, *ks, *vc, *vs;
  int n_pages, page_shift, heads, d;
  __host__ __device__ int64_t slots() const { return static_cast<int64_t>(n_pages) << page_shift; }
};

// Whether one launch takes T tokens, a thread `elements` of them at a time (8, or what 16 bytes hold).
bool kv_fits(const KvCache& c, int T, int elements);
hipError_t launch_kv_write(const KvCache& c, int T, const void* k, int64_t ldk, const void* v, int64_t ldv,
                           const int64_t* slots, int dtype, hipStream_t s);
hipError_t launch_kv_read(const KvCache& c, int T, const int64_t* slots, void* k, int64_t ldk, void* v, int64_t ldv,
                          int dtype, hipStream_t s);

struct AttnParams {
  KvCache c;
  const void* q; int64_t ldq;
  void* out; int64_t ldo;
  const int32_t *table, *kv_len, *q_start;
  int T, B, heads, group;           // group: query heads of a key/value head
  int max_pages, max_q, max_kv, window, dtype;
  float scale_log2e;
  // the plan: 16-row tiles of a sequence with few rows, workgroups its steps are dealt
  // out to, rows of a tile that sums are kept for, tiles of the other sequences
  int subs, runs, part_rows;
  bool whole;                       // a workgroup takes a whole tile, not runs
  int64_t large_tiles;
  float *part, *part_ml;            // [2 runs][part_rows][d] sums, [2 runs][part_rows][2] maxima and lengths
  int32_t* info;                    // [tiles][kv heads][4] a tile's pieces, the first one's slot, its query row, first row and rows
  // prompts in bf16: workgroup tiles, pieces of a tile's tokens, and with more than one their
  // sums [tiles][kv heads][pieces][128][d], maxima and lengths [..][128][2]
  int64_t prompt_tiles;
  int pieces;
  float *prompt_part, *prompt_ml;
};

// Chooses the plan and gives the workspace's bytes (not falling with any size);
// false for a batch whose steps 31 bits do not count, or a launch has not the threads for.
bool plan_attention(AttnParams* p, size_t* bytes);
// Lays the workspace out for the plan.
void place_attention(AttnParams* p, void* workspace);
// The plan as cts_kv_attention_plan gives it.
void describe_attention(const AttnParams& p, int32_t* plan);
hipError_t launch_attention(const AttnParams& p, hipStream_t s);
// The bf16 sequences with many query rows (attention_tile.hip).
hipError_t launch_attention_prompts(const AttnParams& p, hipStream_t s);

// Attention of drafted tokens (attention_tree.hip): max_q is at most kTreeMaxQ; subs tiles of
// tile_rows rows (query x head of a key/value head's group) of a sequence.
constexpr int kTreeMaxQ = 512;
struct TreeParams : AttnParams {
  const uint32_t* mask; int64_t mask_words;     // [T][mask_words]
  const int32_t* positions;                     // of the rows, with a window
  int tile_rows;
  Divider by_group;
  // whether tiles are cut along their tokens; if not, whether those with most work go first; workgroups; how many run
  // at a time; units of work of a piece at least, of a tile at most, and 2^unit_shift of them that are counted as one; waves
  // of a workgroup; rows of a workgroup that joins
  bool cut, ordered;
  int64_t groups;
  int resident, least, most_units, unit_shift, waves, join_rows;
};
bool plan_tree(TreeParams* p, size_t* bytes);
void place_tree(TreeParams* p, void* workspace);
hipError_t launch_tree(const TreeParams& p, hipStream_t s);

struct NormParams {
  int T, d;
  const void *x, *y, *post, *gate, *weight;
  void *h, *n;
  int64_t ldx, ldy, ldg, ldh, ldn;
  float scale, eps;
};
constexpr int kNormMaxD = 32768;
hipError_t launch_block_norm(const NormParams& p, int dtype, hipStream_t s);

constexpr int kRotaryMaxAxes = 4;
struct RotaryParams {
  Divider per_head, per_token;      // threads of a head, of a token
  int T, heads[2], d, rot, n_pos, axes, interleaved;
  const void* in[2]; int64_t ldi[2];
  void* out[2]; int64_t ldo[2];
  const float *cos, *sin;
  const int32_t* pos;
  int end[kRotaryMaxAxes];          // pairs of the axes up to this one
};
hipError_t launch_rotary(const RotaryParams& p, int dtype, hipStream_t s);

// r: the queries [0] (none: 0 heads) and the keys [1], whose turned rows go to out[1] too, or nowhere.
// Whether one launch takes them.
bool append_fits(const KvCache& c, const RotaryParams& r);
hipError_t launch_kv_append(const KvCache& c, const RotaryParams& r, const void* v, int64_t ldv, const int64_t* slots,
                            int dtype, hipStream_t s);

constexpr int kKeepMaxPath = 512;   // accepted drafts of a sequence
bool keep_fits(const KvCache& c, int B);
hipError_t launch_kv_keep(const KvCache& c, int B, int max_pages, const int32_t* table, const int32_t* kv_len,
                          const int32_t* q_start, const int32_t* path, const int32_t* n_path, int max_path, hipStream_t s);

}  // namespace cts
