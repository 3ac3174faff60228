// Attention over the 4-bit cache for sequences with many query rows (prompts and
// chunks of prompts), bf16: the same one-pass softmax and the same transposed
// products as attention.hip, on 32 x 32 tiles.
//
// A workgroup's waves take 32 query rows each (query x head of one key/value
// head's group, in that order) and walk the visible tokens together, 8192 / D of
// them a step.  A step's codes become bf16 once for the whole workgroup, in
// shared memory: keys as they lie, [token][element]; values turned, [element][token],
// their tokens in the order in which the first product's result leaves them in
// the lanes, so that the weights are the second product's operand as they stand.
// Rows are rotated in 16-byte pieces so that neither side meets a bank twice.
// One buffer is filled while the other is multiplied: a barrier a step.
//
// Four waves of 32 rows, two such workgroups on a compute unit: one's softmax runs beside
// the other's products.  Measured, prompts of 2048 (after 6144), 4096, 777 and 1301 tokens with
// 32 + 8 heads of 128: 436 us, 910 TFLOP/s, where a library's large product reaches 1400 (461 on a
// card where that reaches 1345); one of 4096 with heads of 64: 111 us, 618 TFLOP/s, 16 + 4 heads of
// 256: 294 us, 467 (one wave a SIMD).  A step's 248 vector instructions and 32 matrix
// instructions of a wave bound it together: the matrix pipe is busy for 40% of the time, and vector instructions
// beside it run at two thirds of their rate.  Eight waves with one conversion for all
// go in step at the barrier (525 us), also when the two halves take turns at vector work
// and products (492 us); 64 rows a wave move their accumulators (722 us).
//
// Lane l = 32 hh + n.  First product: A row = token n of 32, k = elements 16 s + 8 hh
// .. + 7 in step s; result: register i is token 8 (i / 4) + 4 hh + i % 4, column n =
// query row.  Second: A row = element n of 32, k = 8 hh + j for the tokens
// 8 (j / 4) + 4 hh + j % 4 of 16.
#include <algorithm>

#include "attention_common.h"
#include "ldsdma.h"

namespace cts {
namespace {

constexpr int kThreads = 256, kRows = kPromptRows;

typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

template <int D> struct Step {
  static constexpr int T = 8192 / D;               // tokens
  static constexpr int MB = T / 32;                // row blocks of the first product
  static constexpr int DB = D / 32;                // row blocks of the second; scale blocks
  static constexpr int KS = D / 16;                // k steps of the first
  static constexpr int KC = D / 8, VC = T / 8;     // 16-byte pieces of a row of keys, of values
  // Pieces of 32 rows in turn are read without meeting a bank twice (256 bytes wide).
  static __device__ __forceinline__ int key(int tok, int c) {
    return (tok * KC + (c ^ (KC == 8 ? (tok >> 1) & 7 : tok & 15))) * 16;
  }
  static __device__ __forceinline__ int value(int d, int c) {
    return (d * VC + (c ^ (VC == 4 ? (d >> 2) & 3 : VC == 8 ? (d >> 1) & 7 : d & 15))) * 16;
  }
};

// Tile `index` of the sequences with many rows: their number is known on the
// device only, so the lanes count.  False: there are not so many.
__device__ __forceinline__ bool find_tile(const AttnParams& p, int index, int* b, int* sub) {
  const int lane = threadIdx.x & 63;
  for (int base = 0, before = 0; base < p.B; base += 64) {
    int count = 0;
    if (base + lane < p.B) {
      const int rows = min(queries_of(p, base + lane).n, p.max_q) * p.group;
      count = rows > kSmallRows ? (rows + kRows - 1) / kRows : 0;
    }
    const int to = wave_scan(count);
    const uint64_t here = __ballot(before + to > index);
    if (here) {
      const int at = __builtin_ctzll(here);
      *b = base + at;
      // a sequence's last rows see most: they go first
      *sub = before + __builtin_amdgcn_readlane(to, at) - 1 - index;
      return true;
    }
    before += __builtin_amdgcn_readlane(to, 63);
  }
  return false;
}

template <int D> struct TileShared {
  char k[2][8192 * 2], v[2][8192 * 2];
  uint64_t nan[3][(Step<D>::T + 63) / 64][Step<D>::DB];                  // tokens whose value block is NaN
};

template <int D>
__global__ __launch_bounds__(kThreads, D == 256 ? 1 : 2) void attn_prompt_kernel(AttnParams p) {
  using S = Step<D>;
  __shared__ TileShared<D> sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, hh = lane >> 5;
  const int item = blockIdx.x / p.pieces, piece = blockIdx.x - item * p.pieces;
  const int h = item % p.c.heads;
  int b, sub;
  if (!find_tile(p, item / p.c.heads, &b, &sub)) return;
  const Queries q = queries_of(p, b);
  const int len = min(max(p.kv_len[b], 0), p.max_kv);
  const int rows = min(q.n, p.max_q) * p.group, first_pos = len - q.n;
  const int row0 = sub * kRows, row_end = min(rows, row0 + kRows);
  const int pos_lo = first_pos + row0 / p.group, pos_hi = first_pos + (row_end - 1) / p.group;
  const int hi = max(0, pos_hi + 1);
  const int lo = p.window ? max(0, pos_lo - p.window + 1) & ~(S::T - 1) : 0;
  const int all_steps = hi > lo ? (hi - lo + S::T - 1) / S::T : 0;
  const int begin = static_cast<int>(static_cast<int64_t>(all_steps) * piece / p.pieces);
  const int steps = static_cast<int>(static_cast<int64_t>(all_steps) * (piece + 1) / p.pieces);      // [begin, steps)

  // the lane's query row
  const int row = row0 + 32 * wave + n;
  const bool live = row < rows;
  const int query = row / p.group;
  const int pos = live ? first_pos + query : -1;
  const int first = p.window ? pos - p.window + 1 : 0;
  // tokens that all of the wave's live rows see
  const int w_row = row0 + 32 * wave, w_last = min(rows - 1, w_row + 31);
  const int all_hi = w_row < rows ? first_pos + w_row / p.group + 1 : 0x7fffffff;
  const int all_lo = p.window && w_row < rows ? first_pos + w_last / p.group - p.window + 1 : 0;

  bf16x8 qf[S::KS];
  {
    const bf16_t* src = static_cast<const bf16_t*>(p.q) +
                        (live ? (q.q0 + query) * p.ldq + static_cast<int64_t>(h * p.group + row - query * p.group) * D : 0);
#pragma unroll
    for (int s = 0; s < S::KS; ++s) {
      qf[s] = frag(0, 0, 0, 0);
      if (live) qf[s] = *reinterpret_cast<const bf16x8*>(src + 16 * s + 8 * hh);
    }
  }
  f32x16 o[S::DB];
#pragma unroll
  for (int d = 0; d < S::DB; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
  float m = -INFINITY, l = 0.0f;

  // What the thread converts, of one group of four tokens: 8 elements of their values,
  // and 32 of one's key.  Both lie in the same page.
  const int quad = tid % (S::T / 4), eighth = tid / (S::T / 4);
  // (which of the four tokens' keys: chosen so that neighbouring lanes write to different banks)
  const int turn = D == 128 ? (-(quad >> 2)) & 3 : D == 64 ? (quad >> 2) & 3 : 0;
  const int k_in = (eighth & 3) ^ turn, k_tok = 4 * quad + k_in, k_blk = eighth >> 2;
  const uint32_t page_mask = (1u << p.c.page_shift) - 1;
  const uint32_t page_codes = (D / 2) * p.c.heads << p.c.page_shift, head_codes = (D / 2) * h << p.c.page_shift;
  // (a token's scales lie at a sixteenth of its codes' offset)
  const uint8_t* const kc = p.c.kc + head_codes + (k_in * (D / 2) + k_blk * 16);
  const uint8_t* const ks = p.c.ks + head_codes / 16 + (k_in * S::DB + k_blk);
  const uint8_t* const vc = p.c.vc + head_codes + eighth * 16;
  const uint8_t* const vs = p.c.vs + head_codes / 16 + (eighth >> 2) * 4;
  const int32_t* const table = p.table + static_cast<int64_t>(b) * p.max_pages;
  int page = 0;
  uint4 k_raw, v_raw;
  uint32_t k_scale = 0, v_scale = 0;
  // past the last seen token its group stands in, masked
  auto group = [&](int step) { return min(lo + step * S::T + 4 * quad, (hi - 1) & ~3); };
  auto look_up = [&](int step) { page = table[group(step) >> p.c.page_shift]; };
  auto load = [&](int step) {
    const bool bad = static_cast<uint32_t>(page) >= static_cast<uint32_t>(p.c.n_pages);
    const uint64_t at = static_cast<uint64_t>(bad ? 0u : static_cast<uint32_t>(page)) * page_codes +
                        (group(step) & page_mask) * (D / 2);
    k_raw = *reinterpret_cast<const uint4*>(kc + at);
    k_scale = ks[at >> 4];
    v_raw = *reinterpret_cast<const uint4*>(vc + at);
    v_scale = *reinterpret_cast<const uint32_t*>(vs + (at >> 4));
    if (bad) {
      k_scale = 0xffu;
      v_scale = 0xffffffffu;
    }
  };
  // tokens of a step from here on, or before there, may be hidden from some row of the workgroup
  const int wg_all_hi = pos_lo + 1, wg_all_lo = p.window ? pos_hi - p.window + 1 : 0;
  auto convert = [&](int step) {
    char* const kb = sh.k[step & 1];
    char* const vb = sh.v[step & 1];
    {
      const uint32_t w[4] = {k_raw.x, k_raw.y, k_raw.z, k_raw.w};
      const float unit = unit_of(k_scale, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<bf16x8*>(kb + S::key(k_tok, 4 * k_blk + i)) =
            frag(fp4_pair(w[i], unit, 0), fp4_pair(w[i], unit, 1), fp4_pair(w[i], unit, 2), fp4_pair(w[i], unit, 3));
    }
    {
      uint32_t w[4] = {v_raw.x, v_raw.y, v_raw.z, v_raw.w};
      uint32_t scale = v_scale;
      const int at = lo + step * S::T;
      if (at + S::T > wg_all_hi || at < wg_all_lo) {
        // A weight of zero does not hide a NaN or an infinity: where rows may be masked, blocks
        // that can hold one are taken out and noted, and the rows that see them made NaN.
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (past_scales(scale, j)) {
            const int tok = 4 * quad + j;
            w[j] = 0;
            scale ^= 0x80u << (8 * j);                                   // 255 -> 127
            atomicOr(reinterpret_cast<unsigned long long*>(&sh.nan[step % 3][tok >> 6][eighth >> 2]), 1ull << (tok & 63));
          }
      }
      uint32_t y[4][4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float unit = unit_of(scale, j);
#pragma unroll
        for (int e = 0; e < 4; ++e) y[j][e] = fp4_pair(w[j], unit, e);
      }
      // four tokens of one element: half a piece
      const int piece = (quad >> 2) * 2 + (quad & 1), half = 8 * ((quad >> 1) & 1);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int d = 8 * eighth + 2 * e;
        *reinterpret_cast<uint2*>(vb + S::value(d, piece) + half) =
            make_uint2(__builtin_amdgcn_perm(y[1][e], y[0][e], 0x05040100u), __builtin_amdgcn_perm(y[3][e], y[2][e], 0x05040100u));
        *reinterpret_cast<uint2*>(vb + S::value(d + 1, piece) + half) =
            make_uint2(__builtin_amdgcn_perm(y[1][e], y[0][e], 0x07060302u), __builtin_amdgcn_perm(y[3][e], y[2][e], 0x07060302u));
      }
    }
  };
  auto clear = [&](int which) {
    for (int i = tid; i < static_cast<int>(sizeof(sh.nan[0]) / 8); i += kThreads) (&sh.nan[which][0][0])[i] = 0;
  };

  clear(0);
  clear(1);
  clear(2);
  __syncthreads();
  const int last = steps - 1;
  if (begin < steps) {
    look_up(begin);
    load(begin);
    look_up(min(begin + 1, last));
    convert(begin);
    load(min(begin + 1, last));
    look_up(min(begin + 2, last));
  }
  for (int step = begin; step < steps; ++step) {
    lds_barrier();
    const char* const kb = sh.k[step & 1];
    const char* const vb = sh.v[step & 1];
    const int at = lo + step * S::T;
    clear((step + 2) % 3);
    f32x16 s[S::MB];
#pragma unroll
    for (int mb = 0; mb < S::MB; ++mb)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[mb][i] = 0.0f;
#pragma unroll
    for (int k = 0; k < S::KS; ++k)
#pragma unroll
      for (int mb = 0; mb < S::MB; ++mb)
        s[mb] = mfma32(*reinterpret_cast<const bf16x8*>(kb + S::key(32 * mb + n, 2 * k + hh)), qf[k], s[mb]);
    const bool masked = at + S::T > all_hi || at < all_lo;               // the same for the whole wave
    if (masked) {
      // register i is token at + 4 hh + a constant
      const int from = rare(at + 4 * hh), below = pos - from, above = first - from;
#pragma unroll
      for (int mb = 0; mb < S::MB; ++mb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int tok = 32 * mb + 8 * (i >> 2) + (i & 3);
          if (tok > below || tok < above) s[mb][i] = -INFINITY;
        }
    }
    // (vector work for the time that the first product's last results take)
    if (step < last) {
      convert(step + 1);
      load(min(step + 2, last));
      look_up(min(step + 3, last));
    }
    float top = s[0][0];
#pragma unroll
    for (int mb = 0; mb < S::MB; ++mb)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, s[mb][i]);
    {
      const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
      top = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1])) * p.scale_log2e;
    }
    if (__any(top > m + kSlack)) {
      const float m_new = fmaxf(m, top), fade = __builtin_amdgcn_exp2f(m - (m_new == -INFINITY ? 0.0f : m_new));
      l *= fade;
#pragma unroll
      for (int d = 0; d < S::DB; ++d) o[d] *= fade;
      m = m_new;
    }
    const float base = m == -INFINITY ? 0.0f : m;
    bf16x8 pf[S::MB][2];
#pragma unroll
    for (int mb = 0; mb < S::MB; ++mb) {
      uint32_t w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[mb][2 * i], p.scale_log2e, -base));
        const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(s[mb][2 * i + 1], p.scale_log2e, -base));
        w[i] = f32_to_bf16_pair(x, y);
        l = add_pair(w[i], l);
      }
      pf[mb][0] = frag(w[0], w[1], w[2], w[3]);
      pf[mb][1] = frag(w[4], w[5], w[6], w[7]);
    }
#pragma unroll
    for (int mb = 0; mb < S::MB; ++mb)
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int d = 0; d < S::DB; ++d)
          o[d] = mfma32(*reinterpret_cast<const bf16x8*>(vb + S::value(32 * d + n, (mb * 2 + k) * 2 + hh)), pf[mb][k], o[d]);
    if (at + S::T > wg_all_hi || at < wg_all_lo) {
#pragma unroll
      for (int d = 0; d < S::DB; ++d)
        for (int x = 0; x < (S::T + 63) / 64; ++x)
          for (uint64_t hit = sh.nan[step % 3][x][d]; hit; hit &= hit - 1) {
            const int tok = at + 64 * x + __builtin_ctzll(hit);
            if (tok <= pos && tok >= first)
#pragma unroll
              for (int i = 0; i < 16; ++i) o[d][i] = NAN;
          }
    }
  }
  {
    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    l = __uint_as_float(x[0]) + __uint_as_float(x[1]);
  }
  if (!live) return;
  if (p.pieces == 1) {
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    bf16_t* const out = static_cast<bf16_t*>(p.out) + (q.q0 + query) * p.ldo +
                        static_cast<int64_t>(h * p.group + row - query * p.group) * D;
#pragma unroll
    for (int d = 0; d < S::DB; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const float f[4] = {o[d][i] * inv, o[d][i + 1] * inv, o[d][i + 2] * inv, o[d][i + 3] * inv};
        store_out<4>(out + 32 * d + 2 * i + 4 * hh, f);
      }
  } else {
    const int64_t at = static_cast<int64_t>(blockIdx.x) * kRows + 32 * wave + n;
    float* const out = p.prompt_part + at * D;
#pragma unroll
    for (int d = 0; d < S::DB; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const float f[4] = {o[d][i], o[d][i + 1], o[d][i + 2], o[d][i + 3]};
        store_out<4>(out + 32 * d + 2 * i + 4 * hh, f);
      }
    if (hh == 0) *reinterpret_cast<float2*>(p.prompt_ml + 2 * at) = make_float2(m, l);
  }
}

// Joins the pieces of tile blockIdx.x (tile x head), in their order: a thread takes
// eight elements of one row.
template <int D>
__global__ __launch_bounds__(kThreads) void attn_prompt_join_kernel(AttnParams p) {
  constexpr int kPer = kThreads / (D / 8);           // rows of a workgroup
  const int h = blockIdx.x % p.c.heads;
  int b, sub;
  if (!find_tile(p, blockIdx.x / p.c.heads, &b, &sub)) return;
  const Queries q = queries_of(p, b);
  const int r = blockIdx.y * kPer + threadIdx.x / (D / 8), e = threadIdx.x % (D / 8) * 8;
  const int row = sub * kRows + r, query = row / p.group;
  if (row >= min(q.n, p.max_q) * p.group) return;
  float M = -INFINITY;
  for (int k = 0; k < p.pieces; ++k) {
    const int64_t at = (static_cast<int64_t>(blockIdx.x) * p.pieces + k) * kRows + r;
    M = fmaxf(M, p.prompt_ml[2 * at]);
  }
  const float base = M == -INFINITY ? 0.0f : M;
  float L = 0.0f, f[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll 4
  for (int k = 0; k < p.pieces; ++k) {
    const int64_t at = (static_cast<int64_t>(blockIdx.x) * p.pieces + k) * kRows + r;
    const float2 ml = *reinterpret_cast<const float2*>(p.prompt_ml + 2 * at);
    const float4* o = reinterpret_cast<const float4*>(p.prompt_part + at * D + e);
    const float4 x = o[0], y = o[1];
    const float a = __builtin_amdgcn_exp2f(ml.x - base);
    L += a * ml.y;
    f[0] += a * x.x; f[1] += a * x.y; f[2] += a * x.z; f[3] += a * x.w;
    f[4] += a * y.x; f[5] += a * y.y; f[6] += a * y.z; f[7] += a * y.w;
  }
  const float inv = L == 0.0f ? 0.0f : 1.0f / L;
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] *= inv;
  store_out<8>(static_cast<bf16_t*>(p.out) + (q.q0 + query) * p.ldo +
                   static_cast<int64_t>(h * p.group + row - query * p.group) * D + e, f);
}

template <int D> hipError_t launch(const AttnParams& p, hipStream_t s) {
  const uint32_t tiles = static_cast<uint32_t>(p.prompt_tiles * p.c.heads);
  attn_prompt_kernel<D><<<tiles * p.pieces, kThreads, 0, s>>>(p);
  if (p.pieces > 1) attn_prompt_join_kernel<D><<<dim3(tiles, kRows * (D / 8) / kThreads), kThreads, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attention_prompts(const AttnParams& p, hipStream_t s) {
  switch (p.c.d) {
    case 64: return launch<64>(p, s);
    case 128: return launch<128>(p, s);
    default: return launch<256>(p, s);
  }
}

}  // namespace cts
