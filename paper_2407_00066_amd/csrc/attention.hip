// Attention over the 4-bit cache (cts_kv_attention), one pass over the keys and
// values with the running maximum and sum of the softmax:
//   S = scale log2(e) K q;  m' = max(m, max S);  l' = l 2^(m - m') + sum 2^(S - m');
//   o' = o 2^(m - m') + sum_t 2^(S_t - m') v_t;  at the end out = o / l.
// Both products run on matrix cores transposed, S^T = K Q^T and O^T = V^T P^T: the
// 16 x 16 result of the first holds, in each lane, four tokens' weights for one
// query row, and with the tokens numbered the way the lanes hold them it is the
// second product's operand as it stands.  Nothing crosses lanes but the maximum.
//   Lane l = 16 g + n.  First product: A row = token n of 16, k = elements
//   (d/4) g + 8 s .. + 7 in step s (a lane's codes are consecutive, and the
//   queries are loaded in the same order); result: row = token 4 g + i, column n =
//   query row.  Second: A row = element, k = tokens 4 g .. 4 g + 3 of two groups of 16.
// Codes become bf16 in registers, two an instruction with their scale.
#include <algorithm>

#include "block_internal.h"

namespace cts {
namespace {

constexpr int kRowTile = 16;       // query rows of a tile
constexpr int kUnit = 32;          // tokens of a step
constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;

__device__ __forceinline__ uint32_t fp4_pair(uint32_t w, float unit, int byte) {
  switch (byte) {
    case 0: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 0));
    case 1: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 1));
    case 2: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 2));
    default: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 3));
  }
}

// the float 2^(s - 127) of byte i of w (255: as the conversion's NaN scale)
__device__ __forceinline__ float unit_of(uint32_t w, int i) {
  return __uint_as_float((i < 3 ? w << (23 - 8 * i) : w >> 1) & 0x7f800000u);
}

__device__ __forceinline__ float max_over_groups(float v) {       // over the lanes of the same n
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum_over_groups(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ bf16x8 frag(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  typedef uint32_t u32x4_ __attribute__((ext_vector_type(4)));
  const u32x4_ v = {a, b, c, d};
  return __builtin_bit_cast(bf16x8, v);
}

// eight floats as NS bf16 parts whose sum is the float (to 8, 16 or 24 bits)
template <int NS> __device__ __forceinline__ void split(const float* f, bf16x8* out) {
  float r[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = f[i];
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = f32_to_bf16_pair(r[2 * i], r[2 * i + 1]);
      r[2 * i] -= __uint_as_float(w[i] << 16);
      r[2 * i + 1] -= __uint_as_float(w[i] & 0xffff0000u);
    }
    out[s] = frag(w[0], w[1], w[2], w[3]);
  }
}

struct Tile {                      // what a 16-row tile of a sequence covers
  int q0, rows, row0;              // the sequence's first query row, its rows (query x head of the group), the tile's first
  int first_pos;                   // position of the sequence's first query
  int lo, hi;                      // tokens that some row of the tile sees, [lo, hi)
};

// false: no rows here
__device__ __forceinline__ bool tile_of(const AttnParams& p, int b, int sub, Tile* t) {
  int q0 = b, q1 = b + 1;
  if (p.q_start) {
    q0 = min(max(p.q_start[b], 0), p.T);
    q1 = min(max(p.q_start[b + 1], q0), p.T);
  }
  const int nq = q1 - q0, len = min(max(p.kv_len[b], 0), p.max_kv);
  t->q0 = q0;
  t->rows = min(nq, p.max_q) * p.group;
  t->row0 = sub * kRowTile;
  if (t->row0 >= t->rows) return false;
  t->first_pos = len - nq;
  const int j0 = t->row0 / p.group, j1 = (min(t->rows, t->row0 + kRowTile) - 1) / p.group;
  t->hi = max(0, t->first_pos + j1 + 1);
  t->lo = p.window ? max(0, t->first_pos + j0 - p.window + 1) & ~(kUnit - 1) : 0;
  return true;
}

__device__ __forceinline__ int pieces_of(const AttnParams& p, const Tile& t) {
  return t.hi > t.lo ? (t.hi - t.lo + p.chunk - 1) / p.chunk : 1;
}

template <typename TQ> __device__ __forceinline__ void store_out(TQ* o, const float* f);
template <> __device__ __forceinline__ void store_out<float>(float* o, const float* f) {
  reinterpret_cast<float4*>(o)[0] = make_float4(f[0], f[1], f[2], f[3]);
  reinterpret_cast<float4*>(o)[1] = make_float4(f[4], f[5], f[6], f[7]);
}
template <> __device__ __forceinline__ void store_out<bf16_t>(bf16_t* o, const float* f) {
  *reinterpret_cast<uint4*>(o) = make_uint4(f32_to_bf16_pair(f[0], f[1]), f32_to_bf16_pair(f[2], f[3]),
                                            f32_to_bf16_pair(f[4], f[5]), f32_to_bf16_pair(f[6], f[7]));
}

template <typename TQ> __device__ __forceinline__ void load_q(const TQ* q, float* f);
template <> __device__ __forceinline__ void load_q<float>(const float* q, float* f) {
  const float4 a = reinterpret_cast<const float4*>(q)[0], b = reinterpret_cast<const float4*>(q)[1];
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
  f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
template <> __device__ __forceinline__ void load_q<bf16_t>(const bf16_t* q, float* f) {
  const uint4 v = *reinterpret_cast<const uint4*>(q);
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}

// One step's codes and scales as a lane holds them, of two groups of 16 tokens.
template <int D> struct Raw {
  static constexpr int KW = D / 32;              // words of keys a lane holds: d/4 elements of one token
  static constexpr int NC = D > 128 ? 2 : 1;     // 16-byte pieces of values: 8 elements of 4 tokens each
  uint32_t k[2][KW], ks[2];
  uint4 v[2][NC];
  uint32_t vs[2][NC];
};

// A workgroup takes a piece of one tile's tokens for one key/value head; its
// waves take steps of 32 tokens in turn, each with a softmax of its own, joined
// at the end.
template <int D, typename TQ>
__global__ __launch_bounds__(kThreads) void attn_rows_kernel(AttnParams p) {
  constexpr int NS = sizeof(TQ) == 4 ? 3 : 1;
  constexpr int KS = D / 32;                     // steps of the first product
  constexpr int NC = Raw<D>::NC;
  constexpr int NB = D == 64 ? 4 : 8;            // elements a lane takes of its piece
  __shared__ float lds_o[kWaves][kRowTile][D + 4];
  __shared__ float lds_m[kWaves][kRowTile], lds_l[kWaves][kRowTile];
  int id = blockIdx.x;
  const int piece = id % p.pieces; id /= p.pieces;
  const int h = id % p.c.heads; id /= p.c.heads;
  const int sub = id % p.subs, b = id / p.subs;
  Tile t;
  if (!tile_of(p, b, sub, &t)) return;
  const int n_pieces = pieces_of(p, t);
  if (piece >= n_pieces) return;
  const int t0 = t.lo + piece * p.chunk, t1 = min(t.hi, t0 + p.chunk);

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int n = lane & 15, g = lane >> 4;
  const int row = t.row0 + n;
  const bool live = row < t.rows;
  const int pos = live ? t.first_pos + row / p.group : -1;              // sees tokens first .. pos
  const int first = p.window ? pos - p.window + 1 : 0;

  bf16x8 qf[KS][NS];
  {
    const TQ* q = static_cast<const TQ*>(p.q) + (live ? (t.q0 + row / p.group) * p.ldq +
                                                 static_cast<int64_t>(h * p.group + row % p.group) * D : 0);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      float f[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      if (live) load_q(q + (D / 4) * g + 8 * s, f);
      split<NS>(f, qf[s]);
    }
  }

  f32x4 o[NC][NB];
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int e = 0; e < NB; ++e) o[c][e] = f32x4{0, 0, 0, 0};
  float m = -INFINITY, l = 0.0f;

  const int page_size = 1 << p.c.page_shift;
  const int steps = t1 > t0 ? (t1 - t0 + kUnit - 1) / kUnit : 0;
  // tokens that every live row of the tile sees
  const int all_hi = t.first_pos + t.row0 / p.group + 1;
  const int all_lo = p.window ? t.first_pos + (min(t.rows, t.row0 + kRowTile) - 1) / p.group - p.window + 1 : 0;

  auto load = [&](int step, Raw<D>& r) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      // a group past the piece's end lies past what is seen: the last group's codes stand in, masked
      const int tok = min(t0 + step * kUnit + 16 * i, (t1 - 1) & ~15);
      const int page = __builtin_amdgcn_readfirstlane(p.table[static_cast<int64_t>(b) * p.max_pages + (tok >> p.c.page_shift)]);
      const bool bad = static_cast<uint32_t>(page) >= static_cast<uint32_t>(p.c.n_pages);
      const int64_t base = ((static_cast<int64_t>(bad ? 0 : page) * p.c.heads + h) << p.c.page_shift) + (tok & (page_size - 1));
      const uint8_t* kc = p.c.kc + base * (D / 2) + n * (D / 2) + g * (D / 8);
      const uint8_t* ks = p.c.ks + base * (D / 32) + n * (D / 32);
      const uint8_t* vc = p.c.vc + base * (D / 2);
      const uint8_t* vs = p.c.vs + base * (D / 32);
      if constexpr (D == 64) {
        const uint2 w = *reinterpret_cast<const uint2*>(kc);
        r.k[i][0] = w.x; r.k[i][1] = w.y;
        r.ks[i] = ks[g >> 1];
      } else {
#pragma unroll
        for (int x = 0; x < D / 128; ++x) {
          const uint4 w = reinterpret_cast<const uint4*>(kc)[x];
          r.k[i][4 * x] = w.x; r.k[i][4 * x + 1] = w.y; r.k[i][4 * x + 2] = w.z; r.k[i][4 * x + 3] = w.w;
        }
        if constexpr (D == 128) r.ks[i] = ks[g];
        else r.ks[i] = *reinterpret_cast<const uint16_t*>(ks + 2 * g);
      }
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int eighth = (n & (D / 8 - 1)) + 16 * c;                  // D = 64: lanes n and n + 8 share a piece
        r.v[i][c] = *reinterpret_cast<const uint4*>(vc + (g * (D / 8) + eighth) * 16);
        r.vs[i][c] = *reinterpret_cast<const uint32_t*>(vs + (g * (D / 32) + eighth / 4) * 4);
      }
      if (bad) {
        r.ks[i] = 0xffffu;
#pragma unroll
        for (int c = 0; c < NC; ++c) r.vs[i][c] = 0xffffffffu;
      }
    }
  };

  for (int step = wave; step < steps; step += kWaves) {
    Raw<D> r;
    load(step, r);
    const int at = t0 + step * kUnit;
    // scores of the lane's row against tokens at + 16 i + 4 g + j
    f32x4 s[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      s[i] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int x = 0; x < KS; ++x) {
        const float unit = unit_of(r.ks[i], D == 256 ? x / 4 : 0);
        const bf16x8 a = frag(fp4_pair(r.k[i][x], unit, 0), fp4_pair(r.k[i][x], unit, 1),
                              fp4_pair(r.k[i][x], unit, 2), fp4_pair(r.k[i][x], unit, 3));
#pragma unroll
        for (int y = 0; y < NS; ++y) s[i] = mfma(a, qf[x][y], s[i]);
      }
    }
    float sc[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sc[i] = s[i >> 2][i & 3] * p.scale_log2e;
    const bool masked = at + kUnit > min(all_hi, t1) || at < all_lo;    // the same for the whole wave
    bool nan_value[NC] = {};
    float gone[8];                                                       // weights of the values that are NaN
    if (masked) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int tok = at + 16 * i + 4 * g + j;
          const bool seen = tok <= pos && tok >= first && tok < t1;
          if (!seen) sc[4 * i + j] = -INFINITY;
          gone[4 * i + j] = seen ? 1.0f : 0.0f;
        }
      // A weight of zero does not hide a NaN value: NaN blocks are taken out of
      // the product, and the rows that do see one are made NaN below.
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            nan_value[c] |= ((r.vs[i][c] >> (8 * j)) & 0xffu) == 0xffu;
    }
    float top = sc[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) top = fmaxf(top, sc[i]);
    const float m_new = fmaxf(m, max_over_groups(top));
    const float base = m_new == -INFINITY ? 0.0f : m_new;
    const float fade = __builtin_amdgcn_exp2f(m - base);
    m = m_new;
    float w[8];
    l *= fade;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      w[i] = __builtin_amdgcn_exp2f(sc[i] - base);
      l += w[i];
    }
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < NB; ++e) o[c][e] *= fade;
    bf16x8 pf[NS];
    split<NS>(w, pf);

#pragma unroll
    for (int c = 0; c < NC; ++c) {
      if (masked && __any(nan_value[c])) {
        uint32_t hit[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) hit[i] = 0;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (((r.vs[i][c] >> (8 * j)) & 0xffu) == 0xffu) {
              hit[2 * i + j / 2] |= 0x3f80u << (16 * (j & 1));
              r.vs[i][c] ^= 0x80u << (8 * j);                            // 255 -> 127
              (&r.v[i][c].x)[j] = 0;
            }
        bf16x8 seen[1];
        split<1>(gone, seen);
        const f32x4 count = mfma(frag(hit[0], hit[1], hit[2], hit[3]), seen[0], f32x4{0, 0, 0, 0});
#pragma unroll
        for (int e = 0; e < NB; ++e)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (count[i] > 0.0f) o[c][e][i] = NAN;
      }
      const uint32_t* vw[2] = {&r.v[0][c].x, &r.v[1][c].x};
      uint32_t word[2][4];
      float unit[2][4];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          word[i][j] = D == 64 ? vw[i][j] >> (16 * (n >> 3)) : vw[i][j];
          unit[i][j] = unit_of(r.vs[i][c], j);
        }
#pragma unroll
      for (int e = 0; e < NB / 2; ++e) {
        uint32_t x[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) x[i][j] = fp4_pair(word[i][j], unit[i][j], e);
        const bf16x8 even = frag(__builtin_amdgcn_perm(x[0][1], x[0][0], 0x05040100u), __builtin_amdgcn_perm(x[0][3], x[0][2], 0x05040100u),
                                 __builtin_amdgcn_perm(x[1][1], x[1][0], 0x05040100u), __builtin_amdgcn_perm(x[1][3], x[1][2], 0x05040100u));
        const bf16x8 odd = frag(__builtin_amdgcn_perm(x[0][1], x[0][0], 0x07060302u), __builtin_amdgcn_perm(x[0][3], x[0][2], 0x07060302u),
                                __builtin_amdgcn_perm(x[1][1], x[1][0], 0x07060302u), __builtin_amdgcn_perm(x[1][3], x[1][2], 0x07060302u));
#pragma unroll
        for (int y = 0; y < NS; ++y) {
          o[c][2 * e] = mfma(even, pf[y], o[c][2 * e]);
          o[c][2 * e + 1] = mfma(odd, pf[y], o[c][2 * e + 1]);
        }
      }
    }
  }

  // join the waves: result row 4 g + i of piece c is elements 8 (4 g + i + 16 c) + e (D = 64: 8 of (4 g + i) % 8, half each)
  l = sum_over_groups(l);
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < NB; e += 4) {
        const int r = 4 * g + i;
        const int at = D == 64 ? 8 * (r & 7) + 4 * (r >> 3) + e : 8 * (r + 16 * c) + e;
        *reinterpret_cast<float4*>(&lds_o[wave][n][at]) = make_float4(o[c][e][i], o[c][e + 1][i], o[c][e + 2][i], o[c][e + 3][i]);
      }
  if (g == 0) { lds_m[wave][n] = m; lds_l[wave][n] = l; }
  __syncthreads();

  const int64_t tile = (static_cast<int64_t>(b) * p.subs + sub) * p.c.heads + h;
  const int n_rows = min(kRowTile, t.rows - t.row0);
  float* const ml = p.part + static_cast<int64_t>(p.B) * p.subs * p.c.heads * p.pieces * p.part_rows * D;
  for (int k = threadIdx.x; k < n_rows * (D / 8); k += kThreads) {
    const int r = k / (D / 8), e = (k % (D / 8)) * 8;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) M = fmaxf(M, lds_m[w][r]);
    const float base = M == -INFINITY ? 0.0f : M;
    float L = 0.0f, f[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float a = __builtin_amdgcn_exp2f(lds_m[w][r] - base);
      L += a * lds_l[w][r];
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] += a * lds_o[w][r][e + i];
    }
    if (n_pieces == 1) {
      const float inv = L == 0.0f ? 0.0f : 1.0f / L;
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] *= inv;
      const int q_row = t.row0 + r;
      store_out(static_cast<TQ*>(p.out) + (t.q0 + q_row / p.group) * p.ldo +
                    static_cast<int64_t>(h * p.group + q_row % p.group) * D + e, f);
    } else {
      const int64_t at = (tile * p.pieces + piece) * p.part_rows + r;
      float4* o4 = reinterpret_cast<float4*>(p.part + at * D + e);
      o4[0] = make_float4(f[0], f[1], f[2], f[3]);
      o4[1] = make_float4(f[4], f[5], f[6], f[7]);
      if (e == 0) { ml[2 * at] = M; ml[2 * at + 1] = L; }
    }
  }
}

// Joins a tile's pieces, in their order.
template <int D, typename TQ>
__global__ __launch_bounds__(kThreads) void attn_join_kernel(AttnParams p) {
  int id = blockIdx.x;
  const int h = id % p.c.heads; id /= p.c.heads;
  const int sub = id % p.subs, b = id / p.subs;
  Tile t;
  if (!tile_of(p, b, sub, &t)) return;
  const int n_pieces = pieces_of(p, t);
  if (n_pieces == 1) return;
  const int64_t tile = blockIdx.x;
  const int n_rows = min(kRowTile, t.rows - t.row0);
  const float* const ml = p.part + static_cast<int64_t>(p.B) * p.subs * p.c.heads * p.pieces * p.part_rows * D;
  for (int k = threadIdx.x; k < n_rows * (D / 8); k += kThreads) {
    const int r = k / (D / 8), e = (k % (D / 8)) * 8;
    float M = -INFINITY;
    for (int s = 0; s < n_pieces; ++s) M = fmaxf(M, ml[2 * ((tile * p.pieces + s) * p.part_rows + r)]);
    const float base = M == -INFINITY ? 0.0f : M;
    float L = 0.0f, f[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int s = 0; s < n_pieces; ++s) {
      const int64_t at = (tile * p.pieces + s) * p.part_rows + r;
      const float a = __builtin_amdgcn_exp2f(ml[2 * at] - base);
      L += a * ml[2 * at + 1];
      const float4* o4 = reinterpret_cast<const float4*>(p.part + at * D + e);
      const float4 x = o4[0], y = o4[1];
      f[0] += a * x.x; f[1] += a * x.y; f[2] += a * x.z; f[3] += a * x.w;
      f[4] += a * y.x; f[5] += a * y.y; f[6] += a * y.z; f[7] += a * y.w;
    }
    const float inv = L == 0.0f ? 0.0f : 1.0f / L;
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] *= inv;
    const int q_row = t.row0 + r;
    store_out(static_cast<TQ*>(p.out) + (t.q0 + q_row / p.group) * p.ldo +
                  static_cast<int64_t>(h * p.group + q_row % p.group) * D + e, f);
  }
}

template <int D, typename TQ> hipError_t launch(const AttnParams& p, hipStream_t s) {
  const uint32_t tiles = static_cast<uint32_t>(static_cast<int64_t>(p.B) * p.subs * p.c.heads);
  attn_rows_kernel<D, TQ><<<tiles * p.pieces, kThreads, 0, s>>>(p);
  if (p.pieces > 1) attn_join_kernel<D, TQ><<<tiles, kThreads, 0, s>>>(p);
  return hipGetLastError();
}

// Workgroups that a long axis is split up to: a few for every compute unit.
constexpr int64_t kTargetGroups = 1024;
constexpr int kChunkUnit = kUnit * kWaves;

}  // namespace

size_t plan_attention(AttnParams* p) {
  p->subs = static_cast<int>((static_cast<int64_t>(p->max_q) * p->group + kRowTile - 1) / kRowTile);
  const int64_t tiles = static_cast<int64_t>(p->B) * p->subs * p->c.heads;
  // a window's span: the tile's queries, and its start rounded down to a step
  int64_t span = p->max_kv;
  if (p->window) span = std::min<int64_t>(span, static_cast<int64_t>(p->window) + kRowTile + kUnit);
  span = std::max<int64_t>(span, 1);
  const int64_t most = (span + kChunkUnit - 1) / kChunkUnit;
  const int64_t per = (span * std::max<int64_t>(tiles, 1) + kTargetGroups - 1) / kTargetGroups;
  const int64_t chunk = std::min(most, (per + kChunkUnit - 1) / kChunkUnit) * kChunkUnit;
  p->chunk = static_cast<int>(chunk);
  p->pieces = static_cast<int>((span + chunk - 1) / chunk);
  p->part_rows = static_cast<int>(std::min<int64_t>(kRowTile, static_cast<int64_t>(p->max_q) * p->group));
  // tiles x pieces is at most tiles x most and less than the target and one a tile more
  const uint64_t parts = std::min(tiles * most, kTargetGroups + tiles);
  return 256 + parts * p->part_rows * (p->c.d + 2) * sizeof(float);
}

hipError_t launch_attention(const AttnParams& p, hipStream_t s) {
  const bool f32 = p.dtype == CTS_F32;
  switch (p.c.d) {
    case 64: return f32 ? launch<64, float>(p, s) : launch<64, bf16_t>(p, s);
    case 128: return f32 ? launch<128, float>(p, s) : launch<128, bf16_t>(p, s);
    default: return f32 ? launch<256, float>(p, s) : launch<256, bf16_t>(p, s);
  }
}

}  // namespace cts
