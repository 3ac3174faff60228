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
// Codes become bf16 in registers, two an instruction with their scale; nothing is
// staged in shared memory.  Bound by the cache's bytes where there are many (64 requests of 4000
// tokens: 57 to 60 us, 4.7 to 4.9 TB/s; four of 40000 to 131072: 75 us, 4.9 TB/s), by the chain of
// length, page, codes and join where there are few (one of 709 tokens: 7.4 us).
#include <algorithm>

#include "attention_common.h"

namespace cts {
namespace {

// What a wave holds of a tile: sums, and for its query row n the running maximum
// and (over the lane's own tokens) length.
template <int D> struct State {
  static constexpr int NC = D > 128 ? 2 : 1;     // 16-byte pieces of values a lane takes: 8 elements of 4 tokens each
  static constexpr int NB = D == 64 ? 4 : 8;     // elements of a piece that are the lane's (D = 64: lanes n and n + 8 share)
  f32x4 o[NC][NB];
  float m, l;
  // sum o[c][e][i] of lane 16 g + n is row n's element
  static __device__ __forceinline__ int element(int g, int c, int i) {
    const int r = 4 * g + i;
    return D == 64 ? 8 * (r & 7) + 4 * (r >> 3) : 8 * (r + 16 * c);
  }
};

// Page number of the lane's group of 16 tokens in the steps s0, s0 + stride, ..: two
// groups a step, a lane one.  Groups past the last seen token are looked up too (what
// stands there is masked), so that a tile's first look-up need not wait for its length.
__device__ __forceinline__ int look_up(const AttnParams& p, int b, int lo, int s0, int stride) {
  const int lane = threadIdx.x & 63;
  const int tok = lo + (s0 + (lane >> 1) * stride) * kUnit + 16 * (lane & 1);
  return p.table[static_cast<int64_t>(b) * p.max_pages + min(tok >> p.c.page_shift, p.max_pages - 1)];
}

// `count` of the tile's steps from s0, `stride` apart, for key/value head h, by one
// wave; pages: look_up of the first 32.
template <int D, typename TQ, int stride>
__device__ __forceinline__ void attend(const AttnParams& p, const Tile& t, int h, int s0, int count, int pages,
                                       State<D>& st) {
  // Parts of a query (bf16: itself) and of a weight.  bf16 weights are rounded once:
  // a second part brings the error against 64 bits from 1.25 to 1.0 times that of rounding
  // the output alone, and takes 41 -> 52 us for 64 requests of 40 to 4000 tokens.
  constexpr int NS = sizeof(TQ) == 4 ? 3 : 1;
  constexpr int KS = D / 32;                     // steps of the first product; words of keys a lane holds
  constexpr int NC = State<D>::NC, NB = State<D>::NB;
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int row = t.row0 + n;
  const bool live = row < t.rows;
  const int query = row / p.group;
  const int pos = live ? t.first_pos + query : -1;                      // sees tokens first .. pos
  const int first = p.window ? pos - p.window + 1 : 0;
  auto seen = [&](int from, int i, int j) {                              // token from + a constant
    const int tok = 16 * i + j;
    return tok <= pos - from && tok >= first - from;
  };

  bf16x8 qf[KS][NS];
  {
    const TQ* q = static_cast<const TQ*>(p.q) + (live ? (t.q0 + query) * p.ldq +
                                                 static_cast<int64_t>(h * p.group + row - query * p.group) * D : 0);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      float f[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      if (live) load_q(q + (D / 4) * g + 8 * s, f);
      split<NS>(f, qf[s]);
    }
  }
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int e = 0; e < NB; ++e) st.o[c][e] = f32x4{0, 0, 0, 0};
  st.m = -INFINITY;
  st.l = 0.0f;
  if (t.hi <= t.lo) return;                                             // nothing is seen

  // tokens that every live row of the tile sees
  const int all_hi = t.first_pos + t.row0 / p.group + 1;
  const int all_lo = p.window ? t.first_pos + (min(t.rows, t.row0 + kRowTile) - 1) / p.group - p.window + 1 : 0;

  struct Group { int64_t base; uint32_t bad; };       // a group's first token among its head's; all ones: its page is outside the cache
  const int page_mask = (1 << p.c.page_shift) - 1;
  auto group_of = [&](int it, int i) -> Group {
    const int page = __builtin_amdgcn_readlane(pages, 2 * (it & 31) + i);
    const int tok = t.lo + (s0 + it * stride) * kUnit + 16 * i;
    const bool bad = static_cast<uint32_t>(page) >= static_cast<uint32_t>(p.c.n_pages);
    return {((static_cast<int64_t>(bad ? 0 : page) * p.c.heads + h) << p.c.page_shift) + (tok & page_mask), bad ? ~0u : 0u};
  };
  const uint32_t k_at = n * (D / 2) + g * (D / 8), ks_at = n * (D / 32) + (D == 64 ? g >> 1 : D == 128 ? g : 2 * g);
  uint32_t v_at[NC], vs_at[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int eighth = (n & (D / 8 - 1)) + 16 * c;
    v_at[c] = (g * (D / 8) + eighth) * 16;
    vs_at[c] = (g * (D / 32) + eighth / 4) * 4;
  }
  uint32_t k[2][KS], ks[2], vs[2][NC], v_bad[2];
  uint4 v[2][NC];
  Group gr[2];
  auto load_k = [&](int it) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      gr[i] = group_of(it, i);
      const uint8_t* kc = p.c.kc + gr[i].base * (D / 2);
      const uint8_t* sc = p.c.ks + gr[i].base * (D / 32);
      if constexpr (D == 64) {
        const uint2 w = *reinterpret_cast<const uint2*>(kc + k_at);
        k[i][0] = w.x; k[i][1] = w.y;
      } else {
#pragma unroll
        for (int x = 0; x < D / 128; ++x) {
          const uint4 w = *reinterpret_cast<const uint4*>(kc + k_at + 16 * x);
          k[i][4 * x] = w.x; k[i][4 * x + 1] = w.y; k[i][4 * x + 2] = w.z; k[i][4 * x + 3] = w.w;
        }
      }
      ks[i] = D == 256 ? *reinterpret_cast<const uint16_t*>(sc + ks_at) : sc[ks_at];
    }
  };
  auto load_v = [&]() {                                                  // of the step load_k was last called for
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint8_t* vc = p.c.vc + gr[i].base * (D / 2);
      const uint8_t* sc = p.c.vs + gr[i].base * (D / 32);
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        v[i][c] = *reinterpret_cast<const uint4*>(vc + v_at[c]);
        vs[i][c] = *reinterpret_cast<const uint32_t*>(sc + vs_at[c]);
      }
      v_bad[i] = gr[i].bad;
    }
  };

  load_k(0);
  load_v();
  for (int it = 0; it < count; ++it) {
    const int at = t.lo + (s0 + it * stride) * kUnit;
    // scores of the lane's row against tokens at + 16 i + 4 g + j
    f32x4 x[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      x[i] = f32x4{0, 0, 0, 0};
      const uint32_t units = ks[i] | gr[i].bad;                          // here: asked for sooner, it would be waited for sooner
#pragma unroll
      for (int y = 0; y < KS; ++y) {
        const float unit = unit_of(units, D == 256 ? y / 4 : 0);
        const bf16x8 a = frag(fp4_pair(k[i][y], unit, 0), fp4_pair(k[i][y], unit, 1),
                              fp4_pair(k[i][y], unit, 2), fp4_pair(k[i][y], unit, 3));
#pragma unroll
        for (int z = 0; z < NS; ++z) x[i] = mfma(a, qf[y][z], x[i]);
      }
    }
    // the next keys are on their way during the softmax and the second product,
    // the next values during the next first product (past the end: the last step's again)
    const int next = min(it + 1, count - 1);
    if ((next & 31) == 0 && next != 0) pages = rare(look_up(p, t.b, t.lo, s0 + next * stride, stride));
    load_k(next);

    float sc[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sc[i] = x[i >> 2][i & 3] * p.scale_log2e;
    const bool masked = at + kUnit > all_hi || at < all_lo;              // the same for the whole wave
    if (masked) {
      const int from = rare(at + 4 * g);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (!seen(from, i, j)) sc[4 * i + j] = -INFINITY;
    }
    float top = sc[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) top = fmaxf(top, sc[i]);
    top = max_over_groups(top);
    if (__any(top > st.m + kSlack)) {
      const float m_new = fmaxf(st.m, top), fade = __builtin_amdgcn_exp2f(st.m - (m_new == -INFINITY ? 0.0f : m_new));
      st.l *= fade;
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < NB; ++e) st.o[c][e] *= fade;
      st.m = m_new;
    }
    const float base = st.m == -INFINITY ? 0.0f : st.m;
    float w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      w[i] = __builtin_amdgcn_exp2f(sc[i] - base);
      if (NS == 3) st.l += w[i];
    }
    bf16x8 pf[NS];
    split<NS>(w, pf);
    if (NS == 1) {
      const uint4 x = __builtin_bit_cast(uint4, pf[0]);
      st.l = add_pair(x.x, add_pair(x.y, add_pair(x.z, add_pair(x.w, st.l))));
    }

#pragma unroll
    for (int c = 0; c < NC; ++c) {
      vs[0][c] |= v_bad[0];
      vs[1][c] |= v_bad[1];
      if (masked) {
        // A weight of zero does not hide a NaN or infinite value: blocks that can hold one are
        // taken out of the product, and the rows that do see one are made NaN.
        uint32_t hit[4] = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (past_scales(rare(static_cast<int>(vs[i][c])), j)) hit[2 * i + j / 2] |= 0x3f80u << (16 * (j & 1));
        if (__any((hit[0] | hit[1] | hit[2] | hit[3]) != 0)) {
          float in[8];
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              in[4 * i + j] = seen(at + 4 * g, i, j) ? 1.0f : 0.0f;
              if (past_scales(vs[i][c], j)) {
                vs[i][c] ^= 0x80u << (8 * j);                            // 255 -> 127
                (&v[i][c].x)[j] = 0;
              }
            }
          bf16x8 who[1];
          split<1>(in, who);
          const f32x4 count = mfma(frag(hit[0], hit[1], hit[2], hit[3]), who[0], f32x4{0, 0, 0, 0});
#pragma unroll
          for (int e = 0; e < NB; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (count[i] > 0.0f) st.o[c][e][i] = NAN;
        }
      }
      const uint32_t* vw[2] = {&v[0][c].x, &v[1][c].x};
#pragma unroll
      for (int e = 0; e < NB / 2; ++e) {
        uint32_t y[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            y[i][j] = fp4_pair(D == 64 ? vw[i][j] >> (16 * (n >> 3)) : vw[i][j], unit_of(vs[i][c], j), e);
        const bf16x8 even = frag(__builtin_amdgcn_perm(y[0][1], y[0][0], 0x05040100u), __builtin_amdgcn_perm(y[0][3], y[0][2], 0x05040100u),
                                 __builtin_amdgcn_perm(y[1][1], y[1][0], 0x05040100u), __builtin_amdgcn_perm(y[1][3], y[1][2], 0x05040100u));
        const bf16x8 odd = frag(__builtin_amdgcn_perm(y[0][1], y[0][0], 0x07060302u), __builtin_amdgcn_perm(y[0][3], y[0][2], 0x07060302u),
                                __builtin_amdgcn_perm(y[1][1], y[1][0], 0x07060302u), __builtin_amdgcn_perm(y[1][3], y[1][2], 0x07060302u));
#pragma unroll
        for (int z = 0; z < NS; ++z) {
          st.o[c][2 * e] = mfma(even, pf[z], st.o[c][2 * e]);
          st.o[c][2 * e + 1] = mfma(odd, pf[z], st.o[c][2 * e + 1]);
        }
      }
    }
    load_v();
  }
  st.l = sum_over_groups(st.l);
}

// A query row's address in out.
template <int D, typename TQ>
__device__ __forceinline__ TQ* out_at(const AttnParams& p, const Tile& t, int h, int r) {
  const int row = t.row0 + r, query = row / p.group;
  return static_cast<TQ*>(p.out) + (t.q0 + query) * p.ldo + static_cast<int64_t>(h * p.group + row - query * p.group) * D;
}

// What WAVES waves of a workgroup have of the same rows, in shared memory.
template <int D, int WAVES> struct Shared {
  float sums[WAVES][kRowTile][D + 4];
  float2 ml[WAVES][kRowTile];
};

// The wave's steps (every WAVES-th of `steps` from s0, its own first) into shared memory.
template <int D, typename TQ, int WAVES>
__device__ __forceinline__ void attend_shared(const AttnParams& p, const Tile& t, int h, int s0, int steps, int wave,
                                              int pages, Shared<D, WAVES>& sh) {
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  if (wave < steps) {
    State<D> st;
    attend<D, TQ, WAVES>(p, t, h, s0 + wave, (steps - wave + WAVES - 1) / WAVES, pages, st);
    if (t.row0 + n < t.rows) {
      float* const o = sh.sums[wave][n];
#pragma unroll
      for (int c = 0; c < State<D>::NC; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float f[State<D>::NB];
#pragma unroll
          for (int e = 0; e < State<D>::NB; ++e) f[e] = st.o[c][e][i];
          store_out<State<D>::NB>(o + State<D>::element(g, c, i), f);
        }
      if (g == 0) sh.ml[wave][n] = make_float2(st.m, st.l);
    }
  } else if (lane < kRowTile) {                    // fewer steps than waves
    sh.ml[wave][lane] = make_float2(-INFINITY, 0.0f);
  }
}

// Eight elements of a row, from e: the waves' sums together, their maximum and length.
template <int D, int WAVES>
__device__ __forceinline__ float2 join_waves(const Shared<D, WAVES>& sh, int r, int e, float* f) {
  float M = -INFINITY;
#pragma unroll
  for (int v = 0; v < WAVES; ++v) M = fmaxf(M, sh.ml[v][r].x);
  const float base = M == -INFINITY ? 0.0f : M;
  float L = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = 0.0f;
#pragma unroll
  for (int v = 0; v < WAVES; ++v) {
    const float2 w = sh.ml[v][r];
    if (w.y == 0.0f) continue;                     // saw nothing: no sums
    const float a = __builtin_amdgcn_exp2f(w.x - base);
    L += a * w.y;
    const float4* o = reinterpret_cast<const float4*>(&sh.sums[v][r][e]);
    const float4 x = o[0], y = o[1];
    f[0] += a * x.x; f[1] += a * x.y; f[2] += a * x.z; f[3] += a * x.w;
    f[4] += a * y.x; f[5] += a * y.y; f[6] += a * y.z; f[7] += a * y.w;
  }
  return make_float2(M, L);
}

template <int D, typename TQ>
__device__ __forceinline__ void put_row(const AttnParams& p, const Tile& t, int h, int r, int e, float L, float* f) {
  const float inv = L == 0.0f ? 0.0f : 1.0f / L;
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] *= inv;
  store_out<8>(out_at<D, TQ>(p, t, h, r) + e, f);
}

// The batch's steps (of the sequences with few rows), tile after tile and head
// after head, are dealt out to the workgroups in equal runs, however the lengths
// differ; a run's waves take its steps in turn and join in shared memory (a wave with
// a run of its own leaves eight times the sums to the join: 32 requests of 30000 tokens,
// 32 + 8 heads of 128, 213 / 203 us).  A run starts and ends inside a tile as a rule:
// those two leave their sums in the workspace (slots 2 w and 2 w + 1) for the join,
// the tiles between are whole and final.
// Few tiles are each cut into a whole number of runs, so that no workgroup takes two
// pieces one after the other (one request of 131072 tokens 38.2 / 37.3 us, of 40000
// 20.6 / 17.2).  One workgroup for every compute unit: two, 1 request of 18000 tokens
// 16.0 / 14.6, 4 of 100000 95 / 90.  Heads of 64 leave too few bytes under way so, and
// have two (one of 200000 tokens 37.9 / 36.0); of heads of 256 a compute unit holds one.
template <int D, typename TQ>
__global__ __launch_bounds__(64 * kWaves, D == 256 || sizeof(TQ) == 4 ? 2 : 4) void attn_runs_kernel(AttnParams p) {
  __shared__ __attribute__((aligned(16))) Shared<D, kWaves> sh;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tiles = p.B * p.subs, w = blockIdx.x;
  int4* const info = reinterpret_cast<int4*>(p.info);
  // the lanes count the steps of 64 tiles at a time (a head's); the first 64 are kept
  int n0 = 0, to0 = 0, total = 0, some = 0;           // some: tiles that have any
  for (int base = 0; base < tiles; base += 64) {
    const int i = base + lane, steps = i < tiles ? small_tile(p, i).steps : 0;
    if (i < tiles && steps == 0 && i % p.runs == w && wave == 0)
      for (int h = 0; h < p.c.heads; ++h) info[static_cast<int64_t>(i) * p.c.heads + h] = make_int4(0, 0, 0, 0);
    const int to = wave_scan(steps);
    if (base == 0) {
      n0 = steps;
      to0 = to;
    }
    total += __builtin_amdgcn_readlane(to, 63);
    some += __builtin_popcountll(__ballot(steps > 0));
  }
  total *= p.c.heads;
  if (total == 0) return;
  int runs, len, more = 0;                            // the first `more` runs are one longer
  const bool few = some * p.c.heads <= kFewTiles;
  auto pieces = [&](int n) {                          // runs of a tile, or its steps
    if (!few) return n;
    return len == kWaves ? (n + kWaves - 1) / kWaves : (n + len - 1) / len;        // few steps: no division
  };
  if (few) {
    // as long as the most workgroups allow, a sixteenth longer until their number is kept to
    constexpr int kMost = D == 64 ? kRuns : kRuns / 2;
    len = ((total - 1) / (kMost * kWaves) + 1) * kWaves;
    for (;;) {
      runs = 0;
      for (int base = 0; base < tiles; base += 64) {
        const int to = wave_scan(pieces(base ? (base + lane < tiles ? small_tile(p, base + lane).steps : 0) : n0));
        if (base == 0) to0 = to;
        runs += __builtin_amdgcn_readlane(to, 63) * p.c.heads;
      }
      if (runs <= kMost) break;
      len += (len / (16 * kWaves) + 1) * kWaves;
    }
  } else {
    runs = min(D == 256 ? kRuns / 2 : kRuns, (total + kWaves - 1) / kWaves);
    len = total / runs;
    more = total - len * runs;
  }
  if (w >= runs) return;
  const int u0 = w * len + min(w, more), u1 = u0 + len + (w < more ? 1 : 0);
  // the tile that holds step u0, and that tile's first step
  int index = 0, start = 0;
  for (int base = 0, before = 0; base < tiles; base += 64) {
    int n = n0, to = to0;
    if (base) n = base + lane < tiles ? small_tile(p, base + lane).steps : 0;
    n = pieces(n);
    if (base) to = wave_scan(n);
    const uint64_t here = __ballot((before + to) * p.c.heads > (few ? w : u0));    // the first such lane's tile
    if (here) {
      const int first = __builtin_ctzll(here);
      index = base + first;
      start = (before + __builtin_amdgcn_readlane(to - n, first)) * p.c.heads * (few ? len : 1);
      break;
    }
    before += __builtin_amdgcn_readlane(to, 63);
  }
  Tile t = uniform(small_tile(p, index));
  int all = few ? pieces(t.steps) * len : t.steps;                       // what the tile counts as
  int h = (u0 - start) / all, step = u0 - start - h * all;
  for (int u = u0; u < u1;) {
    const int steps = min(t.steps - step, u1 - u);
    attend_shared<D, TQ, kWaves>(p, t, h, step, steps, wave, look_up(p, t.b, t.lo, step + wave, kWaves), sh);
    __syncthreads();
    const int slot = 2 * w + (u == u0 ? 0 : 1);
    for (int k = threadIdx.x; k < min(kRowTile, t.rows - t.row0) * (D / 8); k += 64 * kWaves) {
      const int r = k / (D / 8), e = (k % (D / 8)) * 8;
      float f[8];
      const float2 ml = join_waves<D, kWaves>(sh, r, e, f);
      if (steps == t.steps) {
        put_row<D, TQ>(p, t, h, r, e, ml.y, f);
      } else {
        const int64_t at = static_cast<int64_t>(slot) * p.part_rows + r;
        store_out<8>(p.part + at * D + e, f);
        if (e == 0) *reinterpret_cast<float2*>(p.part_ml + 2 * at) = ml;
      }
    }
    if (step == 0 && threadIdx.x == 0) {
      // the tile starts here; its pieces end in the run that holds its last step
      const int last = u + all - 1, cut = (len + 1) * more;
      const int to = last < cut ? last / (len + 1) : more + (last - cut) / len;
      info[static_cast<int64_t>(index) * p.c.heads + h] = make_int4(to - w + 1, slot, t.q0, t.row0 << 8 | min(kRowTile, t.rows - t.row0));
    }
    u += steps;
    step = 0;
    if (few || u >= u1) break;
    if (++h == p.c.heads) {
      h = 0;
      do t = uniform(small_tile(p, ++index)); while (t.steps == 0);
      all = t.steps;
    }
    __syncthreads();
  }
}

// Joins the pieces of tile blockIdx.x (tile x head), row blockIdx.y, in their order:
// threads take four elements of every kJoin-th piece.  All that it has to know of
// the tile stands in its info: two trips to memory, not a chain of look-ups.
template <int D, typename TQ>
__global__ __launch_bounds__(kJoinThreads) void attn_join_kernel(AttnParams p) {
  constexpr int kJoin = kJoinThreads / (D / 4);
  __shared__ float4 part[kJoin][D / 4];
  __shared__ float len[kJoin];
  const int4 info = reinterpret_cast<const int4*>(p.info)[blockIdx.x];
  const int h = blockIdx.x % p.c.heads, r = blockIdx.y;
  const int n = info.x;
  if (n < 2 || r >= (info.w & 255)) return;
  const int first = info.y, w = first >> 1;
  auto row_of = [&](int k) { return static_cast<int64_t>(k ? 2 * (w + k) : first) * p.part_rows + r; };
  const int e = threadIdx.x % (D / 4), group = threadIdx.x / (D / 4);
  float M = -INFINITY;
  for (int k = threadIdx.x & 63; k < n; k += 64) M = fmaxf(M, p.part_ml[2 * row_of(k)]);
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) M = fmaxf(M, __shfl_xor(M, k));
  const float base = M == -INFINITY ? 0.0f : M;
  float L = 0.0f;
  float4 f = make_float4(0, 0, 0, 0);
#pragma unroll 4
  for (int k = group; k < n; k += kJoin) {
    const int64_t at = row_of(k);
    const float2 ml = *reinterpret_cast<const float2*>(p.part_ml + 2 * at);
    const float4 x = *reinterpret_cast<const float4*>(p.part + at * D + 4 * e);
    const float a = __builtin_amdgcn_exp2f(ml.x - base);
    L += a * ml.y;
    f.x += a * x.x; f.y += a * x.y; f.z += a * x.z; f.w += a * x.w;
  }
  part[group][e] = f;
  if (e == 0) len[group] = L;
  __syncthreads();
  if (threadIdx.x >= D / 8) return;
  L = 0.0f;
  float s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
  for (int k = 0; k < kJoin; ++k) {
    L += len[k];
    const float4 x = part[k][2 * threadIdx.x], y = part[k][2 * threadIdx.x + 1];
    s[0] += x.x; s[1] += x.y; s[2] += x.z; s[3] += x.w;
    s[4] += y.x; s[5] += y.y; s[6] += y.z; s[7] += y.w;
  }
  const float inv = L == 0.0f ? 0.0f : 1.0f / L;
#pragma unroll
  for (int i = 0; i < 8; ++i) s[i] *= inv;
  Tile t;
  t.q0 = info.z;
  t.row0 = info.w >> 8;
  store_out<8>(out_at<D, TQ>(p, t, h, r) + 8 * threadIdx.x, s);
}

// A workgroup takes a whole tile, its WAVES waves a share of its steps each, and
// joins them in shared memory.  large: the tiles of the sequences with many rows,
// found by counting them (their number is known on the device only).
template <int D, typename TQ, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void attn_tile_kernel(AttnParams p, int large) {
  __shared__ __attribute__((aligned(16))) Shared<D, WAVES> sh;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int index = blockIdx.x / p.c.heads;
  const int h = blockIdx.x - index * p.c.heads;
  if (!large && by_length(p)) {
    // Up to two workgroups for every compute unit: the longest sequences go first, and the
    // second workgroups take the others the other way round.  The waves look for the sequence
    // of that rank, each among its share of them.  32 + 8 heads of 128: 64 requests of 40 to
    // 4000 tokens 42 / 34.5 us, of 1000 to 8000 79 / 66; 64 of 4000 each 59.2 / 60.4 (in fp32
    // 72.6 / 76), of 300 9.8 / 9.8.  Where there are more workgroups they start as others end, and the order
    // (longest first) matters less than what it takes: 128 of 4000 107.5 / 110, of 500 to 4000 68.9 / 67.6.
    __shared__ int found;
    const int b = index / p.subs, first = 256 / (p.subs * p.c.heads);
    const int want = b < first ? b : p.B - 1 - (b - first);
    auto key_of = [&](int i) -> uint32_t {             // by length, then as they come; no two alike
      return i < p.B ? min(max(p.kv_len[i], 0), 1 << 28) / kUnit << 7 | (127 - i) : 0;
    };
    const uint32_t low = key_of(lane), high = key_of(lane + 64);
    for (int i = wave; i < p.B; i += WAVES) {
      const uint32_t mine = __builtin_amdgcn_readlane(i < 64 ? low : high, i & 63);
      if (__builtin_popcountll(__ballot(low > mine)) + __builtin_popcountll(__ballot(high > mine)) == want) found = i;
    }
    __syncthreads();
    index += (__builtin_amdgcn_readfirstlane(found) - b) * p.subs;
  }
  // the waves take steps in turn: their first pages are on their way while the tile's length is
  int pages = 0;
  if (!large && !p.window) pages = look_up(p, index / p.subs, 0, wave, WAVES);
  Tile t;
  if (large) {
    int b = -1, sub = 0;
    for (int base = 0, before = 0; base < p.B && b < 0; base += 64) {
      int n = 0;
      if (base + lane < p.B) {
        const int rows = min(queries_of(p, base + lane).n, p.max_q) * p.group;
        n = rows > kSmallRows ? (rows + kRowTile - 1) / kRowTile : 0;
      }
      const int to = wave_scan(n);
      const uint64_t here = __ballot(before + to > index);
      if (here) {
        const int at = __builtin_ctzll(here);
        b = base + at;
        sub = index - before - __builtin_amdgcn_readlane(to - n, at);
      }
      before += __builtin_amdgcn_readlane(to, 63);
    }
    if (b < 0) return;
    t = uniform(tile_of(p, b, sub));
  } else {
    t = uniform(small_tile(p, index));
  }
  if (t.steps == 0) return;
  if (large || p.window) pages = look_up(p, t.b, t.lo, wave, WAVES);
  attend_shared<D, TQ, WAVES>(p, t, h, 0, t.steps, wave, pages, sh);
  __syncthreads();
  for (int k = threadIdx.x; k < min(kRowTile, t.rows - t.row0) * (D / 8); k += 64 * WAVES) {
    const int r = k / (D / 8), e = (k % (D / 8)) * 8;
    float f[8];
    const float L = join_waves<D, WAVES>(sh, r, e, f).y;
    put_row<D, TQ>(p, t, h, r, e, L, f);
  }
}

template <int D, typename TQ, int WAVES>
void launch_tiles(const AttnParams& p, int64_t tiles, int large, hipStream_t s) {
  attn_tile_kernel<D, TQ, WAVES><<<static_cast<uint32_t>(tiles * p.c.heads), 64 * WAVES, 0, s>>>(p, large);
}

template <int D, typename TQ> hipError_t launch(const AttnParams& p, hipStream_t s) {
  const int64_t small = static_cast<int64_t>(p.B) * p.subs;
  if (p.whole) {
    launch_tiles<D, TQ, kWaves>(p, small, 0, s);
  } else {
    attn_runs_kernel<D, TQ><<<p.runs, 64 * kWaves, 0, s>>>(p);
    attn_join_kernel<D, TQ><<<dim3(static_cast<uint32_t>(small * p.c.heads), p.part_rows), kJoinThreads, 0, s>>>(p);
  }
  if (static_cast<int64_t>(p.max_q) * p.group > kSmallRows) {
    if constexpr (sizeof(TQ) == 2) return launch_attention_prompts(p, s);
    else launch_tiles<D, TQ, D == 256 ? 2 : 4>(p, p.large_tiles, 1, s);
  }
  return hipGetLastError();
}

}  // namespace

bool plan_attention(AttnParams* p, size_t* bytes) {
  const int64_t rows = static_cast<int64_t>(p->max_q) * p->group;
  p->subs = static_cast<int>((std::min<int64_t>(rows, kSmallRows) + kRowTile - 1) / kRowTile);
  p->part_rows = static_cast<int>(std::min<int64_t>(kRowTile, rows));
  // tiles of sequences with more rows than the small ones have
  p->large_tiles = (static_cast<int64_t>(p->T) * p->group + kRowTile - 1) / kRowTile +
                   std::min<int64_t>(p->B, static_cast<int64_t>(p->T) * p->group / kSmallRows);
  // a window's span: the tile's queries, and its start rounded down to a step
  int64_t span = p->max_kv;
  if (p->window) span = std::min<int64_t>(span, static_cast<int64_t>(p->window) + kRowTile + kUnit);
  const int64_t tiles = static_cast<int64_t>(p->B) * p->subs * p->c.heads;
  if (tiles > max_groups(64 * kWaves)) return false;
  if (rows > kSmallRows && p->dtype == CTS_F32 && p->large_tiles * p->c.heads > max_groups(256)) return false;
  const int64_t most_steps = std::max<int64_t>(1, (span + kUnit - 1) / kUnit), steps = tiles * most_steps;
  if (steps > 0x50000000) return false;               // counted in 32 bits, rounded up to runs by less than a half
  // A tile's steps taken by one workgroup need no join, but last as long as the longest
  // sequence does.  Measured at 32 + 8 heads of 128, whole tiles against runs: 1 request of
  // 1024 tokens 8.5 / 10.3 us, of 2048 12.4 / 10.0; 8 of 2000 13.3 / 13.4, of 4000 21 / 16;
  // 24 of 4000 34 / 39, of 8000 46 / 54 (of 1000 to 8000 40 / 33); 32 of 8000 56 / 66 (45 / 47);
  // 64 of 8000 106 / 114 (66 / 83).
  p->whole = span <= (tiles >= 256 ? 8192 : 1024 + 16 * tiles);
  // what the kernel makes at most, of a step or more for each wave
  p->runs = static_cast<int>(std::min<int64_t>(kRuns, tiles * ((most_steps + kWaves - 1) / kWaves)));
  // Few tiles of prompts over many tokens are split along the tokens.  32 + 8 heads of 128,
  // in one piece and so: 128 queries over 4000 tokens 101 / 37 us, 256 over 30000 761 / 170,
  // 512 over themselves 21 / 21 (24 with pieces of four steps).
  p->prompt_tiles = 0;
  p->pieces = 1;
  int64_t prompt_slots = 0;
  if (rows > kSmallRows && p->dtype == CTS_BF16) {
    const int64_t all = static_cast<int64_t>(p->T) * p->group;
    p->prompt_tiles = (all + kPromptRows - 1) / kPromptRows + std::min<int64_t>(p->B, all / kSmallRows);
    const int64_t groups = std::max<int64_t>(1, p->prompt_tiles * p->c.heads);
    if (groups > max_groups(kJoinThreads)) return false;             // (their kernel has as many threads)
    const int64_t most = std::max<int64_t>(1, span * p->c.d / 8192 / kPromptSteps);
    p->pieces = static_cast<int>(std::max<int64_t>(1, std::min(kPromptGroups / groups, most)));
    prompt_slots = std::min(kPromptGroups, groups * most);
  }
  // sums of two slots a run, their maxima and lengths, four numbers a tile; sums, maxima and lengths of prompts' pieces
  const size_t slots = static_cast<size_t>(2) * p->runs * p->part_rows + static_cast<size_t>(prompt_slots) * kPromptRows;
  *bytes = slots * (p->c.d + 2) * sizeof(float) + static_cast<size_t>(tiles) * 16;
  return true;
}

void place_attention(AttnParams* p, void* workspace) {
  const int64_t slots = static_cast<int64_t>(2) * p->runs * p->part_rows;
  const int64_t prompt = p->pieces > 1 ? p->prompt_tiles * p->c.heads * p->pieces * kPromptRows : 0;
  p->part = static_cast<float*>(workspace);
  p->prompt_part = p->part + slots * p->c.d;
  p->part_ml = p->prompt_part + prompt * p->c.d;
  p->prompt_ml = p->part_ml + slots * 2;
  p->info = reinterpret_cast<int32_t*>(p->prompt_ml + prompt * 2);
}

void describe_attention(const AttnParams& p, int32_t* plan) {
  plan[0] = !p.whole ? 2 : by_length(p) ? 1 : 0;
  plan[1] = p.whole ? 0 : kFewTiles;
  plan[2] = static_cast<int64_t>(p.max_q) * p.group > kSmallRows && p.dtype == CTS_BF16 ? p.pieces : 0;
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
