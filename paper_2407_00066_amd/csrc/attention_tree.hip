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
#include <algorithm>

#include "attention_common.h"

namespace cts {
namespace {

constexpr int kMaskRow = kTreeMaxQ / 32 + 2;

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

template <int D, int RG, int WAVES> struct TreeShared {
  uint32_t mask[RG * kRowTile][kMaskRow];          // of the tile's queries
  float sums[WAVES][kRowTile][D + 4];
  float2 ml[WAVES][kRowTile];
};

// Page number of the lane's group of 16 tokens in the steps s0, s0 + stride, ..: two
// groups a step, a lane one.
__device__ __forceinline__ int look_up(const TreeParams& p, int b, int lo, int s0, int stride) {
  const int lane = threadIdx.x & 63;
  const int64_t tok = lo + static_cast<int64_t>(s0 + (lane >> 1) * stride) * kUnit + 16 * (lane & 1);
  return p.table[static_cast<int64_t>(b) * p.max_pages + min(tok >> p.c.page_shift, static_cast<int64_t>(p.max_pages - 1))];
}

// The bits of the tile's queries, into shared memory; those of drafts that do not count are 0.
template <int ROWS> __device__ __forceinline__ void load_masks(const TreeParams& p, const TreeTile& t, uint32_t (*mask)[kMaskRow]) {
  const int first = t.row0 / p.group, last = (min(t.rows, t.row0 + ROWS) - 1) / p.group;
  const int words = (t.drafts + 31) / 32, wide = words + 2;
  for (int k = threadIdx.x; k < (last - first + 1) * wide; k += blockDim.x) {
    const int q = k / wide, w = k - q * wide - 1;
    uint32_t bits = w < 0 ? ~0u : 0u;
    if (w >= 0 && w < words) {
      bits = p.mask[static_cast<int64_t>(t.q0 + first + q) * p.mask_words + w];
      const int left = t.drafts - 32 * w;
      if (left < 32) bits &= (1u << left) - 1;
    }
    mask[q][w + 1] = bits;
  }
}

// `count` of the tile's steps from s0, `stride` apart, for key/value head h, by one
// wave; pages: look_up of the first 32.  The workgroup meets once, for the masks.
template <int D, typename TQ, int RG, int stride>
__device__ __forceinline__ void attend(const TreeParams& p, const TreeTile& t, int h, int s0, int count, int pages,
                                       uint32_t (*mask)[kMaskRow], Sums<D>* st) {
  constexpr int NS = sizeof(TQ) == 4 ? 3 : 1;      // bf16 parts of a query and of a weight
  constexpr int KS = D / 32;                     // steps of the first product; words of keys a lane holds
  constexpr int NC = Sums<D>::NC, NB = Sums<D>::NB;
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;

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
  const bool any = count > 0 && t.hi > t.lo;
  if (any) {
    load_k(0);
    load_v();
  }

  // the lane's rows: which bits are theirs, and the first token before the drafts that they see
  int q_of[RG], first[RG];
  bf16x8 qf[RG][KS][NS];
#pragma unroll
  for (int r = 0; r < RG; ++r) {
    const int row = t.row0 + kRowTile * r + n;
    const bool live = row < t.rows;
    const int query = (live ? row : t.row0) / p.group;
    q_of[r] = query - t.row0 / p.group;
    first[r] = p.window && live ? min(max(p.positions[t.q0 + query], t.past) - p.window + 1, t.past) : 0;
    const TQ* q = static_cast<const TQ*>(p.q) + (live ? (t.q0 + query) * p.ldq +
                                                 static_cast<int64_t>(h * p.group + row - query * p.group) * D : 0);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      float f[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      if (live) load_q(q + (D / 4) * g + 8 * s, f);
      split<NS>(f, qf[r][s]);
    }
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < NB; ++e) st[r].o[c][e] = f32x4{0, 0, 0, 0};
    st[r].m = -INFINITY;
    st[r].l = 0.0f;
  }
  // tokens from here on every row sees, as far as windows go
  int all_lo = 0;
  if (p.window) {
#pragma unroll
    for (int r = 0; r < RG; ++r) all_lo = max(all_lo, first[r]);
#pragma unroll
    for (int x = 1; x < 16; x <<= 1) all_lo = max(all_lo, __shfl_xor(all_lo, x));
    all_lo = __builtin_amdgcn_readfirstlane(all_lo);
  }
  __syncthreads();                                                      // the masks are there
  if (!any) return;

  for (int it = 0; it < count; ++it) {
    const int at = t.lo + (s0 + it * stride) * kUnit;
    // scores of the lane's rows against tokens at + 16 i + 4 g + j
    f32x4 x[RG][2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int r = 0; r < RG; ++r) x[r][i] = f32x4{0, 0, 0, 0};
      const uint32_t units = ks[i] | gr[i].bad;                          // here: asked for sooner, it would be waited for sooner
#pragma unroll
      for (int y = 0; y < KS; ++y) {
        const float unit = unit_of(units, D == 256 ? y / 4 : 0);
        const bf16x8 a = frag(fp4_pair(k[i][y], unit, 0), fp4_pair(k[i][y], unit, 1),
                              fp4_pair(k[i][y], unit, 2), fp4_pair(k[i][y], unit, 3));
#pragma unroll
        for (int r = 0; r < RG; ++r)
#pragma unroll
          for (int z = 0; z < NS; ++z) x[r][i] = mfma(a, qf[r][y][z], x[r][i]);
      }
    }
    // the next keys are on their way during the softmax and the second product,
    // the next values during the next first product (past the end: the last step's again)
    const int next = min(it + 1, count - 1);
    if ((next & 31) == 0 && next != 0) pages = rare(look_up(p, t.b, t.lo, s0 + next * stride, stride));
    load_k(next);

    const bool masked = at + kUnit > t.past || at < all_lo;              // the same for the whole wave
    // which of tokens at + 4 g .. a row sees (bit 16 i + j)
    auto seen_by = [&](int r) -> uint32_t {
      const int from = rare(max(at - t.past, -kUnit));
      const uint32_t* const w = &mask[q_of[r]][(from >> 5) + 1];
      uint32_t bits = static_cast<uint32_t>((static_cast<uint64_t>(w[1]) << 32 | w[0]) >> (from & 31));
      const int hide = first[r] - at;                                    // tokens that a window hides
      if (hide > 0) bits &= hide < 32 ? ~0u << hide : 0u;
      return bits >> (4 * g);
    };
    bf16x8 pf[RG][NS];
#pragma unroll
    for (int r = 0; r < RG; ++r) {
      float sc[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) sc[i] = x[r][i >> 2][i & 3] * p.scale_log2e;
      if (masked) {
        const uint32_t bits = seen_by(r);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (!(bits >> (16 * i + j) & 1)) sc[4 * i + j] = -INFINITY;
      }
      float top = sc[0];
#pragma unroll
      for (int i = 1; i < 8; ++i) top = fmaxf(top, sc[i]);
      top = max_over_groups(top);
      if (__any(top > st[r].m + kSlack)) {
        // (only the rows that have grown follow, so that no row's bits depend on another's)
        const float m_new = top > st[r].m + kSlack ? top : st[r].m;
        const float fade = __builtin_amdgcn_exp2f(st[r].m - (m_new == -INFINITY ? 0.0f : m_new));
        st[r].l *= fade;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int e = 0; e < NB; ++e) st[r].o[c][e] *= fade;
        st[r].m = m_new;
      }
      const float base = st[r].m == -INFINITY ? 0.0f : st[r].m;
      float w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        w[i] = __builtin_amdgcn_exp2f(sc[i] - base);
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
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (past_scales(vs[i][c], j)) {
                vs[i][c] ^= 0x80u << (8 * j);                            // 255 -> 127
                (&v[i][c].x)[j] = 0;
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
        for (int r = 0; r < RG; ++r)
#pragma unroll
          for (int z = 0; z < NS; ++z) {
            st[r].o[c][2 * e] = mfma(even, pf[r][z], st[r].o[c][2 * e]);
            st[r].o[c][2 * e + 1] = mfma(odd, pf[r][z], st[r].o[c][2 * e + 1]);
          }
      }
    }
    load_v();
  }
#pragma unroll
  for (int r = 0; r < RG; ++r) st[r].l = sum_over_groups(st[r].l);
}

// Eight elements of a row, from e: the waves' sums together, their maximum and length.
template <int D, int RG, int WAVES>
__device__ __forceinline__ float2 join_waves(const TreeShared<D, RG, WAVES>& sh, int r, int e, float* f) {
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

template <int D, typename TQ, int RG>
__global__ __launch_bounds__(64 * kWaves) void tree_kernel(TreeParams p) {
  __shared__ __attribute__((aligned(16))) TreeShared<D, RG, kWaves> sh;
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int index = blockIdx.x / p.c.heads, h = blockIdx.x - index * p.c.heads;
  const int b = index / p.subs, sub = index - b * p.subs;
  const TreeTile t = uniform(tree_tile(p, b, sub));
  if (t.steps == 0) return;
  load_masks<RG * kRowTile>(p, t, sh.mask);
  Sums<D> st[RG];
  const int count = wave < t.steps ? (t.steps - wave + kWaves - 1) / kWaves : 0;
  attend<D, TQ, RG, kWaves>(p, t, h, wave, count, look_up(p, b, t.lo, wave, kWaves), sh.mask, st);
#pragma unroll
  for (int r = 0; r < RG; ++r) {
    if (r) __syncthreads();
#pragma unroll
    for (int c = 0; c < Sums<D>::NC; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float f[Sums<D>::NB];
#pragma unroll
        for (int e = 0; e < Sums<D>::NB; ++e) f[e] = st[r].o[c][e][i];
        store_out<Sums<D>::NB>(sh.sums[wave][n] + Sums<D>::element(g, c, i), f);
      }
    if (g == 0) sh.ml[wave][n] = make_float2(st[r].m, st[r].l);
    __syncthreads();
    const int row0 = t.row0 + kRowTile * r;
    for (int k = threadIdx.x; k < min(kRowTile, t.rows - row0) * (D / 8); k += 64 * kWaves) {
      const int at = k / (D / 8), e = (k % (D / 8)) * 8;
      float f[8];
      const float L = join_waves<D, RG, kWaves>(sh, at, e, f).y;
      const float inv = L == 0.0f ? 0.0f : 1.0f / L;
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] *= inv;
      const int row = row0 + at, query = row / p.group;
      store_out<8>(static_cast<TQ*>(p.out) + (t.q0 + query) * p.ldo +
                       static_cast<int64_t>(h * p.group + row - query * p.group) * D + e, f);
    }
  }
}

template <int D, typename TQ> hipError_t launch(const TreeParams& p, hipStream_t s) {
  const uint32_t groups = static_cast<uint32_t>(static_cast<int64_t>(p.B) * p.subs * p.c.heads);
  tree_kernel<D, TQ, 1><<<groups, 64 * kWaves, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace

bool plan_tree(TreeParams* p, size_t* bytes) {
  const int64_t rows = static_cast<int64_t>(p->max_q) * p->group;
  p->tile_rows = kRowTile;
  p->subs = static_cast<int>((rows + kRowTile - 1) / kRowTile);
  *bytes = 16;
  return static_cast<int64_t>(p->B) * p->subs * p->c.heads <= max_groups(64 * kWaves);
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
