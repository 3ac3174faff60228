// C entry points of cts_block.h: argument checks (pure host code, no HIP call
// before every check has passed), plans and launches.
#include <algorithm>
#include <cmath>

#include "block_internal.h"
#include "cts_block.h"
#include "host_checks.h"

namespace {

using cts::misaligned;
using cts::overlap;
using cts::Range;
using cts::Rows;
using cts::same;

constexpr uint64_t kMaxCount = 0x7fffffffull;     // of rows x heads, and of sequences x heads
constexpr float kLog2e = 1.4426950408889634f;
constexpr int64_t kMaxLd = int64_t{1} << 28;      // extents of 2^31 rows stay below 2^63 bytes

uint64_t elt(int dtype) { return dtype == CTS_F32 ? 4 : 2; }
bool known(int dtype) { return dtype == CTS_F32 || dtype == CTS_BF16; }

// Rows of `width` elements, `ld` apart, that are read and written in 16-byte pieces.
bool bad_rows(const void* p, int64_t ld, int64_t width, int dtype) {
  return !p || misaligned(p, 16) || ld < width || ld > kMaxLd || (ld * static_cast<int64_t>(elt(dtype))) % 16 != 0;
}

Rows rows(const void* p, int64_t T, int64_t width, int64_t ld, int dtype) {
  const uint64_t e = elt(dtype);
  return {p, static_cast<uint64_t>(T), width * e, ld * e};
}

int status(hipError_t e) { return e == hipSuccess ? CTS_OK : CTS_ERR_HIP; }

int check_cache_sizes(const cts_kv_cache* c) {
  if (!c || c->n_pages < 1 || c->page_size < 1 || c->n_heads < 1 || c->head_dim < 1) return CTS_ERR_INVALID_ARG;
  if (c->page_size < 16 || c->page_size > 1024 || (c->page_size & (c->page_size - 1)) != 0 || c->n_heads > 4096 ||
      (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256))
    return CTS_ERR_UNSUPPORTED;
  return CTS_OK;
}

// The cache's four arrays as ranges; CTS_ERR_INVALID_ARG for a missing, misaligned or overlapping one.
int check_cache(const cts_kv_cache* c, cts::KvCache* k, Range* r) {
  const int e = check_cache_sizes(c);
  if (e != CTS_OK) return e;
  int shift = 0;
  while ((1 << shift) < c->page_size) ++shift;
  *k = {static_cast<uint8_t*>(c->k_codes), static_cast<uint8_t*>(c->k_scales), static_cast<uint8_t*>(c->v_codes),
        static_cast<uint8_t*>(c->v_scales), c->n_pages, shift, c->n_heads, c->head_dim};
  const size_t head_rows = (static_cast<size_t>(c->n_pages) << shift) * c->n_heads;
  r[0] = {c->k_codes, head_rows * (c->head_dim / 2)};
  r[1] = {c->k_scales, head_rows * (c->head_dim / 32)};
  r[2] = {c->v_codes, head_rows * (c->head_dim / 2)};
  r[3] = {c->v_scales, head_rows * (c->head_dim / 32)};
  for (int i = 0; i < 4; ++i) {
    if (!r[i].p || misaligned(r[i].p, 16)) return CTS_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j)
      if (overlap(r[i], r[j])) return CTS_ERR_INVALID_ARG;
  }
  return CTS_OK;
}

bool meets(Range out, const Range* in, int n) {
  for (int i = 0; i < n; ++i)
    if (overlap(out, in[i])) return true;
  return false;
}

// What cts_kv_write and cts_kv_read check alike: k and v in rows, the slots, the cache's four arrays.
int check_kv(const cts_kv_cache* c, int32_t T, const void* k, int64_t ldk, const void* v, int64_t ldv,
             const int64_t* slots, int32_t dtype, bool write, cts::KvCache* kc) {
  Range r[4];
  const int e = check_cache(c, kc, r);
  if (e != CTS_OK) return e;
  const int64_t width = static_cast<int64_t>(c->n_heads) * c->head_dim;
  if (bad_rows(k, ldk, width, dtype) || bad_rows(v, ldv, width, dtype) || !slots || misaligned(slots, 8))
    return CTS_ERR_INVALID_ARG;
  const Rows kr = rows(k, T, width, ldk, dtype), vr = rows(v, T, width, ldv, dtype);
  const Range sr{slots, 8ull * T};
  if (meets(extent(kr), r, 4) || meets(extent(vr), r, 4) || meets(sr, r, 4)) return CTS_ERR_INVALID_ARG;
  if (!write && (overlap(kr, vr) || overlap(extent(kr), sr) || overlap(extent(vr), sr))) return CTS_ERR_INVALID_ARG;
  if (!cts::kv_fits(*kc, T, write ? 8 : static_cast<int>(16 / elt(dtype)))) return CTS_ERR_UNSUPPORTED;
  return CTS_OK;
}

// Sizes of an attention problem, into a.
int attention_sizes(const cts_attn_problem* p, const cts_kv_cache* c, cts::AttnParams* a) {
  const int e = check_cache_sizes(c);
  if (e != CTS_OK) return e;
  if (!p || p->T < 0 || p->B < 0 || p->n_q_heads < 1 || p->max_pages < 1 || p->max_q < 1 || p->max_kv < 0 ||
      p->window < 0 || !(p->scale > 0.0f) || !std::isfinite(p->scale * kLog2e) || p->n_q_heads % c->n_heads != 0)
    return CTS_ERR_INVALID_ARG;
  if (!known(p->dtype) || p->n_q_heads > 65536 || p->max_q > (1 << 24) || p->max_kv > (1 << 30) || p->window > (1 << 30))
    return CTS_ERR_UNSUPPORTED;
  int shift = 0;
  while ((1 << shift) < c->page_size) ++shift;
  a->c = {static_cast<uint8_t*>(c->k_codes), static_cast<uint8_t*>(c->k_scales), static_cast<uint8_t*>(c->v_codes),
          static_cast<uint8_t*>(c->v_scales), c->n_pages, shift, c->n_heads, c->head_dim};
  a->T = p->T; a->B = p->B; a->heads = p->n_q_heads; a->group = p->n_q_heads / c->n_heads;
  a->max_pages = p->max_pages; a->max_q = p->max_q; a->window = p->window; a->dtype = p->dtype;
  const int64_t room = static_cast<int64_t>(p->max_pages) << shift;
  a->max_kv = static_cast<int>(std::min<int64_t>(p->max_kv, room));
  a->scale_log2e = p->scale * kLog2e;
  // (bounds that keep the plan's own arithmetic in 64 bits)
  if (static_cast<uint64_t>(p->B) * c->n_heads > kMaxCount || static_cast<uint64_t>(p->T) * p->n_q_heads > kMaxCount)
    return CTS_ERR_UNSUPPORTED;
  return CTS_OK;
}

// The same with the plan and the workspace's bytes.
int plan(const cts_attn_problem* p, const cts_kv_cache* c, cts::AttnParams* a, size_t* bytes) {
  const int e = attention_sizes(p, c, a);
  if (e != CTS_OK) return e;
  return cts::plan_attention(a, bytes) ? CTS_OK : CTS_ERR_UNSUPPORTED;
}

int plan(const cts_attn_problem* p, const cts_kv_cache* c, cts::TreeParams* a, size_t* bytes) {
  const int e = attention_sizes(p, c, a);
  if (e != CTS_OK) return e;
  return p->max_q <= cts::kTreeMaxQ && cts::plan_tree(a, bytes) ? CTS_OK : CTS_ERR_UNSUPPORTED;
}

// The arrays of an attention call, into a: r has room for 8 ranges, which out may not meet
// (the cache's, the table, the lengths, the rows and the workspace).
int attention_arrays(const cts_attn_problem* p, const cts_kv_cache* c, const void* q, int64_t ldq,
                     const int32_t* block_table, const int32_t* kv_len, const int32_t* q_start, void* out, int64_t ldo,
                     void* workspace, size_t workspace_bytes, cts::AttnParams* a, Range* r) {
  const int e = check_cache(c, &a->c, r);
  if (e != CTS_OK) return e;
  const int64_t width = static_cast<int64_t>(p->n_q_heads) * c->head_dim;
  if (bad_rows(q, ldq, width, p->dtype) || bad_rows(out, ldo, width, p->dtype) || !block_table || !kv_len ||
      misaligned(block_table, 4) || misaligned(kv_len, 4) || misaligned(q_start, 4) || !workspace ||
      misaligned(workspace, 16))
    return CTS_ERR_INVALID_ARG;
  const Rows qr = rows(q, p->T, width, ldq, p->dtype), orr = rows(out, p->T, width, ldo, p->dtype);
  r[4] = {block_table, 4ull * p->B * p->max_pages};
  r[5] = {kv_len, 4ull * p->B};
  r[6] = {q_start, q_start ? 4ull * (p->B + 1ull) : 0};
  r[7] = {workspace, workspace_bytes};
  if (meets(extent(orr), r, 8) || overlap(orr, qr) || meets(r[7], r, 7) || overlap(r[7], extent(qr)))
    return CTS_ERR_INVALID_ARG;
  a->q = q; a->ldq = ldq; a->out = out; a->ldo = ldo;
  a->table = block_table; a->kv_len = kv_len; a->q_start = q_start;
  return CTS_OK;
}

// Sizes and sections of a rotary call, into a; `heads` of its queries and keys.
int rotary_sizes(int32_t T, int32_t n_q_heads, int32_t n_k_heads, int32_t head_dim, int32_t rot_dim, int32_t dtype,
                 int32_t n_pos, int32_t n_axes, const int32_t* sections, int32_t interleaved, cts::RotaryParams* a) {
  if (T < 0 || n_q_heads < 0 || n_k_heads < 0 || n_q_heads + static_cast<int64_t>(n_k_heads) < 1 || head_dim < 1 ||
      rot_dim < 1 || rot_dim > head_dim || n_pos < 1 || n_axes < 1 || (n_axes > 1 && !sections))
    return CTS_ERR_INVALID_ARG;
  if (!known(dtype) || head_dim % 16 != 0 || rot_dim % 16 != 0 || head_dim > 4096 || n_axes > cts::kRotaryMaxAxes ||
      n_q_heads > 65536 || n_k_heads > 65536)
    return CTS_ERR_UNSUPPORTED;
  int64_t sum = 0;
  for (int i = 0; i < n_axes; ++i) {
    const int32_t n = sections ? sections[i] : rot_dim / 2;
    if (n < 0) return CTS_ERR_INVALID_ARG;
    sum += n;
    a->end[i] = static_cast<int>(std::min<int64_t>(sum, rot_dim / 2));
  }
  if (sum != rot_dim / 2) return CTS_ERR_INVALID_ARG;
  a->T = T; a->heads[0] = n_q_heads; a->heads[1] = n_k_heads; a->d = head_dim; a->rot = rot_dim; a->n_pos = n_pos;
  a->axes = n_axes; a->interleaved = interleaved != 0;
  return CTS_OK;
}

}  // namespace

extern "C" {

int cts_kv_write(const cts_kv_cache* c, int32_t T, const void* k, int64_t ldk, const void* v, int64_t ldv,
                 const int64_t* slots, int32_t dtype, void* stream) {
  if (T < 0) return CTS_ERR_INVALID_ARG;
  const int e = check_cache_sizes(c);
  if (e != CTS_OK) return e;
  if (!known(dtype)) return CTS_ERR_UNSUPPORTED;
  if (T == 0) return CTS_OK;
  cts::KvCache kc;
  const int e2 = check_kv(c, T, k, ldk, v, ldv, slots, dtype, true, &kc);
  if (e2 != CTS_OK) return e2;
  return status(cts::launch_kv_write(kc, T, k, ldk, v, ldv, slots, dtype, static_cast<hipStream_t>(stream)));
}

int cts_kv_read(const cts_kv_cache* c, int32_t T, const int64_t* slots, void* k, int64_t ldk, void* v, int64_t ldv,
                int32_t dtype, void* stream) {
  if (T < 0) return CTS_ERR_INVALID_ARG;
  const int e = check_cache_sizes(c);
  if (e != CTS_OK) return e;
  if (!known(dtype)) return CTS_ERR_UNSUPPORTED;
  if (T == 0) return CTS_OK;
  cts::KvCache kc;
  const int e2 = check_kv(c, T, k, ldk, v, ldv, slots, dtype, false, &kc);
  if (e2 != CTS_OK) return e2;
  return status(cts::launch_kv_read(kc, T, slots, k, ldk, v, ldv, dtype, static_cast<hipStream_t>(stream)));
}

size_t cts_kv_attention_workspace_size(const cts_attn_problem* p, const cts_kv_cache* c) {
  cts::AttnParams a{};
  size_t bytes = 0;
  return plan(p, c, &a, &bytes) == CTS_OK ? bytes : 0;
}

int cts_kv_attention_plan(const cts_attn_problem* p, const cts_kv_cache* c, int32_t* how) {
  cts::AttnParams a{};
  size_t bytes = 0;
  const int e = plan(p, c, &a, &bytes);
  if (e != CTS_OK) return e;
  if (!how) return CTS_ERR_INVALID_ARG;
  cts::describe_attention(a, how);
  return CTS_OK;
}

int cts_kv_attention(const cts_attn_problem* p, const cts_kv_cache* c, const void* q, int64_t ldq,
                     const int32_t* block_table, const int32_t* kv_len, const int32_t* q_start, void* out,
                     int64_t ldo, void* workspace, size_t workspace_bytes, void* stream) {
  cts::AttnParams a{};
  size_t need = 0;
  const int e = plan(p, c, &a, &need);
  if (e != CTS_OK) return e;
  if (!q_start && (p->max_q != 1 || p->T != p->B)) return CTS_ERR_INVALID_ARG;
  if (p->T == 0 || p->B == 0) return CTS_OK;
  Range r[8];
  const int e2 = attention_arrays(p, c, q, ldq, block_table, kv_len, q_start, out, ldo, workspace, workspace_bytes, &a, r);
  if (e2 != CTS_OK) return e2;
  if (workspace_bytes < need) return CTS_ERR_WORKSPACE;
  cts::place_attention(&a, workspace);
  return status(cts::launch_attention(a, static_cast<hipStream_t>(stream)));
}

int cts_block_norm(int32_t T, int32_t d, int32_t dtype, const void* x, int64_t ldx, const void* y, int64_t ldy,
                   const void* post_weight, const void* gate, int64_t ldg, float scale, float eps,
                   const void* weight, void* h, int64_t ldh, void* n, int64_t ldn, void* stream) {
  if (T < 0 || d < 1 || !std::isfinite(scale) || !(eps >= 0.0f) || !std::isfinite(eps)) return CTS_ERR_INVALID_ARG;
  if (!known(dtype) || d > cts::kNormMaxD) return CTS_ERR_UNSUPPORTED;
  if (T == 0) return CTS_OK;
  const uint64_t e = elt(dtype);
  auto bad = [&](const void* p, int64_t ld) { return !p || misaligned(p, e) || ld < d || ld > kMaxLd; };
  if (bad(x, ldx) || bad(weight, d) || bad(n, ldn)) return CTS_ERR_INVALID_ARG;
  if (y) {
    if (bad(y, ldy) || bad(h, ldh) || misaligned(post_weight, e) || (gate && bad(gate, ldg == 0 ? d : ldg)))
      return CTS_ERR_INVALID_ARG;
  } else if (post_weight || gate || h) {
    return CTS_ERR_INVALID_ARG;
  }
  const Rows xr = rows(x, T, d, ldx, dtype), yr = rows(y, T, d, ldy, dtype), hr = rows(h, T, d, ldh, dtype),
             nr = rows(n, T, d, ldn, dtype), gr = rows(gate, gate && ldg == 0 ? 1 : T, d, ldg == 0 ? d : ldg, dtype);
  const Range pr{post_weight, post_weight ? d * e : 0}, wr{weight, d * e};
  for (const Rows& o : {hr, nr}) {
    if (!o.p) continue;
    if ((!same(o, xr) && overlap(o, xr)) || (yr.p && !same(o, yr) && overlap(o, yr)) || (gr.p && overlap(o, gr)) ||
        overlap(extent(o), pr) || overlap(extent(o), wr))
      return CTS_ERR_INVALID_ARG;
  }
  if (hr.p && overlap(hr, nr)) return CTS_ERR_INVALID_ARG;
  const cts::NormParams a{T, d, x, y, post_weight, gate, weight, h, n, ldx, y ? ldy : 0, gate ? ldg : 0, h ? ldh : 0, ldn,
                          scale, eps};
  return status(cts::launch_block_norm(a, dtype, static_cast<hipStream_t>(stream)));
}

int cts_rotary(int32_t T, int32_t n_q_heads, int32_t n_k_heads, int32_t head_dim, int32_t rot_dim, int32_t dtype,
               const void* q, int64_t ldq, const void* k, int64_t ldk, const float* cos, const float* sin,
               int32_t n_pos, const int32_t* positions, int32_t n_axes, const int32_t* sections,
               int32_t interleaved, void* q_out, int64_t ldqo, void* k_out, int64_t ldko, void* stream) {
  cts::RotaryParams a{};
  const int e = rotary_sizes(T, n_q_heads, n_k_heads, head_dim, rot_dim, dtype, n_pos, n_axes, sections, interleaved, &a);
  if (e != CTS_OK) return e;
  if (T == 0) return CTS_OK;
  const int64_t wq = static_cast<int64_t>(n_q_heads) * head_dim, wk = static_cast<int64_t>(n_k_heads) * head_dim;
  if ((wq && (bad_rows(q, ldq, wq, dtype) || bad_rows(q_out, ldqo, wq, dtype))) ||
      (wk && (bad_rows(k, ldk, wk, dtype) || bad_rows(k_out, ldko, wk, dtype))) || !cos || !sin || !positions ||
      misaligned(cos, 16) || misaligned(sin, 16) || misaligned(positions, 4))
    return CTS_ERR_INVALID_ARG;
  const Rows none{nullptr, 0, 0, 0};
  const Rows qi = wq ? rows(q, T, wq, ldq, dtype) : none, ki = wk ? rows(k, T, wk, ldk, dtype) : none;
  const Rows qo = wq ? rows(q_out, T, wq, ldqo, dtype) : none, ko = wk ? rows(k_out, T, wk, ldko, dtype) : none;
  const size_t table = 2ull * rot_dim * n_pos;
  const Range in[3] = {{cos, table}, {sin, table}, {positions, 4ull * n_axes * T}};
  if ((!same(qo, qi) && overlap(qo, qi)) || (!same(ko, ki) && overlap(ko, ki)) || overlap(qo, ki) || overlap(ko, qi) ||
      overlap(qo, ko) || meets(extent(qo), in, 3) || meets(extent(ko), in, 3))
    return CTS_ERR_INVALID_ARG;
  a.in[0] = q; a.ldi[0] = ldq; a.in[1] = k; a.ldi[1] = ldk;
  a.out[0] = q_out; a.ldo[0] = ldqo; a.out[1] = k_out; a.ldo[1] = ldko;
  a.cos = cos; a.sin = sin; a.pos = positions;
  return status(cts::launch_rotary(a, dtype, static_cast<hipStream_t>(stream)));
}

size_t cts_kv_tree_attention_workspace_size(const cts_attn_problem* p, const cts_kv_cache* c) {
  cts::TreeParams a{};
  size_t bytes = 0;
  return plan(p, c, &a, &bytes) == CTS_OK ? bytes : 0;
}

int cts_kv_tree_attention_plan(const cts_attn_problem* p, const cts_kv_cache* c, int32_t* how) {
  cts::TreeParams a{};
  size_t bytes = 0;
  const int e = plan(p, c, &a, &bytes);
  if (e != CTS_OK) return e;
  if (!how) return CTS_ERR_INVALID_ARG;
  how[0] = a.tile_rows;
  how[1] = a.cut ? 2 : a.ordered ? 1 : 0;
  how[2] = a.waves;
  return CTS_OK;
}

int cts_kv_tree_attention(const cts_attn_problem* p, const cts_kv_cache* c, const void* q, int64_t ldq,
                          const int32_t* block_table, const int32_t* kv_len, const int32_t* q_start, const uint32_t* mask,
                          int64_t mask_words, const int32_t* positions, void* out, int64_t ldo, void* workspace,
                          size_t workspace_bytes, void* stream) {
  cts::TreeParams a{};
  size_t need = 0;
  const int e = plan(p, c, &a, &need);
  if (e != CTS_OK) return e;
  if (!q_start && (p->max_q != 1 || p->T != p->B)) return CTS_ERR_INVALID_ARG;
  if (mask_words < (p->max_q + 31) / 32 || mask_words > kMaxLd) return CTS_ERR_INVALID_ARG;
  if (p->T == 0 || p->B == 0) return CTS_OK;
  Range r[8];
  const int e2 = attention_arrays(p, c, q, ldq, block_table, kv_len, q_start, out, ldo, workspace, workspace_bytes, &a, r);
  if (e2 != CTS_OK) return e2;
  if (!mask || misaligned(mask, 4) || (p->window && !positions) || misaligned(positions, 4)) return CTS_ERR_INVALID_ARG;
  const Range more[2] = {{mask, 4ull * p->T * static_cast<uint64_t>(mask_words)},
                         {positions, p->window ? 4ull * p->T : 0}};
  const int64_t width = static_cast<int64_t>(p->n_q_heads) * c->head_dim;
  if (meets(extent(rows(out, p->T, width, ldo, p->dtype)), more, 2) || meets(r[7], more, 2)) return CTS_ERR_INVALID_ARG;
  if (workspace_bytes < need) return CTS_ERR_WORKSPACE;
  a.mask = mask; a.mask_words = mask_words; a.positions = positions;
  cts::place_tree(&a, workspace);
  return status(cts::launch_tree(a, static_cast<hipStream_t>(stream)));
}

int cts_kv_keep(const cts_kv_cache* c, int32_t B, int32_t max_pages, const int32_t* block_table, const int32_t* kv_len,
                const int32_t* q_start, int32_t max_path, const int32_t* path, const int32_t* n_path, void* stream) {
  if (B < 0 || max_pages < 1 || max_path < 0) return CTS_ERR_INVALID_ARG;
  const int e = check_cache_sizes(c);
  if (e != CTS_OK) return e;
  if (max_path > cts::kKeepMaxPath) return CTS_ERR_UNSUPPORTED;
  if (B == 0 || max_path == 0) return CTS_OK;
  cts::KvCache kc;
  Range r[4];
  const int e2 = check_cache(c, &kc, r);
  if (e2 != CTS_OK) return e2;
  for (const void* p : {block_table, kv_len, q_start, path, n_path})
    if (!p || misaligned(p, 4)) return CTS_ERR_INVALID_ARG;
  const Range in[5] = {{block_table, 4ull * B * max_pages}, {kv_len, 4ull * B}, {q_start, 4ull * (B + 1ull)},
                       {path, 4ull * B * max_path}, {n_path, 4ull * B}};
  for (const Range& a : in)
    if (meets(a, r, 4)) return CTS_ERR_INVALID_ARG;
  if (!cts::keep_fits(kc, B)) return CTS_ERR_UNSUPPORTED;
  return status(cts::launch_kv_keep(kc, B, max_pages, block_table, kv_len, q_start, path, n_path, max_path,
                                    static_cast<hipStream_t>(stream)));
}

int cts_kv_append(const cts_kv_cache* c, int32_t T, int32_t n_q_heads, int32_t rot_dim, int32_t dtype, const void* q,
                  int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, const int64_t* slots,
                  const float* cos, const float* sin, int32_t n_pos, const int32_t* positions, int32_t n_axes,
                  const int32_t* sections, int32_t interleaved, void* q_out, int64_t ldqo, void* k_out, int64_t ldko,
                  void* stream) {
  const int e = check_cache_sizes(c);
  if (e != CTS_OK) return e;
  cts::RotaryParams a{};
  const int e2 = rotary_sizes(T, n_q_heads, c->n_heads, c->head_dim, rot_dim, dtype, n_pos, n_axes, sections, interleaved, &a);
  if (e2 != CTS_OK) return e2;
  if (T == 0) return CTS_OK;
  cts::KvCache kc;
  const int e3 = check_kv(c, T, k, ldk, v, ldv, slots, dtype, true, &kc);
  if (e3 != CTS_OK) return e3;
  const int64_t wq = static_cast<int64_t>(n_q_heads) * c->head_dim, wk = static_cast<int64_t>(c->n_heads) * c->head_dim;
  if ((wq && (bad_rows(q, ldq, wq, dtype) || bad_rows(q_out, ldqo, wq, dtype))) || (k_out && bad_rows(k_out, ldko, wk, dtype)) ||
      !cos || !sin || !positions || misaligned(cos, 16) || misaligned(sin, 16) || misaligned(positions, 4))
    return CTS_ERR_INVALID_ARG;
  const Rows none{nullptr, 0, 0, 0};
  const Rows qi = wq ? rows(q, T, wq, ldq, dtype) : none, qo = wq ? rows(q_out, T, wq, ldqo, dtype) : none;
  const Rows ki = rows(k, T, wk, ldk, dtype), vi = rows(v, T, wk, ldv, dtype);
  const Rows ko = k_out ? rows(k_out, T, wk, ldko, dtype) : none;
  const size_t table = 2ull * rot_dim * n_pos;
  Range r[4];
  check_cache(c, &kc, r);
  const Range in[4] = {{cos, table}, {sin, table}, {positions, 4ull * n_axes * T}, {slots, 8ull * T}};
  if ((!same(qo, qi) && overlap(qo, qi)) || (!same(ko, ki) && overlap(ko, ki)) || overlap(qo, ki) || overlap(qo, vi) ||
      overlap(ko, qi) || overlap(ko, vi) || overlap(qo, ko) || meets(extent(qi), r, 4))
    return CTS_ERR_INVALID_ARG;
  for (const Rows& o : {qo, ko})
    if (meets(extent(o), in, 4) || meets(extent(o), r, 4)) return CTS_ERR_INVALID_ARG;
  for (const Range& i : in)
    if (meets(i, r, 4)) return CTS_ERR_INVALID_ARG;
  a.in[0] = q; a.ldi[0] = ldq; a.in[1] = k; a.ldi[1] = ldk;
  a.out[0] = q_out; a.ldo[0] = ldqo; a.out[1] = k_out; a.ldo[1] = ldko;
  a.cos = cos; a.sin = sin; a.pos = positions;
  if (!cts::append_fits(kc, a)) return CTS_ERR_UNSUPPORTED;
  return status(cts::launch_kv_append(kc, a, v, ldv, slots, dtype, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
