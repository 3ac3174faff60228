/*
 * cts_block.h -- C ABI of what a decoder block needs around its multi-adapter
 * layers (cts.h): a paged key/value cache held in 4 bits with its writes and
 * reads, the attention over it, the norms around a block with its residual,
 * and rotary positions.  A block then runs
 *   block_norm -> q/k/v layers -> rotary -> kv_write -> kv_attention -> o layer
 *   -> block_norm -> gate/up layers -> (activation) -> down layer -> block_norm
 *
 * Conventions are those of cts.h: array pointers are device memory owned by
 * the caller, structs and `sections` are host memory read during the call,
 * nothing is allocated or synchronised, calls only enqueue work on `stream`,
 * every argument error is found on the host before any HIP call, T == 0 is
 * a no-op, and a call of more work than a launch has threads for (137 GB of keys
 * to write, 2^23 sequences x heads to attend to) is CTS_ERR_UNSUPPORTED.  Arrays are 16-byte aligned (int32 arrays 4, int64 arrays 8) and
 * rows of elements may lie further apart than they are long, as the slices of a
 * packed q/k/v output do: ld* are row strides in elements, multiples of 16
 * bytes, at least the row's length and at most 2^28.  dtype is CTS_BF16 or
 * CTS_F32.
 */
#ifndef CTS_BLOCK_H
#define CTS_BLOCK_H

#include "cts.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A layer's cache: n_pages pages of page_size tokens (a power of two, 16 ..
 * 1024), n_heads key/value heads of head_dim (64, 128 or 256) elements.
 * Each 32 elements along head_dim share a scale byte s; an element is a 4-bit
 * code, bit 3 the sign and the rest the magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6,
 * standing for magnitude x 2^(s - 127) (a microscaled 4-bit float), s at most 252; a
 * block with s == 255 is NaN throughout.  253 and 254 are no scales of a token that
 * is read (some of their magnitudes lie past the largest float).  Bytes:
 *   k_codes  [n_pages][n_heads][page_size][head_dim / 2]        element 2i in byte i's low half
 *   k_scales [n_pages][n_heads][page_size][head_dim / 32]
 *   v_codes  [n_pages][n_heads][page_size / 4][head_dim / 8][4][4]   8 elements of 4 tokens in 16 bytes
 *   v_scales [n_pages][n_heads][page_size / 4][head_dim / 32][4]
 * (values lie in groups of four tokens because their product runs over the
 * tokens: a lane's one load then brings it four of them). */
typedef struct {
    int32_t n_pages, page_size, n_heads, head_dim;
    void *k_codes, *k_scales, *v_codes, *v_scales;
} cts_kv_cache;

/* Quantises T tokens' keys and values, k and v [T][n_heads][head_dim] of
 * `dtype` with rows ldk and ldv apart, into the slots slots[t] = page *
 * page_size + offset (int64).  A slot that is negative or past the cache is
 * skipped (padding); equal slots in one call leave either token, or parts of
 * both.  Of a block of 32, s is chosen so that the largest magnitude rounds to 6
 * at most, s = exponent(largest, its mantissa rounded up from 1.75) - 2, held to
 * [1, 252]; each element is rounded to the nearest magnitude, ties to the even
 * code.  A block that holds a NaN or an infinity gets s = 255 and reads as NaN
 * throughout.  Magnitudes past 6 x 2^125 are held as that. */
int cts_kv_write(const cts_kv_cache* c, int32_t T, const void* k, int64_t ldk, const void* v, int64_t ldv,
                 const int64_t* slots, int32_t dtype, void* stream);

/* The values that the cache holds for T slots, into k and v (layouts as for
 * cts_kv_write; both types represent them exactly).  A slot outside the cache
 * gives a row of zeros. */
int cts_kv_read(const cts_kv_cache* c, int32_t T, const int64_t* slots, void* k, int64_t ldk, void* v, int64_t ldv,
                int32_t dtype, void* stream);

/* Causal attention of T query rows over the cached tokens of B sequences.
 * Sequence b's token t lies in page block_table[b][t / page_size] (int32
 * [B][max_pages]); kv_len[b] (int32) counts its cached tokens, those of this
 * call's queries (written before it) among them.  Its queries are the rows
 * q_start[b] .. q_start[b + 1] - 1 (int32 [B + 1]); q_start == NULL means one
 * query a sequence (T == B, max_q == 1).  Query j of n sits at position P =
 * kv_len[b] - n + j and sees the tokens max(0, P - window + 1) .. P (window ==
 * 0: all from the first).  For each query head h, with key/value head h /
 * (n_q_heads / n_heads):
 *     out[h] = sum_t w_t v_t,   w = softmax_t(scale q[h] . k_t)
 * A query that sees nothing (P < 0, kv_len 0) gives zeros.  q and out are
 * [T][n_q_heads][head_dim] of dtype, rows ldq and ldo apart.
 * Arithmetic: scores, softmax and sums in fp32.  Cached elements are exact in
 * bf16 (bf16 matrix cores).  bf16: the weights w are rounded to bf16 for the
 * product with v, and their sum is that of the rounded ones (2^-8 each at most, the size
 * of the output's own rounding); f32: queries and weights are split into three
 * bf16 parts, which keep their 24 bits.
 * What is masked is never read into a result, whatever bytes stand there, NaN and
 * scales of 253 and 254 included.
 * max_q and max_kv bound the queries of a sequence and kv_len.  A kv_len past
 * max_kv, or past the table's max_pages, counts as that (P with it), one below 0
 * as 0; queries past max_q, and rows of no sequence, are left out (out keeps what it held there).
 * They choose how the work is split and size the workspace.  A page number
 * outside [0, n_pages) reads as NaN; row and length arrays are clamped, so no
 * content makes a call read or write outside its arrays. */
typedef struct {
    int32_t T;            /* query rows */
    int32_t B;            /* sequences */
    int32_t n_q_heads;    /* a multiple of the cache's n_heads */
    int32_t max_pages;    /* columns of block_table */
    int32_t max_q;        /* queries of a sequence, at most */
    int32_t max_kv;       /* kv_len, at most */
    int32_t window;       /* 0: none */
    int32_t dtype;        /* cts_dtype of q and out */
    float scale;          /* > 0 and at most 2^127, commonly head_dim^-1/2 */
} cts_attn_problem;

/* Bytes of device workspace cts_kv_attention needs (0 for a problem it would
 * refuse): the sizes of `c` count, not its pointers.  It does not fall as T,
 * B, max_q or max_kv grow, and a window never needs more than none. */
size_t cts_kv_attention_workspace_size(const cts_attn_problem* p, const cts_kv_cache* c);

/* How a call with these sizes takes its sequences, for tests and debugging; plan
 * is a host array of 3 entries:
 *   [0] tiles of 16 query rows (sequences of up to 64 rows of a key/value head, all in
 *       f32): 0 a workgroup each, 1 the same by the sequences' lengths, 2 their
 *       steps are dealt out in runs
 *   [1] with 2: tiles (times heads, of those that have rows) up to which each is cut
 *       into runs of its own; with more, runs go from tile to tile
 *   [2] pieces that the tokens of the other sequences' tiles are split into (0:
 *       max_q allows no such sequence, or f32)
 * Errors as for the call's sizes. */
int cts_kv_attention_plan(const cts_attn_problem* p, const cts_kv_cache* c, int32_t* plan);

int cts_kv_attention(const cts_attn_problem* p, const cts_kv_cache* c, const void* q, int64_t ldq,
                     const int32_t* block_table, const int32_t* kv_len, const int32_t* q_start, void* out,
                     int64_t ldo, void* workspace, size_t workspace_bytes, void* stream);

/* The norms around a block, with its gate, residual scale and residual.  For
 * every token, N(a) = a / sqrt(mean(a^2) + eps) over its d elements:
 *     u = N(y) * post_weight            (post_weight NULL: u = y)
 *     h = x + scale * gate * u          (gate NULL: without it)
 *     n = N(h) * weight
 * x is the residual stream before the block, y the block's output, h the
 * stream after it and n the next block's input.  y == NULL: n = N(x) * weight
 * alone (the first norm; post_weight, gate and h are NULL then).
 * x, y, h, n [T][d] with rows ldx, ldy, ldh, ldn apart; weights [d]; gate [d]
 * for all tokens (ldg == 0) or [T][d] with rows ldg apart.  All of `dtype`, any
 * d from 1 to 32768 and any strides (d and all strides and addresses multiples of 16
 * bytes are read in 16-byte pieces, others element by element); arrays are
 * aligned to their elements.  Sums and products are in fp32; h and n are
 * each rounded once (n from the unrounded h).  h may be x or y itself and n y
 * itself (same address and stride); otherwise outputs overlap nothing. */
int cts_block_norm(int32_t T, int32_t d, int32_t dtype, const void* x, int64_t ldx, const void* y, int64_t ldy,
                   const void* post_weight, const void* gate, int64_t ldg, float scale, float eps,
                   const void* weight, void* h, int64_t ldh, void* n, int64_t ldn, void* stream);

/* Rotary positions of queries and keys, q [T][n_q_heads][head_dim] and k
 * [T][n_k_heads][head_dim] (either count may be 0, its pointers then NULL).
 * The first rot_dim elements of a head (a multiple of 16) form rot_dim / 2
 * pairs: elements j and j + rot_dim / 2, or with `interleaved` 2j and 2j + 1.
 * Pair j of token t turns by the angle whose cosine and sine stand in row
 * positions[a][t], column j of cos and sin (fp32 [n_pos][rot_dim / 2]), a the
 * axis that j belongs to:
 *     (x1, x2) -> (x1 cos - x2 sin, x2 cos + x1 sin)
 * positions is int32 [n_axes][T] (1 to 4 axes: a text's one, or time, height
 * and width); sections (host, n_axes counts that sum to rot_dim / 2) gives each
 * axis its pairs, in order; NULL with one axis.  Elements past rot_dim are
 * copied.  Products and sums are in fp32, rounded once.  A position outside
 * the table is clamped into it.  Outputs may be the inputs themselves (same address
 * and stride), otherwise they overlap nothing. */
int cts_rotary(int32_t T, int32_t n_q_heads, int32_t n_k_heads, int32_t head_dim, int32_t rot_dim, int32_t dtype,
               const void* q, int64_t ldq, const void* k, int64_t ldk, const float* cos, const float* sin,
               int32_t n_pos, const int32_t* positions, int32_t n_axes, const int32_t* sections,
               int32_t interleaved, void* q_out, int64_t ldqo, void* k_out, int64_t ldko, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* CTS_BLOCK_H */
