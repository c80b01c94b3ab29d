/*
 * evospec_decode.h -- what a decode step does around the restricted head of evospec.h: a key/value cache held in
 * 8 bits (written, read back, attended over by single tokens, draft trees and chunks of a prompt) and the sampling
 * of tokens from the target's logits.  Conventions (errors, pointers, streams, workspaces) are those of evospec.h.
 */
#ifndef EVOSPEC_DECODE_H
#define EVOSPEC_DECODE_H

#include "evospec.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of what callers bring or take. */
typedef enum evospec_type { EVOSPEC_BF16 = 0, EVOSPEC_FP16 = 1, EVOSPEC_FP32 = 2 } evospec_type;
/* What the 8 bits of a cache stand for. */
typedef enum evospec_kv_kind { EVOSPEC_KV_E4M3 = 0, EVOSPEC_KV_INT8 = 1 } evospec_kv_kind;

#define EVOSPEC_KV_BLOCK 32      /* tokens that share a scale */

/*
 * A paged cache of one layer: `pages` pages of `page` tokens (32, 64, 128 or 256) for `heads` key/value heads of
 * `dim` elements (64, 96, 128, 192 or 256).  The caller owns both buffers (evospec_kv_cache_bytes says how large).
 *   data   dev, 16-B aligned.  [pages][heads][page / 32 blocks][K | V][32 * dim bytes]; in a block
 *            K  [dim / 32][half g][token m][16 bytes b]: dimension 32 s + 16 g + b of token m
 *            V  [dim / 32][half g][dimension 32 s + d][16 bytes 4 a + i]: token 8 a + 4 g + i
 *          so that 64 lanes take 16 bytes each of 1 KB in a row, and hold operands of the matrix cores.
 *   scales dev fp32, 8-B aligned [pages][heads][page / 32][2]: of K and of V of a block and head.  A value is
 *          code * |scale|; a negative scale says that there may be a NaN among the block's values.  A caller's own scales
 *          are finite; V of a scale below 2^-100, zero among them, counts as zero in the attention.
 * Codes: EVOSPEC_KV_E4M3 (4 exponent and 3 mantissa bits, largest 448, 0x7f is NaN) with scales that are powers of
 * two (the least 2^e, -100 <= e <= 120, with amax <= 448 * 2^e); EVOSPEC_KV_INT8 (-127 .. 127, -128 is NaN) with
 * scale max(amax / 127, 2^-100).
 * A sequence's tokens are found through a page table, dev int32 [S, width]: token t of sequence s is in page
 * page_table[s, t / page].  Entries that no call needs may hold anything; tokens of an entry that is needed and not
 * in [0, pages), and tokens past width * page, are left out: not written, read back as zeros, not attended to.
 */
typedef struct evospec_kv_cache {
    void *data;
    float *scales;
    int pages, page, heads, dim, kind;
} evospec_kv_cache;

/* Sizes of both buffers (host only; data and scales of the struct are not looked at). */
int evospec_kv_cache_bytes(const evospec_kv_cache *cache, size_t *out_data_bytes /*host*/, size_t *out_scale_bytes /*host*/);

/*
 * Quantise new tokens into the cache.  Rows [row_off[s], row_off[s+1]) of k and v are the tokens
 * starts[s], starts[s] + 1, ... of sequence s.
 *   k, v      dev `type` [T, heads, dim]: heads and elements contiguous, rows k_stride / v_stride elements apart,
 *             rows 16-B aligned
 *   starts    dev int32 [S], >= 0      row_off dev int32 [S + 1], non-decreasing from 0, values clamped to [0, T]
 *   max_rows  host: no sequence has more rows than that (rows past it are not written)
 * A block whose first token is written is started anew: its scale comes from this call's tokens.  In any other
 * block the scale only grows, and where it does the codes of the tokens before starts[s] become
 * round(code * old / new).  The scale is that of the largest finite magnitude; infinities saturate, NaN stays NaN.
 * Codes of a block behind the last token written are unspecified.  Two sequences of one call must not write to the
 * same block.  int8 codes are rounded again whenever their block's scale grows: a block that is written token by token, up to
 * 31 times.
 * There is a workgroup for each head and each block that max_rows rows of a sequence can touch, S * heads * ((max_rows + 30) / 32 + 1)
 * in all, which have to be fewer than 2^24 - 1023 (as in evospec_kv_read): where lengths lie far apart, call by groups of them.
 */
int evospec_kv_write(const evospec_kv_cache *cache, const void *k, long long k_stride, const void *v, long long v_stride,
                     int type, int T, const int32_t *page_table, int width, const int32_t *starts, const int32_t *row_off,
                     int S, int max_rows, void *stream);

/*
 * Read tokens back: rows [row_off[s], row_off[s+1]) of out_k and out_v (dev `type` [T, heads, dim], contiguous, 16-B
 * aligned) become the values of the tokens starts[s], starts[s] + 1, ... of sequence s, rounded once to `type`.
 */
int evospec_kv_read(const evospec_kv_cache *cache, const int32_t *page_table, int width, const int32_t *starts,
                    const int32_t *row_off, int S, int max_rows, int T, int type, void *out_k, void *out_v, void *stream);

/*
 * Attention over the cache.  Sequence s has lens[s] tokens; its query rows i = 0 .. n - 1, n = row_off[s+1] - row_off[s],
 * stand for its last n tokens (which the cache holds already).  `group` query heads share a key/value head: query head
 * a reads head a / group.
 *   row i sees token t when   tree == NULL:  t <= lens[s] - n + i
 *                             otherwise:     t < lens[s] - n, or bit t - (lens[s] - n) of tree[row] is set (n <= 64)
 *   x = scale * q . k;  out = sum softmax(x) v;  lse = log sum exp x   (a row that sees nothing: 0, -inf)
 * Products with q and with V's codes are summed in fp32, and so is the softmax; its weights are rounded to fp16 for the product with V
 * (to 2^-11 of each, or 2^-25 of the row's largest weight times scale where they are below 2^-14 of that), whatever q's type.
 * Scales of V of the blocks that a row sees may differ by a factor of 2^100.
 * Values of tokens that a row does not see, NaN among them, do not reach it.
 *   q         dev `type` (EVOSPEC_BF16 or EVOSPEC_FP16) [T, heads * group, dim], rows q_stride elements apart and 16-B aligned
 *   lens      dev int32 [S]            row_off, max_rows as above (rows past max_rows of a sequence are not written)
 *   max_len   host: no lens[s] is larger (only the split of the work depends on it)
 *             A lens[s] above width * page or 2^30 is taken as that, which moves the positions of its rows as well: they then
 *             stand for the last n tokens that the table has.  Callers keep lengths, new rows among them, within the table.
 *   tree      dev uint64 [T] or NULL   scale host, > 0 and finite
 *   out       dev `type` [T, heads * group, dim] contiguous, 16-B aligned       lse dev fp32 [T, heads * group] or NULL
 *   workspace dev, 16-B aligned, at least evospec_kv_attention_workspace_bytes(...) bytes, scratch
 */
int evospec_kv_attention_workspace_bytes(const evospec_kv_cache *cache, int group, int S, int T, int max_rows, int max_len,
                                         size_t *out_bytes /*host*/);
int evospec_kv_attention(const evospec_kv_cache *cache, const void *q, long long q_stride, int type, int T, int group,
                         const int32_t *page_table, int width, const int32_t *lens, const int32_t *row_off, int S,
                         int max_rows, int max_len, const uint64_t *tree, float scale, void *out, float *lse,
                         void *workspace, size_t workspace_bytes, void *stream);

/*
 * One token for each row of logits, from a random number that the caller brings.  In a row, tokens are ordered by
 * decreasing logit, equal ones by smaller id; NaN counts as -inf; w_i = exp((z_i - z_max) / temperature).
 *   1. the first top_k tokens are kept (top_k <= 0: all),
 *   2. of these the shortest front part whose w reach top_p of theirs, one token at least (top_p >= 1: all),
 *   3. of these the tokens with w >= min_p, the first at least (min_p <= 0: all),
 *   4. the token drawn is the first whose cumulative w, in that order, exceeds u times the sum of the kept ones (the last
 *      kept one if none does).
 * out_logprob = log of the drawn token's share in the kept ones.  temperature that is not > 0 draws the first token.
 * Tokens with w below 2^-42 may be left out of 4.  A row without a number above -inf gives id -1, logprob NaN.
 * Sums are of weights that are rounded to multiples of 2^-43: a cut of 2 and the draw of 4 are the definition's wherever their place is
 * further than V 2^-43 + 2^-38 from a border between two tokens, as a share of the kept sum, and out_logprob is as exact, in fp32.
 *   logits dev `type` [M, V], rows `stride` elements apart; V <= 2^20, M * ceil(V / 20480) < 2^22
 *   u, temperature, top_p, min_p dev fp32 [M]; top_k dev int32 [M]; each of the last four may be NULL (1, all, all, all)
 *   ids dev int32 [V] or NULL: the id of column i (distinct, not negative); NULL: i
 *   out_ids dev int32 [M]      out_logprob dev fp32 [M] or NULL
 *   workspace dev, 16-B aligned, at least evospec_sample_workspace_bytes(M, V) bytes, scratch
 */
int evospec_sample_workspace_bytes(int M, int V, size_t *out_bytes /*host*/);
int evospec_sample(const void *logits, long long stride, int type, int M, int V, const float *u, const float *temperature,
                   const int32_t *top_k, const float *top_p, const float *min_p, const int32_t *ids, int32_t *out_ids,
                   float *out_logprob, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* EVOSPEC_DECODE_H */
