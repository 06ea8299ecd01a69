/*
 * gqsa_attention.h -- what lies between the q/k/v products and the o product of a decoder layer: norms of the queries and
 * keys of each head with the rotation by position, a paged cache of keys and values in 4 bits, attention of the newest tokens
 * over that cache (token generation, one token or a tree of drafted ones at a time), and causal attention over packed prompts.
 *
 * Same conventions as gqsa.h: plain pointers and sizes, [host] or [device], a gqsa_status_t from every call, nothing thrown.
 * Calls only enqueue on `hip_stream` unless said otherwise: a stream of the current HIP device, where all [device] arrays lie.  All
 * activations are fp16, as x and y of the products are; sums, norms, scores and softmax statistics are fp32.  Softmax weights are
 * rounded to fp16 for the product with the values, and their sum is of the rounded ones: each is within 2^-11 of itself or 2^-32 of
 * the row's largest, whichever is more.
 *
 * An array "[rows, heads, head_dim]" is given by its pointer, the distance from one row to the next and the distance from one
 * head to the next, both in elements; the elements of a head follow each other.  So a slice of a joint q/k/v array, or an array
 * with the heads outermost, is taken as it is.  Pointers must be 16-byte aligned and distances multiples of 8 (GQSA_ERR_ALIGN)
 * and not negative (GQSA_ERR_SHAPE).  Results must not overlap what a call reads, unless it says that they may.  A call with no
 * rows does nothing, whatever its pointers.  At most 2^25 rows.
 *
 * Several sequences lie one behind the other in the rows: sequence b has the rows row_starts[b] .. row_starts[b + 1] - 1
 * (row_starts [device] int32[n_seqs + 1], or NULL: one row per sequence).  Values on the device cannot be refused by the host,
 * so the kernels bound them: rows outside the given array are not touched, a length counts as at least 0 and, in gqsa_cache_attend, at most
 * what the sequence's pages hold, and a page number outside the cache makes the tokens of that page absent (not read, not written).
 */
#ifndef GQSA_ATTENTION_H
#define GQSA_ATTENTION_H

#include "gqsa.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Queries and keys of every head: x rsqrt(mean(x^2) + eps) w over the head's elements (w: q_weight or k_weight; NULL: no norm for
 * that array), then the rotation of `rotary_dim` of them by the row's position: the pair (a, b) becomes (a c - b s, a s + b c),
 * (c, s) = table[position][i] for pair i; the pairs are elements (i, i + rotary_dim / 2) or, interleaved, (2i, 2i + 1); elements from
 * rotary_dim on are not rotated.  Computed in fp32 and rounded once.
 *   q, k         [device] fp16 [n_rows, q_heads, head_dim] and [n_rows, k_heads, head_dim]; k_heads may be 0 (k, k_out unused)
 *   head_dim     a multiple of 16, at most 256; rotary_dim a multiple of 16, 0 .. head_dim (GQSA_ERR_UNSUPPORTED)
 *   q_weight, k_weight  [device] fp16 [head_dim], 16-byte aligned, or NULL
 *   table        [device] fp32 [n_positions, rotary_dim / 2, 2], 16-byte aligned; NULL allowed with rotary_dim 0
 *   positions    [device] int32 [n_rows]; NULL allowed with rotary_dim 0.  The rotated elements of a row whose
 *                position lies outside 0 .. n_positions - 1 come out as NaN
 *   q_out, k_out [device] like q, k: the same array (in place, same distances) or one that does not overlap it
 */
gqsa_status_t gqsa_qk_norm_rotate(const void* q, int64_t q_row_stride, int64_t q_head_stride, int q_heads,
                                  const void* k, int64_t k_row_stride, int64_t k_head_stride, int k_heads,
                                  int64_t n_rows, int head_dim, const void* q_weight, const void* k_weight, float eps,
                                  const float* table, int64_t n_positions, int rotary_dim, int interleaved, const int32_t* positions,
                                  void* q_out, int64_t q_out_row_stride, int64_t q_out_head_stride,
                                  void* k_out, int64_t k_out_row_stride, int64_t k_out_head_stride, void* hip_stream);

/*
 * A cache of keys and values in 4 bits: n_pages pages of page_tokens tokens for kv_heads heads.  Which pages a sequence has,
 * and in which order, the caller decides and says in every call: pages [device] int32 [n_seqs, max_pages], page
 * pages[b][i] holds the tokens i page_tokens .. of sequence b.
 *
 * 32 elements of one token and head share low = the least of them (fp16, exact) and step = fp16((greatest - low) / 15), or the next smaller
 * fp16 number where low + 15 step would otherwise round to infinity; codes are
 * min(15, round-half-even((x - low) / step)), 0 where step is 0, every operation a single fp32 operation.  A code stands for
 * fp16(low + code step), rounded once.  A group with an infinity or a NaN stands for NaN throughout.
 */
typedef struct gqsa_cache* gqsa_cache_t;

typedef struct {
    int64_t n_pages;
    int32_t page_tokens;
    int32_t kv_heads;
    int32_t head_dim;
    int32_t token_bytes;        /* of one token and head: keys and values, codes, low and step */
    int64_t device_bytes;       /* pages */
    int64_t workspace_bytes;    /* partial results of gqsa_cache_attend and gqsa_cache_attend_tree: 34 MB with heads of 128, 17 with 64, whatever the cache's size and whether trees
                                   are attended to or not (gqsa_cache_attend alone would take 13 and 6.5).  Each handle has its own: 32 of them with heads of 128 1.1 GB */
} gqsa_cache_info_t;

/*
 * Allocate a cache on the current HIP device (synchronous).
 *   n_pages      1 .. 2^30
 *   page_tokens  a power of two, 32 .. 4096;  kv_heads 1 .. 1024;  head_dim 64 or 128 (GQSA_ERR_UNSUPPORTED)
 *   out          [host] receives the handle; it owns the pages and the workspace
 * Every call on the handle must be made with that device current (GQSA_ERR_HIP otherwise).  Calls on one handle must not overlap in
 * time: on one stream they are ordered and safe.
 */
gqsa_status_t gqsa_cache_create(int64_t n_pages, int page_tokens, int kv_heads, int head_dim, gqsa_cache_t* out);
gqsa_status_t gqsa_cache_info(gqsa_cache_t c, gqsa_cache_info_t* out);
void gqsa_cache_free(gqsa_cache_t c);

/*
 * Quantise new keys and values into the cache.  The rows of sequence b become its tokens lengths[b] - n .. lengths[b] - 1 (n its
 * rows here): lengths counts the new tokens in, as gqsa_cache_attend after it wants it.  Rows that would be tokens below 0, or
 * beyond what max_pages pages hold, are left out.
 *   k, v     [device] fp16 [n_rows, kv_heads, head_dim]
 *   lengths  [device] int32 [n_seqs];  max_pages 1 .. 2^20, n_seqs 1 .. 65536
 * Two sequences of one call must not write the same page.
 */
gqsa_status_t gqsa_cache_append(gqsa_cache_t c, const void* k, int64_t k_row_stride, int64_t k_head_stride,
                                const void* v, int64_t v_row_stride, int64_t v_head_stride, int64_t n_rows,
                                const int32_t* pages, int max_pages, const int32_t* lengths, const int32_t* row_starts,
                                int n_seqs, void* hip_stream);

/*
 * gqsa_qk_norm_rotate and gqsa_cache_append in one launch: new queries and keys normed and rotated, keys and values quantised into the cache.
 * The norms' factor 1 / sqrt(mean(x^2) + eps) is computed in 64 bits and rounded to fp32, every other operation is a single fp32 operation: what the cache
 * holds does not hang on the order of a sum.  (gqsa_qk_norm_rotate adds in fp32: with norms a few elements in 10^4 differ from its by one rounding; without, none does.)
 *   q        [device] fp16 [n_rows, q_heads, head_dim of the cache]; q_heads 0 .. 1024 (0: q, q_out unused)
 *   k, v, lengths, pages and the rest as in gqsa_cache_append; q_weight .. interleaved as in gqsa_qk_norm_rotate
 *   positions  [device] int32 [n_rows], or NULL: a token's place in its sequence
 *   q_out    like q, k_out like k, or NULL: the rotated keys are wanted in the cache only.  The same arrays as q and k (in place, same distances) or ones that
 *            overlap nothing else.  Rows that are left out of the cache are normed and rotated all the same; rows that belong to no sequence are left as they are
 */
gqsa_status_t gqsa_cache_append_rotated(gqsa_cache_t c, const void* q, int64_t q_row_stride, int64_t q_head_stride, int q_heads,
                                        const void* k, int64_t k_row_stride, int64_t k_head_stride,
                                        const void* v, int64_t v_row_stride, int64_t v_head_stride, int64_t n_rows,
                                        const void* q_weight, const void* k_weight, float eps,
                                        const float* table, int64_t n_positions, int rotary_dim, int interleaved, const int32_t* positions,
                                        void* q_out, int64_t q_out_row_stride, int64_t q_out_head_stride,
                                        void* k_out, int64_t k_out_row_stride, int64_t k_out_head_stride,
                                        const int32_t* pages, int max_pages, const int32_t* lengths, const int32_t* row_starts,
                                        int n_seqs, void* hip_stream);

/*
 * The values that the last tokens of each sequence stand for: row i of the n rows of sequence b is its token lengths[b] - n + i (a whole
 * sequence: n = lengths[b]).  Rows without a token (below 0, beyond the pages, or on an absent page) are zero.
 *   k_out, v_out [device] fp16 [n_rows, kv_heads, head_dim]
 */
gqsa_status_t gqsa_cache_read(gqsa_cache_t c, void* k_out, int64_t k_row_stride, int64_t k_head_stride,
                              void* v_out, int64_t v_row_stride, int64_t v_head_stride, int64_t n_rows,
                              const int32_t* pages, int max_pages, const int32_t* lengths, const int32_t* row_starts,
                              int n_seqs, void* hip_stream);

/*
 * out = softmax(scale q K^T) V over the cache: the newest n rows of sequence b are its tokens lengths[b] - n .. lengths[b] - 1, and the row of
 * token t sees the tokens 0 .. t.  q_heads / kv_heads neighbouring query heads share a head of the cache (grouped and multi-query
 * attention).  A row that sees no token is zero.
 *   q, out   [device] fp16 [n_rows, q_heads, head_dim]; q_heads a multiple of kv_heads, at most 1024; every row of out is written
 *            that belongs to a sequence
 *   scale    finite (GQSA_ERR_RANGE), head_dim^-0.5 usually
 * Every sequence may have any number of rows; the cache is read once per 16 rows of the heads of a group.  GQSA_ERR_SHAPE where n_rows times
 * q_heads / kv_heads passes 2^30, or where the pages that the table has room for could be 2^31 steps of 128 tokens and more, over all rows and
 * heads.  A query with an infinity or a NaN makes its row NaN.  Results are bit-identical
 * from run to run.  Can be captured (nothing is allocated, nothing is read back).
 */
gqsa_status_t gqsa_cache_attend(gqsa_cache_t c, const void* q, int64_t q_row_stride, int64_t q_head_stride, int q_heads,
                                int64_t n_rows, const int32_t* pages, int max_pages, const int32_t* lengths,
                                const int32_t* row_starts, int n_seqs, float scale, void* out, int64_t out_row_stride,
                                int64_t out_head_stride, void* hip_stream);

/*
 * The same for rows that are a tree of drafted tokens (or any others that do not see all rows before their own): row i of the n rows of sequence b sees the
 * tokens 0 .. lengths[b] - n - 1, which lie before all rows, and of the rows those that its mask names -- itself only if it names it.  A row that
 * sees no token is zero.
 *   masks    [device] int32 [n_rows, mask_words]: bit j % 32 of word j / 32 stands for row j of the row's own sequence (bits of rows that it does not have, and rows
 *            from 32 mask_words on: not seen); mask_words 1 .. 2^15 (GQSA_ERR_UNSUPPORTED)
 * Keys and values that a row does not see have no effect on it, whatever they hold.  Rows that would be tokens beyond what the pages hold, which gqsa_cache_append leaves
 * out, are seen by nobody, and see what there is like any other.
 * Which of two kernels runs hangs on what the host knows: max_pages and the mean number of rows, not the lengths.  With more than 32 rows (of a sequence times heads of a group) on average
 * the one for many rows is taken where the table has much room.  Short sequences under a wide table are slower for it: 500 tokens, 64 rows for each of 8 heads 15.7 us with a table for
 * 131072 tokens, 9.3 with one for 500; 16 x 1000 tokens, the same 27 and 20; so give no more pages than the longest sequence has where that is known.  One large tree among sequences of
 * one row goes to the kernel for few: 32 x 4000 tokens, 32 heads for 8, one of 64 rows among 31 of one 41 us.  The rest as in gqsa_cache_attend.
 */
gqsa_status_t gqsa_cache_attend_tree(gqsa_cache_t c, const void* q, int64_t q_row_stride, int64_t q_head_stride, int q_heads,
                                     int64_t n_rows, const int32_t* pages, int max_pages, const int32_t* lengths,
                                     const int32_t* row_starts, int n_seqs, const int32_t* masks, int mask_words, float scale,
                                     void* out, int64_t out_row_stride, int64_t out_head_stride, void* hip_stream);

/*
 * Of the newest rows of each sequence some become neighbours: with n rows of sequence b, whose tokens are lengths[b] - n .. lengths[b] - 1, token lengths[b] - n + i
 * becomes what token lengths[b] - n + path[row_starts[b] + i] was, for i = 0 .. accepted[b] (path and accepted as gqsa_verify gives them; afterwards the
 * sequence is lengths[b] - n + accepted[b] + 1 tokens long, which the caller notes).  The tokens behind stay.  Codes are moved as they are: nothing is rounded anew.
 *   path     [device] int32 [n_rows], accepted [device] int32 [n_seqs] (counts as at most n - 1).  Entries of path that are below i, or n and more, are left out: their token stays
 *            as it is; so does one whose old or new place lies on an absent page, beyond the pages or below 0
 */
gqsa_status_t gqsa_cache_keep(gqsa_cache_t c, int64_t n_rows, const int32_t* pages, int max_pages, const int32_t* lengths, const int32_t* row_starts,
                              int n_seqs, const int32_t* path, const int32_t* accepted, void* hip_stream);

/*
 * Causal attention over packed prompts: sequence b has the query rows q_starts[b] .. q_starts[b + 1] - 1 and the keys and values
 * k_starts[b] .. k_starts[b + 1] - 1 ([device] int32[n_seqs + 1] both); the last query row sees all its keys, the one before one key fewer, and so on
 * (more keys than queries: an earlier part of the prompt that has been seen already).  A row that sees no key is zero.
 *   q, out   [device] fp16 [n_q_rows, q_heads, head_dim];  k, v [device] fp16 [n_k_rows, kv_heads, head_dim]
 *   head_dim 64 or 128; q_heads a multiple of kv_heads (grouped heads as in gqsa_cache_attend), at most 1024; rows of k and of v
 *            at most 2^23 elements apart (GQSA_ERR_UNSUPPORTED); (n_q_rows / 128 + n_seqs) q_heads at most 2^23 (GQSA_ERR_SHAPE)
 * Keys and values that a row does not see have no effect on it, whatever they hold.  An infinite value that it sees makes that element of the row
 * infinite, a NaN or infinities of both signs make it NaN, however small their weights are.
 */
gqsa_status_t gqsa_prompt_attend(const void* q, int64_t q_row_stride, int64_t q_head_stride, int q_heads, int64_t n_q_rows,
                                 const void* k, int64_t k_row_stride, int64_t k_head_stride,
                                 const void* v, int64_t v_row_stride, int64_t v_head_stride, int kv_heads, int64_t n_k_rows,
                                 int head_dim, const int32_t* q_starts, const int32_t* k_starts, int n_seqs, float scale,
                                 void* out, int64_t out_row_stride, int64_t out_head_stride, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* GQSA_ATTENTION_H */
