/*
 * gqsa_verify.h -- which of several drafted tokens stand, and what follows them: verification of a chain or a tree of drafted tokens
 * against the target's probabilities, from random numbers that the caller gives.  The result has the distribution of the target, whatever the draft was.
 *
 * Same conventions as gqsa_attention.h; probabilities are fp32.
 *
 * A sequence's rows are the last token that is certain (row 0) and the drafted tokens behind it; every row has a parent among the rows before it, of
 * which its token was thought to be the continuation.  (The same rows go through the model at once: see gqsa_cache_attend_tree.)
 */
#ifndef GQSA_VERIFY_H
#define GQSA_VERIFY_H

#include "gqsa.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * The workspace of gqsa_verify, on the current HIP device (synchronous), for calls of up to max_seqs sequences and max_vocab tokens in the vocabulary.
 *   max_seqs   1 .. 65536; max_vocab 1 .. 2^22 (GQSA_ERR_UNSUPPORTED); max_seqs max_vocab at most 2^34 (GQSA_ERR_SHAPE)
 *   out        [host] receives the handle
 * Every call on the handle must be made with that device current (GQSA_ERR_HIP otherwise).  Calls on one handle, graphs that hold such calls among
 * them, must not overlap in time: on one stream they are ordered and safe.
 */
typedef struct gqsa_verifier* gqsa_verifier_t;
gqsa_status_t gqsa_verify_create(int max_seqs, int max_vocab, gqsa_verifier_t* out);
void gqsa_verify_free(gqsa_verifier_t v);

/*
 * Row i of a sequence, with token x and parent g, stands if u_i m < p, where p = target[g][x] and
 *   with `draft` (a chain whose tokens were drawn from it):  m = draft[i][x];
 *   without (tokens chosen in any way that does not depend on the u):  m = 1 - the sum of target[g] at the tokens of g's children before i.
 * From row 0 the way goes to the first child that stands, from there on to its first child that does, and so on.  Behind the way's last row g one more token
 * is drawn: the first x at which the running sum of the weights passes v times their sum; the weights are
 *   with `draft`:  max(target[g] - draft[g + 1], 0), or target[g] where g is the sequence's last row;
 *   without:       target[g], but 0 at the tokens of g's children;
 * and target[g] where all those are 0.  (If no running sum passes, as where v is 1 or more, the last x of a positive weight.)  Products and sums are in 64 bits, so a result
 * does not hang on the order of additions but where v falls within some 2^-50 of a border.  Without `draft` and with one row to a sequence: a token drawn from target.
 *
 *   target   [device] fp32 [n_rows, vocab], rows `target_row` elements apart: behind each row's token, the target's probabilities of the next one (what
 *            is not a positive finite number counts as 0, here and in draft)
 *   draft    [device] fp32 [n_rows, vocab], rows `draft_row` apart: what the row's token was drawn from (row 0 of a sequence is not read); or NULL
 *   tokens   [device] int32 [n_rows]; a drafted token outside 0 .. vocab - 1 does not stand
 *   parents  [device] int32 [n_rows]: number of the parent within the sequence, less than the row's own (a row with any other does not stand); NULL: a chain.  With `draft`
 *            only NULL (GQSA_ERR_UNSUPPORTED).  Where siblings have the same token the first counts
 *   uniforms [device] fp32 [n_rows]: u, from [0, 1);  finals [device] fp32 [n_seqs]: v, from [0, 1)
 *   row_starts [device] int32 [n_seqs + 1], or NULL: one row per sequence.  Rows of a sequence from the 1025th on are not looked at
 *   path     [device] int32 [n_rows]: the way -- its rows' numbers within the sequence, row 0 first -- from the sequence's first row on, -1 behind it
 *   out      [device] int32 [n_rows]: the tokens that stand and the one drawn behind them, from the sequence's first row on, -1 behind.  (-1, too, for a token
 *            drawn where all weights and target[g] are 0)
 *   accepted [device] int32 [n_seqs]: rows on the way behind row 0; -1 for a sequence without rows
 * A call without rows reads no array and writes `accepted` only; without sequences either (n_seqs 0) it does nothing.
 * Rows that belong to no sequence are left as they are.  n_seqs and vocab as the handle was made for (GQSA_ERR_BUFSIZE).  Results are bit-identical from run to run.  Can be captured.
 */
gqsa_status_t gqsa_verify(gqsa_verifier_t v, const float* target, int64_t target_row, const float* draft, int64_t draft_row, int vocab, int64_t n_rows,
                          const int32_t* tokens, const int32_t* parents, const float* uniforms, const float* finals, const int32_t* row_starts, int n_seqs,
                          int32_t* path, int32_t* out, int32_t* accepted, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* GQSA_VERIFY_H */
