/*
 * dycl_decode.h - operators of networks that emit a token at a time: what
 * stands around the layers of dycl_tokens.h when every call brings one new
 * token per sequence (Sec. 5.3's generative networks, whose loop ends at an
 * end token or a length bound).  The rotation of heads by their positions,
 * the entry of new keys and values into a paged cache, the attention of one
 * token to it, the choice of the next tokens over beams and vocabulary, and
 * the reordering of the cache behind that choice.
 *
 * The cache of a layer is two tensors of bf16 (uint16_t bits), contiguous
 * and 16-byte aligned: keys and values, [pages][heads][page][dim].  A page
 * holds `page` consecutive tokens (a power of two from 8 to 1024) of one
 * sequence, dim is a multiple of 8 up to 256.  tables [sequences][max_pages]
 * int32 (row pitch ldt) names each sequence's pages in order: the token at
 * place p is in page tables[s][p / page], slot p % page.  Pages may be shared between
 * sequences, layers may share tables.  A table's entry outside [0, pages), a
 * place past the table and a sequence outside [0, sequences) are told by
 * the kernels and never followed: nothing is written there, and a key there
 * is none.
 *
 * Other tensors are row-major matrices with a row pitch `ld*` in elements (at
 * least the row length); device pointers, caller-owned, aligned to their
 * element.  A row is one token; its heads lie side by side (a slice of the
 * wider output of one product is taken as it is).  Work is queued on
 * `hip_stream`; no call allocates, copies to the host or waits, so all may be
 * captured into a HIP graph.  Outputs and workspaces must not overlap inputs
 * or one another, except where said; a workspace belongs to one call at a
 * time.  Errors are dycl_status codes with dycl_last_error() (dycl.h);
 * validation happens before any launch.  A row's results are the same bits
 * whatever the number and the values of the rows beside it.
 */
#ifndef DYCL_DECODE_H_
#define DYCL_DECODE_H_

#include <stddef.h>
#include <stdint.h>

#include "dycl_tokens.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Which two of a head's first 2 * pairs values form pair i. */
typedef enum { DYCL_ROTATE_HALF = 0 /* i, i + pairs */, DYCL_ROTATE_INTERLEAVED = 1 /* 2 i, 2 i + 1 */ } dycl_rotate_layout;

/*
 * Each pair (a, b) of each head, turned by the angle t = position * frequencies[i]:
 *   magnitude * (a cos t - b sin t),  magnitude * (b cos t + a sin t)
 * adjoint != 0: by -t, which is the gradient of x for a gradient of y.
 * Values past the pairs are copied.  The angle is 64 bits, so positions may
 * be any; the rest is float32 with one rounding to the type.
 *   x, y          [n][heads * dim] type; y may be x itself (same pitch).
 *   positions     [n] int32.
 *   frequencies   [pairs] float64, radians per position.
 * 1 <= pairs <= dim / 2, pairs <= 2048, heads * dim <= 65536, n >= 0.
 */
int dycl_op_rotate(const void* x, int type, int64_t ldx, const int32_t* positions, const double* frequencies, int pairs,
                   int layout, float magnitude, int adjoint, int64_t n, int heads, int dim, void* y, int64_t ldy,
                   void* hip_stream);

/*
 * Entry of n tokens into the cache: row r's keys, turned by its position
 * as by dycl_op_rotate, and values go to place positions[r] of sequence
 * sequence[r]; its queries are turned into q_out.
 *   k, v          [n][heads * dim] type.
 *   q, q_out      [n][q_heads * dim] type, or both NULL; q_out may be q (same pitch).
 *   positions     [n] int32.  A negative one is padding: nothing enters the
 *                 cache, and its q_out is 0.
 *   sequence      [n] int32 or NULL: row r is sequence r (n == sequences).
 *   frequencies   [pairs], or NULL with pairs 0: nothing is turned.
 * Two rows of one call must not have the same place of the same page: which of
 * their values remain is then not defined (no other row is affected).
 * heads, q_heads * dim as above; n >= 0 (0 does nothing).
 */
int dycl_op_append(const void* k, int64_t ldk, const void* v, int64_t ldv, const void* q, int64_t ldq, void* q_out,
                   int64_t ldo, int type, const int32_t* positions, const int32_t* sequence, const double* frequencies,
                   int pairs, int layout, float magnitude, int64_t n, int q_heads, int heads, int dim,
                   const int32_t* tables, int64_t ldt, int64_t sequences, int max_pages, uint16_t* keys,
                   uint16_t* values, int64_t pages, int page, void* hip_stream);

/*
 * Attention of n tokens, one row of queries each, to the cache:
 *   out[r][h] = sum_j p_j v_j,  p = softmax over j of scale * q[r][h] . k_j
 * over the keys j of row r's sequence in [lengths[r] - window, lengths[r])
 * (from 0 without a window) whose mask is not 0.  Query head h reads the
 * cache's head h / (q_heads / heads).  A key whose score is -infinity has
 * weight 0 and adds nothing, however large its value.  (An infinite value makes its column's result
 * infinite where its key's weight is 2^-64 of the row's largest or more, and infinite or NaN where it is less; weights below 2^-94 of
 * it may count as 0.)  A row without a key is 0.  What the cache holds in places that a row does not see is not used, whatever it is.
 *   q, out        [n][q_heads * dim] bf16; out may not be q.
 *   lengths       [n] int32: keys that the row sees.  Below 0 as 0, past
 *                 max_length as max_length.
 *   sequence      [n] int32 or NULL, as above.  (Rows of one sequence may have
 *                 lengths of their own: a prompt's tokens as rows.  Each reads
 *                 its keys anew.)
 *   mask          [n][max_length] uint8, pitch ldm, or NULL.  0: the token at that place
 *                 skipped this block and has no key here.
 *   max_length    at least every length, at most max_pages * page; the work
 *                 is laid out and divided for it.  (Give a tight one: where it is 32 times the lengths a call takes several times as long.)
 *   window        0 (none) or the number of last places seen.
 *   workspace     dycl_op_attend_workspace(...) bytes, 16-byte aligned, or NULL when that is 0.
 * Scores, softmax and sums are float32.  The softmax's weights enter the second product as
 * three bf16 terms, all of float32's 24 significant bits.  The keys are summed in parts that the
 * dim alone sets, joined in a fixed order.  -1e38 < scale < 1e38,
 * q_heads a multiple of heads, n * q_heads < 2^31, max_length < 2^31 - 4096.
 */
size_t dycl_op_attend_workspace(int64_t n, int q_heads, int heads, int dim, int64_t max_length, int64_t window);
int dycl_op_attend(const uint16_t* q, int64_t ldq, int64_t n, int q_heads, int heads, int dim, float scale,
                   const uint16_t* keys, const uint16_t* values, int64_t pages, int page, const int32_t* tables,
                   int64_t ldt, int64_t sequences, int max_pages, const int32_t* lengths, const int32_t* sequence,
                   int64_t max_length, int64_t window, const uint8_t* mask, int64_t ldm, uint16_t* out, int64_t ldo,
                   void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * The choice of the next tokens: of the beams * words candidates (w, t) of
 * each sequence, valued
 *   c = scores[w] + logits[w][t] - log sum_t' exp logits[w][t']
 * the k largest, largest first, the lowest w * words + t among equals.
 * A beam that has ended is one candidate: `end`, with its score as it is.
 * A logit of -infinity or NaN is a closed token, +infinity counts as the
 * largest finite value, of a score too; a beam whose score is -infinity or NaN has no candidates.
 * An end token outside [0, words) ends no beam (then `ended` must be NULL).
 *   logits     [sequences * beams][words] type, pitch ldl.
 *   scores     [sequences * beams] float32: sums of logarithms so far.
 *   ended      [sequences * beams] uint8 or NULL.
 *   parents    [sequences][k] int32: the row of logits that goes on; -1 where
 *              fewer than k candidates are there (token -1, score -infinity, ended 0).
 *   tokens     [sequences][k] int32.   new_scores  [sequences][k] float32.
 *   new_ended  [sequences][k] uint8: the parent had ended, or the token is `end`.
 * float32; the sum's order depends on words alone.  Candidates are compared as rounded to
 * float32: of two that round to the same value either may be taken or come first, unless
 * their logits are the same.
 *   workspace  dycl_op_beam_workspace(...) bytes, 16-byte aligned.
 * 1 <= beams <= 64, 1 <= k <= 64, 1 <= words <= 2^20, sequences * beams < 2^24.
 */
size_t dycl_op_beam_workspace(int64_t sequences, int beams, int words, int k);
int dycl_op_beam(const void* logits, int type, int64_t ldl, const float* scores, const uint8_t* ended, int end,
                 int64_t sequences, int beams, int words, int k, int32_t* parents, int32_t* tokens, float* new_scores,
                 uint8_t* new_ended, void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * The cache behind such a choice, without moving full pages: row i goes on
 * from rows' sequence parents[i].  Its table is its parent's, with fresh[i]
 * as the page of its next token, and its length is the parent's.  Where that page is begun
 * already (length % page != 0), the parent's tokens in it are copied into fresh[i].
 * A parent outside [0, rows) leaves an empty row: length 0, table -1.
 * A length past the table counts as a full table.
 *   tables      [rows][max_pages], lengths [rows].
 *   parents, fresh  [n] int32.  The fresh pages are distinct, and none of them is read by a sequence that goes on.
 *   new_tables  [n][max_pages] (pitch ldn), new_lengths [n]; NULL: not written, only the pages
 *               are (for a further layer with the same tables).
 *   keys, values  one layer's cache, or both NULL: only tables and lengths.
 * n == 0 does nothing, but refuses a cache that is refused otherwise: a caller of several layers can check all before the first.
 */
int dycl_op_fork(const int32_t* tables, int64_t ldt, const int32_t* lengths, int64_t rows, int max_pages,
                 const int32_t* parents, const int32_t* fresh, int64_t n, int32_t* new_tables, int64_t ldn,
                 int32_t* new_lengths, uint16_t* keys, uint16_t* values, int64_t pages, int heads, int page, int dim,
                 void* hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* DYCL_DECODE_H_ */
