/*
 * siso_kv.h - what a query costs that the semantic cache does not answer: the paged
 * key/value cache of the target model, its attention over that cache, and the
 * verification of drafted tokens.
 *
 * A lookup (siso.h) ends in a hit, which is answered from the cache, or in a miss, which
 * the target model answers: the prompt's tokens are read in chunks, the answer is written
 * token by token.  A near miss has a stored answer that is probably right for the most
 * part: its tokens are a draft, which the model verifies several at a time.
 *
 *   siso_kv_write   puts the keys and values of new tokens into the cache, as 16-bit
 *                   rows or quantised to 8 bits as they are written;
 *   siso_kv_read    reads them back;
 *   siso_kv_attend  attention of a chunk of new tokens over the cache: one token of each
 *                   sequence (decoding), a draft's few, or thousands of a prompt;
 *   siso_kv_verify  judges drafted tokens by the target's probabilities, from random
 *                   numbers that the caller gives, and chooses the token that follows.
 *
 * Conventions are those of siso.h: device pointers owned by the caller, all work enqueued
 * on the stream of siso_kv_set_stream, SISO_OK or a negative code, a message for the last
 * failure, calls on one handle not thread-safe against each other.  No call but
 * siso_kv_create, siso_kv_destroy and siso_kv_bad_pages allocates, frees or synchronises:
 * all others can be captured in a graph.  Calls share a workspace of the handle: work
 * enqueued on one stream has to be ordered before work that is enqueued on another.
 */
#ifndef SISO_KV_H
#define SISO_KV_H

#include "siso.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct siso_kv siso_kv; /* opaque; owns the pages on the device */

/*
 * A batch of sequences and their newest tokens, for all calls below.  Rows first[b] to
 * first[b + 1] - 1 of the batch are the m newest of the length[b] tokens of sequence b:
 * row first[b] + i stands at position length[b] - m + i.  Position p is slot
 * p % page_tokens of page pages[b * width + p / page_tokens].
 *   n:      sequences, at most 65,535;  rows: new tokens in all, at most 2^24.
 *   first:  device pointer, n + 1 ints, not decreasing, from 0 to rows.
 *   length: device pointer, n ints, 0 to width * page_tokens;
 *   pages:  device pointer, [n][width] page numbers (NULL length and pages: siso_kv_verify);
 *           width * page_tokens is at most 2^31 - 2^25 (SISO_EINVAL otherwise).
 *   max_new, max_length: no sequence has more new tokens / more tokens (0: not known; rows
 *           and width * page_tokens are taken).  They size launches: a sequence of more rows
 *           than max_new may be left out, max_length only weighs on speed.
 * The arrays are read when the work runs.  What does not keep to these ranges is never
 * read or written at: lengths are taken as the closest allowed one, positions below 0 are
 * no positions (nothing is written; a query there sees nothing), and a page number that
 * is not one of the cache's pages is counted (siso_kv_bad_pages): writes to it are left
 * out, reads give zeros, attention does not see its tokens.
 */
typedef struct siso_kv_batch {
    long n, rows;
    const int *first, *length, *pages;
    long width, max_new, max_length;
} siso_kv_batch;

/*
 * A cache of `pages` pages of `page_tokens` tokens for each of `layers` layers.
 *   kv_heads: 1 to 1,024;  head_dim: a multiple of 8, 8 to 256;
 *   page_tokens: a power of two, 16 to 1,024;  layers, pages: from 1 on.
 *   dtype: SISO_BF16 keeps keys and values as given; SISO_FP8 keeps every vector (a
 *          token's key or value of one head) as E4M3 codes and a float scale, as an
 *          8-bit cache of siso_create_ex keeps a row: scale = max|x| / 448, code = x / scale
 *          rounded to the nearest E4M3 value, ties to the even mantissa; a vector that holds a
 *          NaN or an infinity has the scale NaN.  Both take and give 16-bit rows (bfloat16);
 *          SISO_F32 is refused: single-precision rows double what decoding reads.
 * Takes layers * pages * page_tokens * kv_heads * 2 * (2 * D, or D + 4) bytes, D = head_dim
 * rounded up to a multiple of 64, and a workspace.  Synchronises.
 */
int siso_kv_create(int layers, int kv_heads, int head_dim, int page_tokens, long pages, int dtype, siso_kv **out);
void siso_kv_destroy(siso_kv *kv); /* waits for the handle's stream first */
int siso_kv_set_stream(siso_kv *kv, void *hip_stream);

/*
 * Keys and values of the batch's rows into layer `layer`.
 *   k, v: device pointers, 16-bit rows: element e of head h of row r at
 *         [r * token_stride + h * head_stride + e] (strides in elements, any).
 * No two rows of a batch may name one position: elements of both, in 8 bits also the scale of one beside codes of the other,
 * may stand there until it is written again.  Asynchronous.
 */
int siso_kv_write(siso_kv *kv, int layer, const siso_kv_batch *batch, const void *k, long k_token_stride, long k_head_stride,
                  const void *v, long v_token_stride, long v_head_stride);

/*
 * What the cache holds at the positions of the batch's rows (all of a sequence: a batch
 * whose rows are all of its tokens): code * scale in single precision, or the 16-bit rows.
 *   out_type: SISO_BF16 (rounded once, to nearest even) or SISO_F32.
 *   out_k, out_v: device pointers, [rows][kv_heads][head_dim], 16-byte aligned.
 * Rows without a position are zeros.  Asynchronous.
 */
int siso_kv_read(siso_kv *kv, int layer, const siso_kv_batch *batch, int out_type, void *out_k, void *out_v);

/*
 * Attention of the batch's rows over layer `layer` (which holds these rows' own keys and
 * values, too: siso_kv_write comes first).  For row r at position P and query head h,
 * which shares kv head h / (heads / kv_heads) with its neighbours:
 *     s_j = scale * <q, k_j>,   j <= P, and j > P - window if window > 0
 *     out = sum_j exp(s_j) v_j / sum_j exp(s_j),   lse = log sum_j exp(s_j)
 *   q:     device pointer, 16-bit rows, strides as for siso_kv_write.
 *   heads: a multiple of kv_heads, at most 128 of them for each; rows * heads at most 2^30
 *          (SISO_EINVAL otherwise).
 *   scale: finite; scores have to stay within single precision's range.
 *   out:   device pointer, [rows][heads][head_dim], 16 bits, 16-byte aligned.
 *   lse:   device pointer, [rows][heads] floats, or NULL.
 * A row that sees nothing gets zeros and lse = -inf.  Infinities and NaN at positions that
 * a row does not see do not touch it.  Statistics and sums are held in single precision;
 * exp(s_j - max), times v's scale in an 8-bit cache, is rounded to 16 bits before it is multiplied with v.
 * Results do not depend on scheduling.  Asynchronous.
 */
int siso_kv_attend(siso_kv *kv, int layer, const siso_kv_batch *batch, const void *q, long q_token_stride, long q_head_stride,
                   int heads, float scale, int window, void *out, float *lse);

/*
 * Verification of drafted tokens.  The rows of sequence b are the tokens that the target
 * model was given: row 0 the last token that stands, rows 1 to m - 1 the draft; the target's
 * distribution behind row i judges the token of row i + 1.
 *   tokens:  device pointer, [rows] ints.
 *   target:  device pointer, [rows][vocab] probabilities (type SISO_F32 or SISO_BF16), row r
 *            at r * target_stride elements.
 *   draft:   device pointer, as target: row i holds the distribution that the token of row
 *            i + 1 was drawn from (row m - 1 is not read); NULL: the draft has none (a
 *            stored answer's tokens).
 *   u_accept: device pointer, [rows] floats in [0, 1), that of row i for the token of row i + 1;
 *   u_sample: device pointer, [n] floats in [0, 1).
 *   vocab:   1 to 2^24.
 * With p the target's row i, x the token of row i + 1 and q = draft's probability of x (1
 * without draft): x is accepted if u_accept * q < p(x); the first token that is not ends the
 * draft, and the token that follows is drawn with the weights max(p - q, 0) over the
 * vocabulary (without draft: p, without x), or with p of row m - 1 if all were accepted: the
 * first token at which the running sum of the weights exceeds u_sample times their sum.
 * So the tokens are distributed as the target's own (for weights that are all zero: p is taken; if that is zero, too, -1).
 * Weights below zero and NaN count as zero.  A token outside the vocabulary is not accepted.
 *   u_accept = u_sample = NULL: greedy.  A token is accepted if it is the one with the
 *            largest entry of its row (the lowest index of equal ones; NaN never), which
 *            is also the token that follows: target may hold logits.  draft must be NULL.
 *   out_accepted: device pointer, [n] ints: draft tokens accepted (-1: a sequence without rows).
 *   out_tokens: device pointer, [rows] ints: per sequence the accepted tokens, the token
 *            that follows, then -1.
 * With that the sequence stands at length[b] - (m - 1) + out_accepted[b] tokens: the rest of
 * the draft's keys and values is written over by what comes next.
 * Products and sums are formed in double precision.  Asynchronous.
 */
int siso_kv_verify(siso_kv *kv, const siso_kv_batch *batch, const int *tokens, int vocab, int type, const void *target,
                   long target_stride, const void *draft, long draft_stride, const float *u_accept, const float *u_sample,
                   int *out_accepted, int *out_tokens);

/* Page numbers outside the cache that calls have met since it was created (each counted at least once per call and layer).
 * Synchronises with the stream.  Negative = error code. */
long siso_kv_bad_pages(siso_kv *kv);

/* Message for the last error on this handle ("" if none).  Owned by the handle. */
const char *siso_kv_last_error(const siso_kv *kv);

#ifdef __cplusplus
}
#endif
#endif /* SISO_KV_H */
