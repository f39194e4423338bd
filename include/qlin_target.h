/*
 * qlin_target.h -- C ABI of what the target runs between its quantized linears,
 * on MI355X (gfx950): the norms and rotation of queries and keys with the append
 * to the key/value cache, the causal attention that reads the cache, and the
 * decision on the drafted tokens.  Part of libqlin.so; status codes,
 * qlin_last_error() and qlin_last_status() are those of qlin.h.
 *
 * The operations (Kim, Lee, Kim, arXiv 2607.04244): Sec. 2.2, the target verifies
 * the 16 tokens of a draft block in one forward pass and the loop keeps a prefix,
 * without loss.  The target's prompt, its draft blocks and plain single-token
 * decoding all run through the same calls, for any number of sequences at once.
 *
 * Conventions of qlin.h: bf16 values travel as uint16_t bit patterns, every call
 * is asynchronous on its stream and returns a QLIN_* status, argument checks run
 * before any HIP call.  The lengths of the sequences are DEVICE arrays: a captured
 * graph can be replayed after they changed.
 */
#ifndef QLIN_TARGET_H
#define QLIN_TARGET_H

#include <stdint.h>

#include "qlin.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * The new tokens of a batch.  Sequence b owns the rows new_start[b] ..
 * new_start[b + 1] - 1 of the row arrays (q, k, v, out), its new tokens in order;
 * its cache then holds length[b] tokens, the new ones last, so its new token i is
 * at position length[b] - (new_start[b + 1] - new_start[b]) + i.
 *
 * Rows from new_start[n_seq] on (padding) are neither read nor written.  A
 * sequence without new tokens is skipped.  Whatever the device arrays hold, no
 * call reads or writes outside the row arrays and the cache's slots: bounds are
 * clamped to [0, rows], new tokens past the first max_new of a sequence are left
 * out, and a sequence whose slots are not all inside the cache, and inside its own
 * room there (capacity below), counts as one without cached tokens.
 */
typedef struct qlin_batch {
    int64_t n_seq;               /* sequences, 1 .. 65536 */
    int64_t rows;                /* rows of the row arrays, 0 .. 2^22 */
    int64_t max_new;             /* upper bound of any sequence's new tokens, 0 .. rows */
    int64_t max_len;             /* upper bound of any length[b] (0 .. 2^28): sizes the work split, never the result */
    const int32_t *new_start;    /* DEVICE [n_seq + 1], ascending */
    const int32_t *length;       /* DEVICE [n_seq] */
    const int64_t *cache_start;  /* DEVICE [n_seq]: slot of the sequence's token 0; NULL: b * cache.seq_slots */
} qlin_batch;

/*
 * The key/value cache: slot s of key/value head h holds 128 bf16 values at element
 * s * token_stride + h * head_stride of k and of v.  Token j of sequence b is slot
 * start + j (start: see cache_start above).  Two layouts among others:
 *   [sequences][heads][capacity][128]  token_stride 128, head_stride capacity * 128,
 *                                      seq_slots heads * capacity
 *   [tokens][heads][128] (packed)      token_stride heads * 128, head_stride 128,
 *                                      cache_start given
 * In the first, the slots past a sequence's capacity are other heads' or sequences':
 * capacity tells where its room ends, and a longer sequence counts as one without cached
 * tokens.  Rooms begin every seq_slots slots; with cache_start a sequence may begin inside
 * one, and has the rest of it.
 */
typedef struct qlin_kv_cache {
    int64_t capacity;            /* slots of one sequence's room, 0 .. 2^40; 0: no bound but slots */
    uint16_t *k, *v;             /* DEVICE, 16-byte aligned */
    int64_t heads;               /* key/value heads */
    int64_t slots;               /* slots that may be addressed: s < slots, 1 .. 2^40 */
    int64_t token_stride;        /* elements, 128 .. 2^28, a multiple of 8 */
    int64_t head_stride;         /* elements, 128 .. 2^40, a multiple of 8 */
    int64_t seq_slots;           /* slots between sequences where cache_start is NULL, and between rooms, 0 .. 2^40 */
} qlin_kv_cache;

/*
 * qlin_norm_rope_append -- for every new token at position p, with fp32 arithmetic
 * and one rounding to bf16:
 *   q_out[m][h] = rotate(p, norm(q[m][h], q_norm))     h < q_heads
 *   k cache slot of p, head h = rotate(p, norm(k[m][h], k_norm))
 *   v cache slot of p, head h = v[m][h]
 *   norm(x, w)[d] = x[d] / sqrt(mean(x^2) + eps) * w[d], or x where w is NULL; the
 *     squares' sum is fp32: a row of values above 2^60 comes out as zeros
 *   rotate(p, x): with angle a_i = p * inv_freq[i], i < rotary_dim / 2, the pairs
 *     (x[i], x[i + rotary_dim / 2]), or (x[2 i], x[2 i + 1]) if interleaved, become
 *     (x cos a - y sin a, x sin a + y cos a); dimensions >= rotary_dim stay.
 * Angles are reduced to one turn in 64 bits, so far positions lose nothing.
 *
 *   q, k, v     DEVICE bf16 rows of q_heads (cache heads) x 128, row_stride
 *               elements apart (multiples of 8): outputs of separate linears, or
 *               slices of one
 *   q_norm, k_norm   DEVICE bf16 [128], or NULL: no norm
 *   eps         >= 0
 *   inv_freq    DEVICE double [rotary_dim / 2], radians a position (NULL if
 *               rotary_dim is 0)
 *   rotary_dim  a multiple of 16, 0 .. 128
 *   q_out       DEVICE bf16 [rows][q_heads][128], rows q_out_stride elements
 *               apart; q itself (same stride), or elements apart from every input
 *               and the cache
 * All pointers 16-byte aligned (norm weights and inv_freq: 8).  k and v must not
 * overlap the cache, and neither the batch's arrays nor the weights and inv_freq may
 * overlap q_out or the cache.  Two new tokens must not share a slot (sequences sharing
 * slots: which of them is stored is not defined).
 * Errors: INVALID (NULL, sizes, strides, overlap, eps), UNSUPPORTED (head_dim !=
 * 128, limits), ALIGN, HIP.
 */
int qlin_norm_rope_append(const qlin_batch *batch, const qlin_kv_cache *cache, int64_t q_heads, int64_t head_dim,
                          const uint16_t *q, int64_t q_stride, const uint16_t *k, int64_t k_stride,
                          const uint16_t *v, int64_t v_stride, const uint16_t *q_norm, const uint16_t *k_norm,
                          float eps, const double *inv_freq, int64_t rotary_dim, int interleaved, uint16_t *q_out,
                          int64_t q_out_stride, void *stream);

/*
 * qlin_causal_plan -- the kernel and work split qlin_causal_attention would use,
 * without launching anything (the device arrays of batch are not read and may be
 * NULL).
 *   splits           0 = the planner's choice, else the number of key ranges
 *                    (at most 256)
 * Outputs (each may be NULL): *splits_out, *workspace_bytes (0 when one range
 * suffices), and text such as "kernel=k_causal_few splits=32 grid=256 combine=1"
 * in buf (at most buflen bytes).
 * Errors: INVALID, UNSUPPORTED, HIP (device query).
 */
int qlin_causal_plan(const qlin_batch *batch, int64_t q_heads, int64_t kv_heads, int64_t head_dim, int64_t splits,
                     int64_t *splits_out, int64_t *workspace_bytes, char *buf, int64_t buflen);

/*
 * qlin_causal_attention -- for the new token of row m at position p of its
 * sequence, every query head h and key/value head g = h / (q_heads / heads):
 *   s_j = scale * q[m][h] . k[g][j],  j <= p       (fp32)
 *   out[m][h] = RNE_bf16( sum_j softmax_j(s) v[g][j] )
 * A token that sees no key (p < 0, or a sequence without cached tokens) gives
 * zeros; one whose visible scores are all -infinity gives NaN (its softmax is 0 / 0),
 * as does one with a score of +infinity or NaN.  Keys and values behind p, infinities
 * and NaN among them, have no influence.  Scores, softmax statistics and sums are
 * fp32; each weight is rounded to bf16 once (the matrix cores' operand) and the sum
 * adds the rounded weights.
 *
 *   q, out      DEVICE bf16 rows of q_heads x 128, q_stride / out_stride elements
 *               apart (multiples of 8), 16-byte aligned; out must not share elements
 *               with q nor overlap the cache, the workspace or the batch's arrays
 *   q_heads     a multiple of cache->heads, at most 64 times it, at most 4096
 *   scale       > 0, scale log2(e) a finite float, or 0 for 1 / sqrt(128)
 *   workspace   DEVICE scratch of the bytes qlin_causal_plan reports for the same
 *               arguments (NULL when 0), 16-byte aligned, no initialisation, apart from
 *               q, out, the cache and the batch's arrays
 * max_new chooses the kernel: a batch of single tokens is read at the cache's rate only
 * if max_new says 1, so single tokens and long chunks are better two calls.
 * For fixed splits the same inputs give the same bits.  Calls sharing a workspace
 * must be ordered on one stream.
 * Errors: INVALID (NULL, sizes, overlap, workspace too small), UNSUPPORTED
 * (head_dim != 128, limits), ALIGN, HIP.
 */
int qlin_causal_attention(const qlin_batch *batch, const qlin_kv_cache *cache, int64_t q_heads, int64_t head_dim,
                          float scale, int64_t splits, const uint16_t *q, int64_t q_stride, uint16_t *out,
                          int64_t out_stride, void *workspace, int64_t workspace_bytes, void *stream);

/*
 * qlin_verify_plan -- device workspace of qlin_verify_draft for n_seq sequences of
 * up to n_draft drafted tokens over a vocabulary, in *workspace_bytes.
 * Errors: INVALID, UNSUPPORTED (limits).
 */
int qlin_verify_plan(int64_t n_seq, int64_t n_draft, int64_t vocab, int64_t *workspace_bytes);

/*
 * qlin_verify_draft -- keep the longest accepted prefix of each sequence's drafted
 * tokens and choose the token behind it, so that the tokens are distributed as the
 * target alone would draw them (the loop is lossless, Sec. 2.2).  Sequence b, with
 * n = count[b] drafted tokens x_0 .. x_{n-1} and uniform numbers u in [0, 1):
 *   P_i = softmax(target[b][i] / T),  i <= n;  T = temperature[b]
 *   Q_i = softmax(draft[b][i] / T),  i < n;  all mass on x_i if draft is NULL
 *   a = the first i with not u[b][i] Q_i(x_i) < P_i(x_i), or n
 *   W = max(P_a - Q_a, 0) (P_a itself where that is zero everywhere) if a < n, or P_n;
 *       a difference below 2^-44 P_a is the rounding of 64-bit sums and counts as zero
 *   next = the lowest index whose running sum of W exceeds u[b][n_draft] sum(W)
 *          (the last index of positive W if rounding leaves none); tokens less likely
 *          than 2^-900 times the row's likeliest may count as impossible
 * T = 0 (or below, or NaN) is the greedy limit: P_i is the lowest index of the
 * largest logit, Q_i all mass on x_i.  A logit of -infinity or NaN is a masked token
 * of probability 0.  A row without any token has P = 0 everywhere; next is then -1.
 * A drafted token outside [0, vocab) has probability 0.  Each weight e^(x / T) has a
 * relative error of at most 7e-11, sums are 64-bit, in a fixed order: the same
 * inputs give the same tokens.
 *
 *   target      DEVICE bf16 [n_seq][n_draft + 1][vocab], rows target_stride
 *               elements apart, 16-byte aligned
 *   draft       DEVICE bf16 [n_seq][n_draft][vocab], rows draft_stride apart, 16-byte
 *               aligned, or NULL
 *   drafted     DEVICE int32 [n_seq][n_draft]
 *   count       DEVICE int32 [n_seq], clamped to [0, n_draft], or NULL: n_draft each
 *   temperature DEVICE float [n_seq], or NULL: 1
 *   uniform     DEVICE float [n_seq][n_draft + 1]
 *   accepted    DEVICE int32 [n_seq] output: a
 *   tokens      DEVICE int32 [n_seq][n_draft + 1] output: x_0 .. x_{a-1}, next, then -1
 *   workspace   DEVICE scratch of at least qlin_verify_plan's bytes, 16-byte
 *               aligned, no initialisation
 * 0 <= n_draft <= 64 (0: plain sampling; drafted may then be NULL), 1 <= vocab <=
 * 2^24, n_seq <= 65535 (0 is a no-op).  Outputs and the workspace must not overlap
 * inputs or each other.
 * Calls sharing a workspace must be ordered on one stream.
 * Errors: INVALID, UNSUPPORTED, ALIGN, HIP.
 */
int qlin_verify_draft(int64_t n_seq, int64_t n_draft, int64_t vocab, const uint16_t *target, int64_t target_stride,
                      const uint16_t *draft, int64_t draft_stride, const int32_t *drafted, const int32_t *count,
                      const float *temperature, const float *uniform, int32_t *accepted, int32_t *tokens,
                      void *workspace, int64_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* QLIN_TARGET_H */
