/*
 * qlin_lowbit.h -- C ABI of a target layer's operators in fewer bits, on MI355X
 * (gfx950): the norms around a block with its gate and the residual, the linear of
 * 8-bit integers with the quantization of its tokens, and the key/value cache in 4
 * bits with its append and its causal attention.  Part of libqlin.so; status codes,
 * qlin_last_error() and qlin_last_status() are those of qlin.h, batches those of
 * qlin_target.h.
 *
 * Beside the W4A16 linears (Kim, Lee, Kim, arXiv 2607.04244, Sec. 2.1) these serve
 * what a long step is bound by: the matrix cores in prompts, which take 8-bit integers
 * at twice the rate of bf16, and the cache in long contexts, which 4 bits make 3.8
 * times smaller.  Inference only: none has a backward pass.
 *
 * Conventions of qlin.h: bf16 values travel as uint16_t bit patterns, every call is
 * asynchronous on its stream and returns a QLIN_* status, argument checks run before
 * any HIP call.
 */
#ifndef QLIN_LOWBIT_H
#define QLIN_LOWBIT_H

#include <stdint.h>

#include "qlin_target.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * qlin_block_norm -- between two blocks of a layer, for every row m, in fp32:
 *   t = y[m]; t = norm(t, post_norm); t = t * act(gate)
 *   h = RNE_bf16(residual[m] + scale t)                          -> residual_out[m]
 *   out[m] = RNE_bf16(norm(h, pre_norm))
 *   norm(x, w)[i] = x[i] / sqrt(mean(x^2) + eps) * w[i]; the squares' sum is fp32, so
 *   a row of values above 2^60 comes out as zeros, and with eps 0 one below 2^-60 loses
 *   bits, down to no numbers at all.  act is the identity, or the
 *   logistic function with gate_sigmoid.
 * Left out where its argument is NULL: the norm of y (post_norm), the gate, and the
 * second norm (pre_norm and out both NULL).  With y NULL the residual is normed as it
 * is (residual_out, post_norm and gate NULL too; scale unused).
 *
 *   y, residual, residual_out, out   DEVICE bf16 rows, strides in elements, multiples
 *               of 8.  An output may be y or residual themselves (same stride), not
 *               both outputs the same; other overlaps are errors
 *   post_norm, pre_norm   DEVICE bf16 [width]
 *   gate        DEVICE bf16 rows gate_stride apart, or [width] for all rows with
 *               gate_stride 0
 *   width       a multiple of 8, 8 .. 65536;  rows 0 .. 2^22 - 1 (0 is a no-op)
 *   scale       finite;  eps >= 0
 * All pointers 16-byte aligned.
 * Errors: INVALID, UNSUPPORTED (limits), ALIGN, HIP.
 */
int qlin_block_norm(int64_t rows, int64_t width, const uint16_t *y, int64_t y_stride, const uint16_t *residual,
                    int64_t residual_stride, const uint16_t *post_norm, const uint16_t *gate, int64_t gate_stride,
                    int gate_sigmoid, float scale, const uint16_t *pre_norm, float eps, uint16_t *residual_out,
                    int64_t residual_out_stride, uint16_t *out, int64_t out_stride, void *stream);

/*
 * qlin_quantize_tokens -- 8-bit integers with one scale a token, for qlin_eight_bit_linear:
 *   v = x[m], or silu(a) b with a = x[m][0 .. width), b = x[m][width .. 2 width) if
 *       gated (silu(a) = a / (1 + e^-a), in fp32)
 *   scale[m] = max |v| / 127  (fp32);  codes[m][i] = RNE(v[i] / scale[m]), -127 .. 127
 * A row with an infinity or NaN has scale NaN and codes 0; one whose largest value is
 * below 2^-100 counts as zeros (scale 0).  Rows of bf16 weights, a channel each, give that
 * linear's w and w_scale in the same way.
 *   x           DEVICE bf16 rows x_stride elements apart (a multiple of 8)
 *   codes       DEVICE int8 rows codes_stride apart (a multiple of 16)
 *   scale       DEVICE float [rows]
 *   width       a multiple of 16, 16 .. 65536;  rows 0 .. 2^22 - 1 (0 is a no-op)
 * x and codes 16-byte aligned; the outputs must not overlap x or each other.
 * Errors: INVALID, UNSUPPORTED, ALIGN, HIP.
 */
int qlin_quantize_tokens(int64_t rows, int64_t width, const uint16_t *x, int64_t x_stride, int gated, int8_t *codes,
                         int64_t codes_stride, float *scale, void *stream);

/*
 * qlin_eight_bit_plan -- the kernel and work split qlin_eight_bit_linear would use, without
 * launching anything.
 *   splits           0 = the planner's choice, else the number of K ranges (at most 64,
 *                    clamped to the steps of K there are)
 * Outputs (each may be NULL): *splits_out, *workspace_bytes (0 with one range), text in
 * buf (at most buflen bytes).
 * Errors: INVALID, UNSUPPORTED, HIP (device query).
 */
int qlin_eight_bit_plan(int64_t M, int64_t N, int64_t K, int64_t splits, int64_t *splits_out,
                        int64_t *workspace_bytes, char *buf, int64_t buflen);

/*
 * qlin_eight_bit_linear -- y[m][n] = RNE_bf16( float(sum_k x[m][k] w[n][k]) * (x_scale[m] * w_scale[n]) )
 * The sum is a 32-bit integer, exact for any order of its terms; its conversion and
 * the two products are fp32.
 *   x           DEVICE int8 [M] rows x_stride bytes apart;  x_scale DEVICE float [M]
 *   w           DEVICE int8 [N] rows w_stride bytes apart;  w_scale DEVICE float [N]
 *   y           DEVICE bf16 [M] rows y_stride elements apart (a multiple of 8)
 *   K           a multiple of 16, 16 .. 131056 (where sums of products of -128 .. 127
 *               stay below 2^31); 0 <= M <= 2^22 (0 is a no-op), 1 <= N <= 2^22
 *   workspace   DEVICE scratch of the bytes qlin_eight_bit_plan reports for the same arguments
 *               (NULL when 0), 16-byte aligned, no initialisation
 * x, w and y 16-byte aligned, x_stride and w_stride multiples of 16; scales 4-byte
 * aligned.  y and the workspace must not overlap inputs or each other.
 * Calls sharing a workspace must be ordered on one stream.
 * Errors: INVALID, UNSUPPORTED, ALIGN, HIP.
 */
int qlin_eight_bit_linear(int64_t M, int64_t N, int64_t K, int64_t splits, const int8_t *x, int64_t x_stride,
                          const float *x_scale, const int8_t *w, int64_t w_stride, const float *w_scale, uint16_t *y,
                          int64_t y_stride, void *workspace, int64_t workspace_bytes, void *stream);

/*
 * The key/value cache in 4 bits: slot s of key/value head h is row s * token_stride +
 * h * head_stride.  A row stands for 128 values step * c[d] + offset: 16 words of eight
 * codes, that of dimension d in bits 4 (d % 8) .. + 3 of word d / 8, and a pair of bf16
 * (step, offset), either of any sign.  Layouts, rooms, capacity and cache_start as for
 * qlin_kv_cache, in rows: [sequences][heads][capacity] has token_stride 1, head_stride
 * capacity, seq_slots heads * capacity; [tokens][heads] has token_stride heads,
 * head_stride 1.
 */
typedef struct qlin_kv4_cache {
    int64_t capacity;             /* slots of one sequence's room, 0 .. 2^40; 0: no bound but slots */
    uint32_t *k, *v;              /* DEVICE, 16-byte aligned: row r at word 16 r */
    uint16_t *k_grid, *v_grid;    /* DEVICE, 4-byte aligned: row r at element 2 r */
    int64_t heads;                /* key/value heads */
    int64_t slots;                /* slots that may be addressed: s < slots, 1 .. 2^40 */
    int64_t token_stride;         /* rows, 1 .. 2^20 */
    int64_t head_stride;          /* rows, 1 .. 2^36 */
    int64_t seq_slots;            /* slots between sequences where cache_start is NULL, and between rooms */
} qlin_kv4_cache;

/*
 * qlin_norm_rope_append_four_bit -- qlin_norm_rope_append into a 4-bit cache: q_out is the
 * same, and the keys' and values' rows of 128 bf16 values x (keys after norm and
 * rotation, which for them run in 64 bits, where no square or product of bf16 values
 * leaves the range, rounded once to fp32 and from there to bf16) are stored as
 *   offset = min(x), step = RNE_bf16((max(x) - offset) / 15), both steps fp32
 *   c[d] = min(RNE((x[d] - offset) / step), 15), ties to even, or 0 where step is 0
 * A step below 2^-126 is 0.  A row with an infinity or NaN, or whose max - min is past
 * fp32, has step and offset NaN and stands for NaN throughout.
 * Arguments, sequences and errors as qlin_norm_rope_append; two new tokens must not
 * share a slot.
 */
int qlin_norm_rope_append_four_bit(const qlin_batch *batch, const qlin_kv4_cache *cache, int64_t q_heads,
                                   int64_t head_dim, const uint16_t *q, int64_t q_stride, const uint16_t *k,
                                   int64_t k_stride, const uint16_t *v, int64_t v_stride, const uint16_t *q_norm,
                                   const uint16_t *k_norm, float eps, const double *inv_freq, int64_t rotary_dim,
                                   int interleaved, uint16_t *q_out, int64_t q_out_stride, void *stream);

/*
 * qlin_unpack_four_bit -- RNE_bf16(step * c + offset) (one fp32 fused product) of the batch's
 * cached tokens into a bf16 cache of as many heads: token j of sequence b goes from its
 * slot of `cache` to the same slot of `to`.  new_only: the new tokens (the first max_new of
 * the last new_start[b + 1] - new_start[b]), else all, those of sequences without new
 * tokens too.  batch->rows only bounds new_start.  A sequence whose slots are not inside
 * both caches and their rooms, or that is longer than max_len, counts as one without
 * cached tokens.  Sequences sharing slots store the same values there.
 * Errors: INVALID (NULL, sizes, the caches overlap, different heads), UNSUPPORTED, ALIGN, HIP.
 */
int qlin_unpack_four_bit(const qlin_batch *batch, const qlin_kv4_cache *cache, const qlin_kv_cache *to,
                         int64_t head_dim, int new_only, void *stream);

/*
 * qlin_causal_four_bit_plan -- as qlin_causal_plan, for qlin_causal_attention_four_bit.  Long
 * chunks take "unpack" forms where that is estimated faster and at most 16 GiB: the
 * workspace then holds the batch's cache in f16 (512 bytes a slot and head of n_seq *
 * heads * max_len, and 4 for powers of two of its rows) and what qlin_causal_attention
 * needs.  Every sequence has room for max_len there, so that is as much as a bf16 cache of
 * such rooms and more than a packed one: keep max_len near the longest length, and large
 * chunks of a few sequences a call where memory is short.
 * Errors: INVALID, UNSUPPORTED, HIP (device query).
 */
int qlin_causal_four_bit_plan(const qlin_batch *batch, int64_t q_heads, int64_t kv_heads, int64_t head_dim,
                              int64_t splits, int64_t *splits_out, int64_t *workspace_bytes, char *buf, int64_t buflen);

/*
 * qlin_causal_attention_four_bit -- qlin_causal_attention over a 4-bit cache: the keys and
 * values are step * c + offset.  What differs from qlin_causal_attention:
 *   - a sequence longer than max_len counts as one without cached tokens (its rows
 *     are zeros): max_len sizes the workspace;
 *   - the products of q with codes are scaled afterwards, in fp32, so the sum of a
 *     row's |q| and the cache's steps and offsets should be below 2^56, where nothing
 *     overflows; beyond, rows may come out as NaN.  Sizes below 2^-84 lose bits;
 *   - products run in f16: q, taken to f16's range by a power of two a row, and each
 *     weight times its value's step are rounded to 11 bits once, codes are exact, and
 *     offsets are added in fp32; in the unpack forms keys and values are rounded to 11
 *     bits instead, and weights as well.  The powers of two change what is rounded away,
 *     nothing else.
 * A token that sees no key gives zeros; codes, steps and offsets behind a token's
 * position, infinities and NaN among them, take no part in its result.  The forms that read
 * codes keep its every bit whatever lies there; in the unpack forms the powers of two go
 * by all finite rows of a sequence, so there finite later rows far larger or smaller than
 * the earlier ones can change how these are rounded.
 * Errors: as qlin_causal_attention.
 */
int qlin_causal_attention_four_bit(const qlin_batch *batch, const qlin_kv4_cache *cache, int64_t q_heads,
                                   int64_t head_dim, float scale, int64_t splits, const uint16_t *q, int64_t q_stride,
                                   uint16_t *out, int64_t out_stride, void *workspace, int64_t workspace_bytes,
                                   void *stream);

#ifdef __cplusplus
}
#endif

#endif /* QLIN_LOWBIT_H */
