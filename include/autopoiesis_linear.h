/*
 * autopoiesis_linear.h -- C ABI of the weights of a serving replica in 4 bits, and of its answers (MI355X, gfx950).
 *
 * Beside the cache and attention (autopoiesis_attn.h) a replica's step is products of its tokens' rows with the model's
 * weights, and at its end the probabilities of tokens.  These calls are that part: packing weights in 4 bits, products with
 * them (for one token as for whole prompts), the gated half of a feed-forward block, and log probabilities of given tokens
 * with entropy and alternatives.
 *
 * All pointers inside the structures are DEVICE pointers; the structures themselves are read on the host during the call.
 * All calls return an ap_status and never throw or abort, allocate nothing, keep nothing from one call for the next,
 * and run on the caller's stream (a hipStream_t; NULL is the default stream), so a stream capture records them.
 * Strides are in bytes and not negative; rows that a call writes do not overlap (rows that it reads may).  What lies on the
 * device cannot be checked by the host; whatever it holds, no kernel reads or writes outside the memory that is described
 * here.  Results do not depend on timing.
 * A workspace is device memory of at least the bytes that the call named ..._workspace gives for the same description, aligned
 * to 16 bytes (it may be NULL where that is 0), for the call alone until it has run.
 * Errors: AP_ERR_INVALID (null, zero, misaligned or contradicting arguments, an unknown type, a workspace that is too small),
 * AP_ERR_RANGE (more rows than a grid holds), AP_ERR_DEVICE.
 */
#ifndef AUTOPOIESIS_LINEAR_H
#define AUTOPOIESIS_LINEAR_H

#include <stdint.h>

#include "autopoiesis_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

#define AP_FP32 2u              /* for logits */
#define AP_SILU 0u
#define AP_GELU 1u

/* Weights [n_out][n_in] in 4 bits; n_in is a multiple of 8, n_out any number.  A row is blocks = (n_in + 127) / 128 blocks of
 * 128 columns, the last one filled up.
 *   codes : row r at codes + r * code_stride, blocks * 64 bytes.  Block b is 16 words of 32 bits; word 4 q + m of it has the
 *           columns 128 b + 32 m + 8 q + j, j = 0 .. 7: an even j in bits 2 j .. 2 j + 3, an odd one in bits 2 j + 14 ..
 *           2 j + 17.  Address and stride are multiples of 16.
 *   pairs : row r at pairs + r * pair_stride: for each `group` (32, 64 or 128) columns of the blocks a pair (step, lo) of the
 *           16-bit type `dtype`.  Address and stride are multiples of a block's bytes, 512 / group.
 * A code stands for lo + step * code.  Columns from n_in on stand for nothing, but pairs of groups that have no other column have to
 * be numbers (ap_weights_pack makes them zero).  n_out, n_in and n_out * blocks are below 2^31. */
typedef struct {
    uint32_t dtype, group, n_out, n_in;
    void *codes, *pairs;
    int64_t code_stride, pair_stride;
} ap_weights;

/* Rows [token][..] of values of the 16-bit type.  Where rows are read as a matrix of inputs or of weights, data and stride
 * are multiples of 16 bytes; elsewhere of 2. */
typedef struct {
    void *data;
    int64_t stride;
} ap_vectors;

/* Pack n_out rows of n_in values (16-byte aligned).  As the cache does it: a group gets lo = its smallest value, step = (largest -
 * lo) / 15 rounded up to the 16-bit type (down where 15 steps up from lo would leave the type's range), and code = (x - lo) / step
 * rounded to the nearest (ties to even); where a group holds a NaN or an infinity its pair is NaN.  Columns from n_in on get zeros. */
ap_status ap_weights_pack(const ap_weights *weights, const ap_vectors *values, void *stream);

/* The values that packed weights stand for (16-byte aligned): lo + step * code in 32 bits, rounded once. */
ap_status ap_weights_read(const ap_weights *weights, const ap_vectors *values, void *stream);

/* y = x W^T (+ add) for n_tokens rows: y[t][n] = add[t][n] + sum_k x[t][k] (lo + step * code)[n][k], in 32 bits with each
 * rounded once, at its end.  x (16-byte aligned) has n_in columns, y and add have n_out; all are of the weights' type.  add may
 * be NULL, or y itself; with a stride of 0 it is a bias.  y must not overlap x.  Rows are apart: what is not a number in one
 * of x reaches only the same row of y.  A call gives the same each time; the order in which a sum's terms are added goes by
 * n_out, n_in, n_tokens and the output's place, so the same product in a larger matrix or among other rows can differ by
 * roundings in 32 bits.  No weight is rounded: sums over a group's columns of x (16 + code) and of x meet
 * step and lo - 16 step in 32 bits.  Where such a sum or product passes 32 bits (x and weights of 2^120 and more) or x holds an
 * infinity the row can be NaN.  Fewer tokens can need a larger workspace than more do (their inputs are cut into more parts): one
 * buffer for several numbers of tokens has the largest of what they need. */
ap_status ap_linear_workspace(const ap_weights *weights, uint32_t n_tokens, uint64_t *bytes);
ap_status ap_linear(const ap_weights *weights, const ap_vectors *x, const ap_vectors *add, const ap_vectors *y, uint32_t n_tokens,
                    void *workspace, uint64_t workspace_bytes, void *stream);

/* h[t][i] = act(x . gate_i) (x . up_i) in 32 bits, rounded once: the half of a feed-forward block that comes before its last
 * product.  gate and up are alike in type, group and sizes; h must not overlap x.  act: AP_SILU is g / (1 + e^-g), AP_GELU is
 * g (1 + tanh(sqrt(2 / pi) (g + 0.044715 g^3))) / 2. */
ap_status ap_gated_workspace(const ap_weights *gate, const ap_weights *up, uint32_t n_tokens, uint64_t *bytes);
ap_status ap_gated(const ap_weights *gate, const ap_weights *up, const ap_vectors *x, const ap_vectors *h, uint32_t n_tokens,
                   uint32_t act, void *workspace, uint64_t workspace_bytes, void *stream);

/* Rows of logits [n_rows][vocab]: AP_BF16, AP_FP16 or AP_FP32, data and stride multiples of a value's bytes. */
typedef struct {
    uint32_t dtype, n_rows, vocab;
    void *data;
    int64_t stride;
} ap_logits;

/* With p = e^s / sum e^s over s = scale * logits (one over the temperature; log2(e) times it is at least 2^-120 and finite), of each
 * row:
 *   logprob     : log p of tokens[row], 0 where that is outside [0, vocab); tokens may be NULL, then logprob is too.
 *   entropy     : - sum p log p; may be NULL.
 *   top_id, top_logprob : [n_rows][top], the `top` (at most 64) tokens of the largest logits, of equal ones the lowest token
 *                 first, and their log p.  Places beyond the tokens that are above minus infinity get -1 and minus infinity.
 * A logit of minus infinity is a token that is ruled out.  In a row where all are, log p is minus infinity and the entropy 0.  Where
 * a row holds a NaN or plus infinity, its logprob, entropy and top_logprob are NaN (0 still where no token is given), and what is
 * not a number is no alternative.  Sums are in 32 bits; what is made of them is in 64, and rounded once. */
ap_status ap_logprobs_workspace(const ap_logits *logits, uint32_t top, uint64_t *bytes);
ap_status ap_logprobs(const ap_logits *logits, const int32_t *tokens, float scale, uint32_t top, float *logprob, float *entropy,
                      int32_t *top_id, float *top_logprob, void *workspace, uint64_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* AUTOPOIESIS_LINEAR_H */
