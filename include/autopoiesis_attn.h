/*
 * autopoiesis_attn.h -- C ABI of the cache and attention operators of a serving replica (MI355X, gfx950).
 *
 * The evaluator prices a replica's prefill and decode steps (autopoiesis_eval.h); the part of those costs that goes by
 * the lengths in a trace is the cache of keys and values and the attention that reads it.  These calls are that part
 * itself: appending the new tokens of a batch of sequences to a paged cache with the position rotation on the way,
 * attention of the new tokens over their sequences, and reading rows of the cache back.  A replica's step can so be
 * run, or measured by length and handed to ap_costtable_set.
 *
 * All pointers inside the structures are DEVICE pointers; the structures themselves are read on the host during the call.
 * All calls return an ap_status and never throw or abort, allocate nothing, keep nothing from one call for the next,
 * and run on the caller's stream (a hipStream_t; NULL is the default stream), so a stream capture records them.
 * Strides are in bytes.  Lengths, tables and offsets on the device cannot be checked by the host; whatever they hold,
 * no kernel reads or writes outside the memory that is described here.
 */
#ifndef AUTOPOIESIS_ATTN_H
#define AUTOPOIESIS_ATTN_H

#include <stdint.h>

#include "autopoiesis_eval.h"

#ifdef __cplusplus
extern "C" {
#endif

#define AP_BF16 0u
#define AP_FP16 1u

/* A cache of keys and values in pages.  A page holds page_size tokens (any number >= 1) of every key/value head.
 *   bits == 16 : row (page, head, slot) of k is head_dim values of the 16-bit type `dtype`, at
 *                k + page * page_stride + head * head_stride + slot * slot_stride.
 *   bits == 4  : the row is head_dim / 2 bytes of codes at the same kind of address, channel 2i in the low and channel
 *                2i + 1 in the high half of byte i; each 64 channels have a pair (step, lo) of the 16-bit type at
 *                k_pairs + page * pair_page_stride + head * pair_head_stride + slot * pair_slot_stride + 4 * (channel / 64);
 *                a code stands for lo + step * code.
 * The same strides hold for v and v_pairs.  head_dim is 64 or 128.  k, v and their strides are multiples of 16 bytes,
 * the pairs and theirs of 4 * head_dim / 64.  Strides are not negative. */
typedef struct {
    uint32_t dtype, bits;
    uint32_t n_pages, page_size, kv_heads, head_dim;
    void *k, *v;
    void *k_pairs, *v_pairs;
    int64_t page_stride, head_stride, slot_stride;
    int64_t pair_page_stride, pair_head_stride, pair_slot_stride;
} ap_kv_cache;

/* The sequences of a call and their new tokens.
 *   new_first  : int32 [n_seqs + 1], not decreasing, new_first[0] = 0 and new_first[n_seqs] = n_tokens: sequence s has
 *                the new tokens new_first[s] .. new_first[s + 1] - 1 of the call's rows (there may be none).
 *   kv_len     : int32 [n_seqs], the tokens that sequence s holds, its new ones included.  New token i of m is at
 *                position kv_len[s] - m + i; one whose position is negative is not in the cache and sees nothing.
 *   page_table : int32 [n_seqs] rows of table_width entries, table_stride entries apart: page of position p is entry
 *                p / page_size.  An entry outside [0, n_pages) is no page: its tokens are not there (never read, not
 *                written, seen by nobody), so pages that a window has left behind can be given away.
 *   max_new    : no sequence has more new tokens (rows beyond are left out of attention).
 *   max_kv     : positions from here on are taken as not there; at most table_width * page_size.  Grids and workspaces
 *                go by max_new and max_kv, so that no length has to come back to the host. */
typedef struct {
    uint32_t n_seqs, n_tokens, max_new, max_kv, table_width;
    const int32_t *new_first, *kv_len, *page_table;
    int64_t table_stride;
} ap_seq_batch;

/* Rows [token][head][head_dim] of the 16-bit type; data and strides are multiples of 16 bytes. */
typedef struct {
    void *data;
    int64_t token_stride, head_stride;
} ap_rows;

/* Position rotation: table float [n_positions][rot_dim / 2][2] holds (cos, sin).  The pair (a, b) of channels becomes
 * (a cos - b sin, a sin + b cos), in 32 bits and rounded once; neighbours == 0 pairs channel i with i + rot_dim / 2,
 * otherwise 2i with 2i + 1.  Channels from rot_dim on stay.  rot_dim is a multiple of 16, at most head_dim;
 * n_positions >= max_kv.  The table is aligned to 16 bytes. */
typedef struct {
    const float *table;
    uint32_t n_positions, rot_dim, neighbours;
} ap_rotation;

/* Append the batch's new tokens to the cache: keys rotated, values as they are.  In 4 bits each group of 64 channels
 * (after rounding to the 16-bit type) gets lo = its smallest, step = (largest - lo) / 15 rounded up to the 16-bit type
 * (down where 15 steps up from lo would leave the type's range), and code = (x - lo) / step rounded to the nearest (ties
 * to even); where a group holds a NaN or an infinity its pair is NaN.  With q (else NULL, then q_out is ignored): rows of
 * q_heads heads, rotated alike and written to q_out, which may be q itself; a token that has no position in
 * [0, min(kv_len, max_kv)) gets zeros.  rotation may be NULL: nothing turns.
 * Two tokens of one call that fall on the same slot (pages shared between sequences) leave either of them there.
 * Errors: AP_ERR_INVALID (null, zero, misaligned or contradicting arguments, an unknown type), AP_ERR_RANGE (a table that
 * is too short: n_positions < max_kv or table_width * page_size < max_kv; more rows than a grid holds), AP_ERR_DEVICE. */
ap_status ap_kv_append(const ap_kv_cache *cache, const ap_seq_batch *batch, const ap_rows *k, const ap_rows *v,
                       const ap_rotation *rotation, const ap_rows *q, const ap_rows *q_out, uint32_t q_heads, void *stream);

/* Read the batch's new tokens back from the cache as rows of the 16-bit type (in 4 bits: lo + step * code in 32 bits,
 * rounded once); rows that are not there get zeros.  A batch whose tokens are all "new" reads whole sequences. */
ap_status ap_kv_read(const ap_kv_cache *cache, const ap_seq_batch *batch, const ap_rows *k_out, const ap_rows *v_out,
                     void *stream);

/* Attention of the new tokens over their sequences, which the cache already holds (ap_kv_append first):
 *     out = sum_j w_j v_j / sum_j w_j,   w_j = exp(scale * q . k_j)   over the positions j that the token at p sees:
 *     j <= p, j < kv_len, j < max_kv, on a page, and with window > 0 also j > p - window or j < sinks.
 * A row that sees nothing (or only scores of minus infinity) is zero.  Keys and values that a row does not see do not
 * reach it, whatever they hold.  q_heads is a multiple of kv_heads: q head h reads key/value head h / (q_heads / kv_heads).
 * Scores, maxima and sums are in 32 bits.  Weights are rounded to 16 bits before they meet the values, and summed as rounded: that
 * moves a row by at most half a step of the type (2^-8 bf16, 2^-11 fp16) of the weighted mean of |v_j - out|, beside the half step of
 * its own last rounding.  With random rows the two together are 1.3 to 1.4 times the last rounding alone (0.0022 of a row's size
 * in bf16, 0.00027 in fp16).  Up to 32 rows over 4 bits round a weight times its key's step, against what codes are off the middle one.
 * Weights are held up to 2^15 times their size, so a row whose sum of values passes 2^112 can overflow to an infinity.  q . k, its
 * parts and scale times it are numbers of 32 bits: where one overflows, the row can be NaN.  Values in 4 bits are used as
 * lo + step * code with at least the 16-bit type's precision.
 *   scale     : > 0, and log2(e) times it finite.
 *   workspace : device memory of at least ap_attention_workspace bytes, aligned to 16 bytes (may be NULL where that
 *               is 0), for this call alone until it has run.
 * Results do not depend on timing.  Errors as above; a workspace that is too small is AP_ERR_INVALID. */
ap_status ap_attention_workspace(const ap_kv_cache *cache, const ap_seq_batch *batch, uint32_t q_heads, uint32_t window,
                                 uint32_t sinks, uint64_t *bytes);
ap_status ap_attention(const ap_kv_cache *cache, const ap_seq_batch *batch, const ap_rows *q, const ap_rows *out,
                       uint32_t q_heads, float scale, uint32_t window, uint32_t sinks, void *workspace,
                       uint64_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* AUTOPOIESIS_ATTN_H */
