/*
 * dmi_kv8.h -- operators on a paged KV cache held in 8 bits (gfx950), part of libdmi.so.
 *
 * A serving program keeps K and V of every cached token as e4m3 codes with one fp32 scale per
 * (block of tokens, head); it appends the tokens of a step, attends over the cache, and, where a
 * request has outgrown its budget, keeps the tokens that received the most attention.  The weight
 * that attention gave to every cached token exists nowhere outside the attention kernel; dmi_kv8_attend
 * writes it out, for eviction and for observation alike (a row of it is an fp32 row that dmi_observe takes).
 *
 *   dmi_kv8_append   x (bf16 / fp16 / fp32) -> codes and scales
 *   dmi_kv8_attend   softmax attention of the newest tokens of each request over its cache
 *   dmi_kv8_evict    the tokens with the largest weights and the newest ones, moved into other blocks
 *
 * Conventions are those of dmi.h: pointers are marked [host] or [device], the caller owns all memory and
 * keeps it valid until the launched kernels have run, no call synchronises, allocates or copies from the
 * device, every call launches on hip_stream of the calling thread's current device and returns a status,
 * dmi_last_error() has the message, nothing throws.  The calls may be recorded into a graph; contents of
 * device memory (lengths, tables, tensors) may then change between replays.
 *
 * Values in device memory cannot be checked by the host.  The kernels never leave the given tensors:
 * a length counts as at least 0 and at most max_len, a number of new tokens as at most max_new, rows past
 * total_new do not exist, a request whose row lies outside the block table is as one of length 0, and tokens
 * of a block whose entry lies outside the cache are neither stored nor attended to.
 */
#ifndef DMI_KV8_H
#define DMI_KV8_H

#include "dmi.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The cache.  Element (block b, slot s, head h, dim d) of K or V is the code at
 * base + b*block_stride + s*slot_stride + h*head_stride + d (strides in bytes, the same for K and V); it stands for
 * number(code) * scale, scale at scale_base + b*scale_block_stride + h*scale_head_stride (in floats), a positive normal number.
 * k, v 16-byte aligned, strides multiples of 16 bytes, slot_stride from 0 to 2^26.  block_size: a multiple of 16, at most 1024.  head_dim: a multiple of 16, at
 * most 256.  block_table_dev [device] int32 [n_seqs][block_table_stride], of which max_blocks columns are used (rows do not
 * overlap: block_table_stride >= max_blocks): physical block of logical block t / block_size of a sequence. */
typedef struct {
    void *k, *v;                /* [device] e4m3 codes */
    float *k_scale, *v_scale;   /* [device] */
    int64_t block_stride, slot_stride, head_stride;
    int64_t scale_block_stride, scale_head_stride;
    uint32_t block_size, n_heads, head_dim;
    uint32_t n_blocks;          /* physical blocks */
    uint32_t n_seqs, max_blocks;    /* rows and columns of the block table */
    const int32_t *block_table_dev; /* [device] */
    int64_t block_table_stride;
} dmi_kv8_t;

/* The requests of a call.
 *   lens_dev   [device] n_reqs lengths: tokens in the cache, those of this call included
 *   starts_dev [device] n_reqs + 1 offsets, ascending: request r's new tokens are rows starts[r] .. starts[r+1]-1 of
 *              the tensors of new tokens, and the last of its length.  NULL: one new token each, row r
 *              (total_new = n_reqs, max_new = 1).
 *   rows_dev   [device, optional] n_reqs different rows of the block table (and of weights); NULL: request r has row r.
 * total_new, max_new, max_len are upper bounds of the rows, of one request's new tokens and of the lengths: launches
 * are sized by them (n_reqs * max_len at most 2^35 for dmi_kv8_attend). */
typedef struct {
    uint32_t n_reqs, total_new, max_new, max_len;
    const int32_t *lens_dev, *starts_dev, *rows_dev;
} dmi_kv8_batch_t;

/* Rows of heads: element (row i, head h, dim d) at data + i*row_stride + h*head_stride + d, strides in elements.
 * data 16-byte aligned, strides multiples of 16 bytes. */
typedef struct {
    void *data;                 /* [device] */
    uint32_t dtype;             /* DMI_DTYPE_* */
    int64_t row_stride, head_stride;
} dmi_kv8_heads_t;

/* fp32 weights of cached tokens: (row r of the block table, head h, position t) at data + r*row_stride + h*head_stride + t. */
typedef struct {
    float *data;                /* [device] */
    int64_t row_stride, head_stride;
} dmi_kv8_weight_t;

/*
 * Writes the new tokens' K and V (BF16 / FP16 / FP32, total_new rows of n_heads heads) into their places.  For every block
 * they reach and every head, K and V apart:
 *     a = max |x| over the new tokens in the block (finite ones),   s = the smallest power of two >= a / 448, at least 2^-100,
 *     s = max(s, its scale) if the block holds older tokens, whose codes become RN(code * scale / s),
 *     code = RN(x / s), RN to the nearest e4m3 number, ties to even; +-inf -> +-448, NaN -> NaN.
 * A power of two moves codes without rounding them again, except where they leave e4m3's normal range.
 * Slots behind the last new token keep their bytes.
 */
dmi_status_t dmi_kv8_append(const dmi_kv8_t *cache /*[host]*/, const dmi_kv8_batch_t *batch /*[host]*/,
                            const dmi_kv8_heads_t *key /*[host]*/, const dmi_kv8_heads_t *value /*[host]*/,
                            void *hip_stream);

/*
 * Causal attention of the new tokens over the cache (which holds them: append first).  Query i of a request's n new tokens
 * sees positions t <= len - n + i.  Query heads h*g .. h*g+g-1 read head h of the cache, g = n_q_heads / n_heads.
 *     z_t = scale * q . k_t,   p = softmax(z),   out = sum_t p_t v_t,   lse = log sum_t exp(z_t)
 * A query that sees nothing (or no score above -inf) gives out = 0 and lse = -inf.  A NaN in K makes the queries that see it NaN, a NaN in V that
 * element of theirs.
 *   q, out     BF16 or FP16, the same; total_new rows of n_q_heads heads (at most 2^30 of them in all).  out may be q, or share no
 *              element with it; where weights are asked for it shares none
 *   lse_dev    [device, optional] fp32 [total_new][n_q_heads]
 *   weight     [host, optional] for every request, head of the cache and position t < len:
 *              weight = decay * prior + sum of p_t over the call's new tokens and the g query heads (without new tokens: decay * prior).
 *              prior [host, optional]: the same layout, may be the same memory; positions of new tokens count as 0 in it.
 *   workspace  [device] 256-byte aligned, at least dmi_kv8_attend_workspace(...) bytes; contents need not be kept.  (That function
 *              looks at sizes alone, and gives 0 for those that this call refuses.)
 * Scores, softmax, sums and weights are fp32; products are of q as it is and the codes' exact values; p (with what V's scale is between
 * powers of two) is rounded to q's type for its product with V.  In fp16 the scales that V has within 64 tokens may lie 2^22 apart; what
 * lies below that is rounded to 2^-32 of the largest.
 */
uint64_t dmi_kv8_attend_workspace(const dmi_kv8_t *cache /*[host]*/, const dmi_kv8_batch_t *batch /*[host]*/,
                                  uint32_t n_q_heads, int with_weight);
dmi_status_t dmi_kv8_attend(const dmi_kv8_t *cache /*[host]*/, const dmi_kv8_batch_t *batch /*[host]*/,
                            const dmi_kv8_heads_t *q /*[host]*/, uint32_t n_q_heads, float scale,
                            const dmi_kv8_heads_t *out /*[host]*/, float *lse_dev,
                            const dmi_kv8_weight_t *weight /*[host]*/, const dmi_kv8_weight_t *prior /*[host]*/, float decay,
                            void *workspace, uint64_t workspace_bytes, void *hip_stream);

/*
 * Cuts requests longer than `keep` to `keep` tokens, for every head of the cache by itself: the last `recent` ones, and of
 * the others the keep - recent with the largest weights (equal weights: the lowest position; NaN counts as -inf).  They
 * stay in order of position, and are copied into the blocks that `to`'s table (same row numbers, n_heads, head_dim and
 * block_size) lists, whose scale becomes the largest among the tokens that meet in it (a code becomes
 * RN(code * scale / new scale)).  Shorter requests are copied whole.  `to` may lie in the same memory, but no block that it
 * lists may be listed by `cache` for a row of this call.  new_len = min(len, keep).
 *   batch         lens_dev, rows_dev, n_reqs and max_len are used
 *   to_weight     [host] the kept tokens' weights, in their new positions (not in weight's memory)
 *   positions_dev [device] int32 [n_reqs][n_heads][keep]: the kept tokens' old positions, -1 from new_len on
 *   to_lens_dev   [device] int32 [n_reqs]: the new lengths (not in lens_dev's memory)
 */
dmi_status_t dmi_kv8_evict(const dmi_kv8_t *cache /*[host]*/, const dmi_kv8_batch_t *batch /*[host]*/,
                           const dmi_kv8_weight_t *weight /*[host]*/, const dmi_kv8_t *to /*[host]*/,
                           const dmi_kv8_weight_t *to_weight /*[host]*/, uint32_t keep, uint32_t recent,
                           int32_t *positions_dev, int32_t *to_lens_dev, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* DMI_KV8_H */
