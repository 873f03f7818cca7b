/*
 * dmi_kv8_long.h -- operators for long contexts on the 8-bit KV cache of dmi_kv8.h (gfx950), part of libdmi.so.
 *
 * The cache, the requests of a call and rows of heads are described by dmi_kv8.h's structs, and its conventions hold here:
 * asynchronous on hip_stream, nothing allocated, every content of device memory kept within the given tensors, calls may be
 * recorded into a graph.
 *
 *   dmi_kv8_append_rotated   dmi_kv8_append with K, and the call's queries, rotated by the tokens' positions on the way
 *   dmi_kv8_bound            the least and the largest K of blocks, as codes: what a selection goes by
 *   dmi_kv8_select           for each new token and head of the cache: the blocks that can hold the largest scores
 *   dmi_kv8_attend_blocks    attention over the blocks that are listed for each new token and head
 *   dmi_kv8_attend_shared    dmi_kv8_attend for groups of requests whose contexts begin alike: what they share is read once
 */
#ifndef DMI_KV8_LONG_H
#define DMI_KV8_LONG_H

#include "dmi_kv8.h"

#ifdef __cplusplus
extern "C" {
#endif

/* How tokens' positions rotate rows of a head: of its first rotary_dim elements, pair i is turned by position * freq[i] radians,
 *     x' = x cos - y sin,   y' = x sin + y cos,
 * the angle in 64 bits, its cosine and sine rounded to fp32; the other elements stay as they are.
 *   freq_dev       [device] fp32 [rotary_dim / 2]
 *   positions_dev  [device, optional] int32 [total_new]: the position of each new token.  NULL: its place in the cache, which runs
 *                  behind its position where dmi_kv8_evict has cut the request
 *   rotary_dim     a multiple of 16 up to head_dim
 *   pairs          0: pair i is elements i and i + rotary_dim / 2;  1: elements 2 i and 2 i + 1 */
typedef struct {
    const float *freq_dev;
    const int32_t *positions_dev;
    uint32_t rotary_dim, pairs;
} dmi_kv8_rotary_t;

/*
 * Writes the new tokens' K, rotated, and V into their places as dmi_kv8_append does (a rotated element is rounded to fp32, and from
 * there on is dmi_kv8_append's x).  With q, the new tokens' queries are rotated into q_out: those
 * of FP32 in 64 bits and rounded once, those of 16 bits in fp32 (at most three roundings: two products and their sum) and then rounded to their type.
 *   q, q_out  [host, optional, both or neither] total_new rows of n_q_heads heads, of key's dtype.  q_out may be q, or share no element
 *             with q, key or value.  Rows of tokens that no request has, or whose place lies below 0, are left as they were.  n_q_heads need
 *             not be a multiple of n_heads.
 */
dmi_status_t dmi_kv8_append_rotated(const dmi_kv8_t *cache /*[host]*/, const dmi_kv8_batch_t *batch /*[host]*/,
                                    const dmi_kv8_heads_t *key /*[host]*/, const dmi_kv8_heads_t *value /*[host]*/,
                                    const dmi_kv8_rotary_t *rotary /*[host]*/, const dmi_kv8_heads_t *q /*[host]*/,
                                    uint32_t n_q_heads, const dmi_kv8_heads_t *q_out /*[host]*/, void *hip_stream);

/* The least and the largest K of every block of a cache, head and element, as e4m3 codes that K's scale of that block and head multiplies:
 * (block b, head h, element d) at data + b*block_stride + h*head_stride + d, the largest head_dim behind the least.
 * data 16-byte aligned, strides multiples of 16 bytes. */
typedef struct {
    uint8_t *data;              /* [device] */
    int64_t block_stride, head_stride;
} dmi_kv8_bounds_t;

/*
 * Brings the bounds of every block that new tokens reach up to date (behind the append that wrote them), from all tokens that the block
 * has.  An element that is NaN in one of them has NaN bounds.  Behind dmi_kv8_evict: a call on the cache it filled, all of whose tokens
 * are new (starts and lengths say so).
 */
dmi_status_t dmi_kv8_bound(const dmi_kv8_t *cache /*[host]*/, const dmi_kv8_batch_t *batch /*[host]*/,
                           const dmi_kv8_bounds_t *bounds /*[host]*/, void *hip_stream);

/*
 * For every new token, at position p of its request, and every head of the cache: n_select of the blocks 0 .. p / block_size, or all of
 * them where there are no more.  The first n_first and the last n_recent ones (1 or more: a token's own among them) are taken, and of
 * the others those with the largest
 *     score = k_scale * max over the query heads that read the head of  sum_d max(q_d least_d, q_d largest_d),
 * which no token of the block exceeds with any of these queries (for a positive scale of the attention); equal scores: the lower block.
 * Scores are computed in 64 bits.  A score that is NaN, and a block whose entry lies outside the cache, count as -inf.
 *   q           BF16 or FP16
 *   blocks_dev  [device] int32 [total_new][n_heads][n_select]: logical blocks in ascending order, -1 behind the last (a token whose
 *               position lies below 0 has none).  Rows of tokens that no request has are left as they were.
 *   workspace   as in dmi_kv8_attend, dmi_kv8_select_workspace(...) bytes
 */
uint64_t dmi_kv8_select_workspace(const dmi_kv8_t *cache /*[host]*/, const dmi_kv8_batch_t *batch /*[host]*/, uint32_t n_select);
dmi_status_t dmi_kv8_select(const dmi_kv8_t *cache /*[host]*/, const dmi_kv8_batch_t *batch /*[host]*/,
                            const dmi_kv8_bounds_t *bounds /*[host]*/, const dmi_kv8_heads_t *q /*[host]*/, uint32_t n_q_heads,
                            uint32_t n_select, uint32_t n_first, uint32_t n_recent, int32_t *blocks_dev,
                            void *workspace, uint64_t workspace_bytes, void *hip_stream);

/*
 * As dmi_kv8_attend, every new token by itself, over those tokens that it sees and that lie in the blocks listed for it and the head.  Of
 * a row of blocks_dev as many entries are looked at as the token sees blocks; those below 0, and those behind the token's own block, stand for
 * nothing, and a block that is listed twice counts twice.
 *   blocks_dev  [device] int32 [total_new][n_heads][n_select], as dmi_kv8_select writes it
 *   n_q_heads   up to 32 query heads read a head of the cache, up to 16 of more than 128 elements
 */
uint64_t dmi_kv8_attend_blocks_workspace(const dmi_kv8_t *cache /*[host]*/, const dmi_kv8_batch_t *batch /*[host]*/,
                                         uint32_t n_q_heads, uint32_t n_select);
dmi_status_t dmi_kv8_attend_blocks(const dmi_kv8_t *cache /*[host]*/, const dmi_kv8_batch_t *batch /*[host]*/,
                                   const int32_t *blocks_dev, uint32_t n_select, const dmi_kv8_heads_t *q /*[host]*/,
                                   uint32_t n_q_heads, float scale, const dmi_kv8_heads_t *out /*[host]*/, float *lse_dev,
                                   void *workspace, uint64_t workspace_bytes, void *hip_stream);

/* Requests that share the beginning of their contexts: group g is requests group_starts[g] .. group_starts[g+1]-1 of a batch (ascending;
 * requests outside of all groups share nothing), whose first prefix[g] tokens are the same.
 * max_prefix is an upper bound of the prefixes: launches are sized by it, and a longer one counts as max_prefix. */
typedef struct {
    uint32_t n_groups, max_prefix;
    const int32_t *group_starts_dev;    /* [device] n_groups + 1 */
    const int32_t *prefix_dev;          /* [device] n_groups */
} dmi_kv8_prefix_t;

/*
 * dmi_kv8_attend (without weights) for such groups.  The whole blocks of a prefix that lie in front of the first request's new tokens are
 * read once for the group, through that request's row of the block table (the others' rows need not list them), by every request that has as
 * many tokens in front of its new ones.  All other tokens, and all tokens of a request that has not, are read through its own row.
 * (Where that takes less time, each request reads them by itself, through that row too.)
 */
uint64_t dmi_kv8_attend_shared_workspace(const dmi_kv8_t *cache /*[host]*/, const dmi_kv8_batch_t *batch /*[host]*/,
                                         const dmi_kv8_prefix_t *prefix /*[host]*/, uint32_t n_q_heads);
dmi_status_t dmi_kv8_attend_shared(const dmi_kv8_t *cache /*[host]*/, const dmi_kv8_batch_t *batch /*[host]*/,
                                   const dmi_kv8_prefix_t *prefix /*[host]*/, const dmi_kv8_heads_t *q /*[host]*/,
                                   uint32_t n_q_heads, float scale, const dmi_kv8_heads_t *out /*[host]*/, float *lse_dev,
                                   void *workspace, uint64_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* DMI_KV8_LONG_H */
