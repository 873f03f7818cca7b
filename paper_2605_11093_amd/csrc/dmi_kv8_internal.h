// Internals shared by the operators on the 8-bit KV cache (dmi_kv8.hip: checks and plans, dmi_kv8_*.hip: kernels).
#pragma once
#include "dmi_kv8.h"

#include <hip/hip_runtime.h>

namespace dmi {
namespace kv8 {

constexpr uint32_t kMaxLen = 1u << 24;          // tokens of a request
constexpr uint32_t kMaxBlock = 1024;            // tokens of a block
constexpr uint32_t kMaxDim = 256;
constexpr int64_t kMaxSlotStride = 1 << 26;     // sixteen tokens lie within 32-bit offsets of the first
constexpr uint32_t kMaxReqs = 65535;            // requests of a call: what a launch's second dimension holds

// A cache as the kernels see it; [0] is K, [1] is V.
struct Cache {
    uint8_t *code[2];
    float *scale[2];
    const int32_t *table;
    int64_t block_stride, slot_stride, head_stride, scale_block_stride, scale_head_stride, table_stride;
    uint32_t bs, heads, dim, n_blocks, n_seqs, max_blocks;
    uint32_t per_block;                         // 2^31 / (bs / 16), rounded up: see block_of
};

struct Batch {
    const int32_t *lens, *starts, *rows;
    uint32_t n_reqs, total_new, max_new, max_len;
};

struct Rows {
    void *data;
    int64_t row_stride, head_stride;
};

struct Weight {
    float *data;
    int64_t row_stride, head_stride;
};

struct AppendArgs {
    Cache c;
    Batch b;
    Rows x[2];
    uint32_t touched;                           // blocks that a request's new tokens may reach
    bool counted;                               // requests' new tokens differ much: see append_kernel
};

struct EvictArgs {
    Cache c, to;
    Batch b;
    Weight w, to_w;
    uint32_t keep, recent;
    int32_t *positions, *to_lens;
};

struct AttendArgs {
    Cache c;
    Batch b;
    Rows q, out;
    float *lse;
    Weight w, prior;                            // data NULL: none
    float decay, scale_log2;                    // scale * log2(e): scores are kept as powers of two
    uint32_t group, q_heads;
};

typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr uint32_t kFewRows = 32;               // query rows that share a head: up to here by tokens_kernel

// How few query rows are attended to: see dmi_kv8_tokens.hip.
struct TokensPlan {
    bool whole;                                 // a workgroup takes a request and head, or one of its equal splits: no ranges
    uint32_t splits;
    uint32_t ranges;                            // equal parts of all contexts
    uint32_t tile_rows, row_tiles;              // query rows of a wavefront; wavefronts for the rows that share a head
    uint32_t join_blocks;                       // workgroups of the second launch that join parts, 0 if there can be none
    uint32_t score_stride;
    f32x2 *sums;                                // of parts: maximum, sum of 2^(score - maximum)
    float *parts;                               // [part][dim]
    float *totals;                              // [row of out]: log2 of the sum of 2^score of contexts whole in a range; NULL: no weights
    float *scores;                              // [head][query row][score_stride]; NULL: no weights
};

// How many query rows are attended to: see dmi_kv8_parts.hip.
struct PartsPlan {
    uint32_t row_tiles;                         // workgroups for the rows that share a head
    bool counted;                               // requests' rows differ much: see parts_kernel
    uint32_t splits, chunk;                     // parts of the longest context, their tokens
    f32x2 *sums;                                // [row of out][split]: maximum, sum of 2^(score - maximum); one split: unused
    float *parts;                               // [row of out][split][dim]
    float *totals;                              // [row of out]: log2 of the sum of 2^score; NULL: no weights
};

// What a launch may have in its first dimension: threads are counted in 32 bits.  A call whose launches need more is refused before
// the first of them (hipErrorInvalidConfiguration).
inline bool launchable(uint64_t groups, uint32_t threads) { return groups <= 0xffffffffu / threads; }

hipError_t launch_append(AppendArgs a, uint32_t dtype, hipStream_t s);
hipError_t launch_evict(const EvictArgs &a, hipStream_t s);
hipError_t launch_parts(const AttendArgs &a, const PartsPlan &p, uint32_t dtype, hipStream_t s);
hipError_t launch_tokens(const AttendArgs &a, const TokensPlan &p, uint32_t dtype, hipStream_t s);

// ---------------------------------------------------------------- device side
#ifdef __HIPCC__
// One request of a batch: its row of the block table, its length, its new tokens' rows.
struct Request {
    int row, len, start, fresh;
};

__device__ __forceinline__ Request request_of(const Batch &b, const Cache &c, int r)
{
    Request q;
    q.row = b.rows ? b.rows[r] : r;
    q.len = min(max(b.lens[r], 0), (int)b.max_len);
    if ((uint32_t)q.row >= c.n_seqs) q.row = 0, q.len = 0;
    if (b.starts) {
        q.start = min(max(b.starts[r], 0), (int)b.total_new);
        q.fresh = min(max(b.starts[r + 1] - q.start, 0), min((int)b.max_new, (int)b.total_new - q.start));
    } else {
        q.start = r;
        q.fresh = 1;
    }
    return q;
}

// Sums over the lanes up to each one
__device__ __forceinline__ int lanes_scan(int v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);     // within 16 lanes: shifts by 1, 2, 4, 8
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);     // the totals of 16 lanes carried on
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);
    return v;
}

// A request that a lane has
__device__ __forceinline__ Request request_in(const Request &q, int lane)
{
    return {__builtin_amdgcn_readlane(q.row, lane), __builtin_amdgcn_readlane(q.len, lane), __builtin_amdgcn_readlane(q.start, lane),
            __builtin_amdgcn_readlane(q.fresh, lane)};
}

// Logical block of the 16 tokens from 16 * sixteen on.  bs / 16 is at most 64 and sixteen below 2^20: with the reciprocal
// rounded up the error of the product stays below 2^31 / (bs / 16).
__device__ __forceinline__ uint32_t block_of(const Cache &c, uint32_t sixteen)
{
    return (uint32_t)(((uint64_t)sixteen * c.per_block) >> 31);
}
// Physical block of a logical one, -1 if the table has none in the cache there.
__device__ __forceinline__ int entry_of(const Cache &c, int row, uint32_t block)
{
    if (block >= c.max_blocks) return -1;
    const int e = c.table[(int64_t)row * c.table_stride + block];
    return (uint32_t)e < c.n_blocks ? e : -1;
}
__device__ __forceinline__ uint8_t *code_at(const Cache &c, int kv, int block, uint32_t slot, uint32_t head)
{
    return c.code[kv] + (int64_t)block * c.block_stride + (int64_t)slot * c.slot_stride + (int64_t)head * c.head_stride;
}
__device__ __forceinline__ float *scale_at(const Cache &c, int kv, int block, uint32_t head)
{
    return c.scale[kv] + (int64_t)block * c.scale_block_stride + (int64_t)head * c.scale_head_stride;
}

// Four values to e4m3 codes: nearest, ties to even; beyond +-448 the largest number, NaN stays NaN.
__device__ __forceinline__ float within(float x)
{
    return x > 448.0f ? 448.0f : x < -448.0f ? -448.0f : x;
}
__device__ __forceinline__ uint32_t to_codes(float a, float b, float c, float d)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(within(a), within(b), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(within(c), within(d), w, true);
}
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Codes in a word times a factor, as codes again.
__device__ __forceinline__ uint32_t scaled_codes(uint32_t w, float f)
{
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    return to_codes(a[0] * f, a[1] * f, b[0] * f, b[1] * f);
}
#endif

}  // namespace kv8
}  // namespace dmi
