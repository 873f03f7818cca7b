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

typedef float f32x2 __attribute__((ext_vector_type(2)));

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

struct RotateArgs {
    Cache c;
    Batch b;
    Rows x[2], q, q_out;
    const float *freq;
    const int32_t *positions;                   // NULL: a token's place
    uint32_t rotary, q_heads;                   // q_heads 0: no queries
    bool neighbours;                            // what makes a pair: see dmi_kv8_rotary_t
    bool counted;                               // as in AppendArgs
    uint32_t tokens;                            // whose cosines are in LDS at a time
    uint32_t each, groups;                      // items of a workgroup, workgroups of a block
    uint32_t q_each, q_part;                    // tokens whose queries an item has; 2^32 / q_heads, rounded up
};

struct BoundArgs {
    Cache c;
    Batch b;
    uint8_t *bounds;
    int64_t bounds_block_stride, bounds_head_stride;
    uint32_t touched;
    bool counted;
};

struct SelectArgs {
    Cache c;
    Batch b;
    Rows q;
    const uint8_t *bounds;
    int64_t bounds_block_stride, bounds_head_stride;
    uint32_t group, n_select, n_first, n_recent;
    uint32_t stride;                            // blocks of the longest request
    f32x2 *scores;                              // [new token][head][stride]: a score, how far it may be off; one launch: unused
    uint64_t *keys;                             // the same places: scores in 64 bits, as unsigned numbers in their order
    int32_t *blocks;
    uint32_t several;                           // tokens that a pass over the bounds is for
};

struct AttendArgs {
    Cache c;
    Batch b;
    Rows q, out;
    float *lse;
    Weight w, prior;                            // data NULL: none
    float decay, scale_log2;                    // scale * log2(e): scores are kept as powers of two
    uint32_t group, q_heads;
    const int32_t *blocks;                      // kListed: those attended to, [new token][head][n_select]
    uint32_t n_select;
    uint32_t n_groups, max_prefix;              // kPrefix, kLast, kRest, kThrough: see dmi_kv8_prefix_t
    const int32_t *group_starts, *prefix;
};

// What the attention kernels do: a whole context; the rest of one behind a shared prefix, whose sums are left as parts whatever their
// number; such a prefix, for all rows of a group of requests, whose sums are left as parts, or which goes on from the rests' sums to outputs;
// listed blocks, for each new token by itself; a whole context whose prefix is read through its group's first request's row.
enum Kind { kWhole, kRest, kPrefix, kLast, kListed, kThrough };

constexpr uint32_t kFewRows = 32;               // query rows that share a head: up to here by tokens_kernel

// What a prefix has left: of every row of out, splits parts, those behind a row's prefix not written where `chunk` tokens make one.
struct PrefixParts {
    uint32_t splits, chunk;                     // chunk 0: all are there
    const f32x2 *sums;                          // [row of out][split]
    const float *parts;                         // [row of out][split][dim]
};

// How few query rows are attended to: see dmi_kv8_tokens.hip.
struct TokensPlan {
    bool whole;                                 // a workgroup takes a request and head, or one of its equal splits: no ranges
    uint32_t splits;
    uint32_t ranges;                            // equal parts of all contexts
    uint32_t waves;                             // of a workgroup, not kWhole: 4 or 8, kListed and kRest also 1
    bool through;                               // kRest: prefixes too, through the first request's row
    bool by_xcd;                                // kPrefix: what reads the same codes on one XCD
    uint32_t tile_rows, row_tiles;              // query rows of a wavefront; wavefronts for the rows that share a head
    uint32_t join_blocks;                       // workgroups of the second launch that join parts, 0 if there can be none
    uint32_t score_stride;
    f32x2 *sums;                                // of parts: maximum, sum of 2^(score - maximum)
    float *parts;                               // [part][dim]
    float *totals;                              // [row of out]: log2 of the sum of 2^score of contexts whole in a range; NULL: no weights
    float *scores;                              // [head][query row][score_stride]; NULL: no weights
    bool before;                                // kRest, one split: joined with the parts of prefixes, to outputs
    PrefixParts prefix;
};

// How many query rows are attended to: see dmi_kv8_parts.hip.
struct PartsPlan {
    uint32_t row_tiles;                         // workgroups for the rows that share a head
    bool counted;                               // requests' rows differ much: see parts_kernel
    bool spread;                                // not kWhole, and counted: row tiles go to the XCDs in turn
    uint32_t splits, chunk;                     // parts of the longest context, their tokens
    f32x2 *sums;                                // [row of out][split]: maximum, sum of 2^(score - maximum); one split: unused
    float *parts;                               // [row of out][split][dim]
    float *totals;                              // [row of out]: log2 of the sum of 2^score; NULL: no weights
};

// How contexts behind shared prefixes are attended to: see dmi_kv8_parts.hip.
struct SharedPlan {
    PartsPlan prefix;                           // splits 0: there is none
    bool few_rows;                              // few rows for it: by tokens_kernel, whose splits are all there
    TokensPlan prefix_few;
    bool through;                               // not read once: each request reads it, in one launch
    bool last;                                  // the prefix goes on from the rests' sums: nothing is split
    bool tokens;                                // few rows a head behind it: by tokens_kernel
    TokensPlan few;
    PartsPlan many;
    uint32_t splits;                            // of what is behind the prefix
    f32x2 *sums;                                // [row of out][split]
    float *parts;
};

// Whether a selection, of `items` new tokens and heads over up to `blocks` blocks each, takes one launch, with scores in LDS: where a
// workgroup goes through a head's blocks in the time that a second launch takes, or there are workgroups enough; scores over more workgroups, and
// in memory, otherwise.  Measured (us, one launch / two; tokens x heads, blocks): 8, 500 15 / 19, 128, 500 15 / 20, 8, 2000 27 / 20, 128, 2000 29 / 31,
// 256, 2000 34 / 47, 512, 2000 73 / 95, 8, 7000 72 / 23, 128, 7000 98 / 81.
constexpr uint32_t kMostInLds = 8192;           // blocks whose scores a workgroup keeps
inline bool selects_in_one(uint64_t items, uint32_t blocks) { return blocks <= kMostInLds && (blocks <= 1024u || items >= blocks / 16u); }

// What a launch may have in its first dimension: threads are counted in 32 bits.  A call whose launches need more is refused before
// the first of them (hipErrorInvalidConfiguration).
inline bool launchable(uint64_t groups, uint32_t threads) { return groups <= 0xffffffffu / threads; }

hipError_t launch_append(AppendArgs a, uint32_t dtype, hipStream_t s);
hipError_t launch_rotate(RotateArgs a, uint32_t dtype, hipStream_t s);
hipError_t launch_bound(BoundArgs a, hipStream_t s);
hipError_t launch_select(const SelectArgs &a, uint32_t dtype, hipStream_t s);
hipError_t launch_evict(const EvictArgs &a, hipStream_t s);
hipError_t launch_parts(const AttendArgs &a, const PartsPlan &p, uint32_t dtype, hipStream_t s);
hipError_t launch_parts_apart(const AttendArgs &a, const PartsPlan &p, Kind kind, uint32_t dtype, hipStream_t s);
bool tokens_apart_fit(const AttendArgs &a, const TokensPlan &p, Kind kind);        // whether a launch has workgroups enough
hipError_t launch_shared(const AttendArgs &a, const SharedPlan &p, uint32_t dtype, hipStream_t s);
hipError_t launch_tokens_apart(const AttendArgs &a, const TokensPlan &p, Kind kind, uint32_t dtype, hipStream_t s);
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

// The last request whose rows begin at a token or in front of it.  64 places at a time are looked at, so 65535 requests take three trips to
// memory.
__device__ __forceinline__ Request request_with(const Batch &b, const Cache &c, int token)
{
    int r = token;
    if (b.starts) {
        int n = (int)b.n_reqs;
        r = 0;
        while (n > 1) {
            const int step = (n + 63) >> 6, at = (int)(threadIdx.x & 63u) * step;
            const int k = max(1, __popcll(__ballot(at < n && b.starts[r + min(at, n - 1)] <= token)));
            r += (k - 1) * step;
            n = min(step, n - (k - 1) * step);
        }
    }
    return request_of(b, c, min(r, (int)b.n_reqs - 1));
}
// A new token as a request of its own, with a length of what it sees, if it is one of that request's
__device__ __forceinline__ Request token_of(const Batch &b, const Cache &c, int token)
{
    const Request q = request_with(b, c, token);
    const int nth = token - q.start;
    return {q.row, min(q.len, max(0, q.len - q.fresh + nth + 1)), token, nth >= 0 && nth < q.fresh ? 1 : 0};
}

// Groups of requests that share the beginning of their contexts.  What a group shares hangs on its first request alone, and whether
// another request takes part on that request alone, so that nothing has to be counted before a launch.
// A group as a request: the rows of all its requests' new tokens; `row` is its first request here.
__device__ __forceinline__ Request group_rows(const AttendArgs &a, int g)
{
    const int n = (int)a.b.n_reqs, first = min(max(a.group_starts[g], 0), n), last = min(max(a.group_starts[g + 1], first), n);
    const int start = a.b.starts ? min(max(a.b.starts[first], 0), (int)a.b.total_new) : first;
    const int end = a.b.starts ? min(max(a.b.starts[last], start), (int)a.b.total_new) : last;
    return {first, 0, start, first < last ? end - start : 0};
}
// Tokens that are read once for the group of requests `start` to `end`: whole blocks of its prefix, in front of its first request's new tokens.
// `row`: that one's in the table.
__device__ __forceinline__ int tokens_of(const AttendArgs &a, int start, int end, int prefix, int &row)
{
    const int first = min(max(start, 0), (int)a.b.n_reqs);
    row = 0;
    if (first >= min(end, (int)a.b.n_reqs)) return 0;
    const Request q = request_of(a.b, a.c, first);
    row = q.row;
    const int tokens = min(min(max(prefix, 0), (int)a.max_prefix), max(q.len - q.fresh, 0));
    return (int)(((uint32_t)(((uint64_t)((uint32_t)tokens >> 4) * a.c.per_block) >> 31)) * a.c.bs);
}
__device__ __forceinline__ int group_tokens(const AttendArgs &a, int g, int &row)
{
    return tokens_of(a, a.group_starts[g], a.group_starts[g + 1], a.prefix[g], row);
}
// How many of them a request takes: all, where it has as many in front of its new tokens, or none.  All lanes of a wavefront look for its
// group, the last one that begins at or in front of it, 64 places at a time; up to 64 groups in one trip to memory.
__device__ __forceinline__ int shared_tokens(const AttendArgs &a, int r, const Request &q, int &row)
{
    int n = (int)a.n_groups, start, end, prefix;
    if (!n) return 0;
    const int lane = (int)(threadIdx.x & 63u);
    if (n <= 64) {
        const int i = min(lane, n - 1), from = a.group_starts[i], to = a.group_starts[i + 1], tokens = a.prefix[i];
        const int g = max(1, __popcll(__ballot(lane < n && from <= r))) - 1;
        start = __builtin_amdgcn_readlane(from, g), end = __builtin_amdgcn_readlane(to, g), prefix = __builtin_amdgcn_readlane(tokens, g);
    } else {
        int g = 0;
        while (n > 1) {
            const int step = (n + 63) >> 6, at = lane * step;
            const int k = max(1, __popcll(__ballot(at < n && a.group_starts[g + min(at, n - 1)] <= r)));
            g += (k - 1) * step;
            n = min(step, n - (k - 1) * step);
        }
        start = a.group_starts[g], end = a.group_starts[g + 1], prefix = a.prefix[g];
    }
    if (r < start || r >= end) return 0;
    const int tokens = tokens_of(a, start, end, prefix, row);
    return q.len - q.fresh >= tokens ? tokens : 0;
}
__device__ __forceinline__ int shared_tokens(const AttendArgs &a, int r, const Request &q)
{
    int row;
    return shared_tokens(a, r, q, row);
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
