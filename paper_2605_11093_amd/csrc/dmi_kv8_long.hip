// The C entry points of the operators for long contexts on the 8-bit KV cache: arguments checked, kernels' arguments made.
#include "dmi_kv8_long.h"
#include "dmi_kv8_checks.h"

using namespace dmi;
using namespace dmi::host;
using namespace dmi::kv8;

namespace {

bool same(const Rows &x, const Rows &y) { return x.data == y.data && x.row_stride == y.row_stride && x.head_stride == y.head_stride; }

dmi_status_t check_bounds(const dmi_kv8_bounds_t *k)
{
    if (!k || !k->data) return fail(DMI_ERR_INVALID_ARG, "bounds are NULL");
    if ((uintptr_t)k->data % 16u || !whole(k->block_stride, 1) || !whole(k->head_stride, 1))
        return fail(DMI_ERR_INVALID_ARG, "bounds must be 16-byte aligned with strides that are multiples of 16");
    return DMI_OK;
}

// Arguments that all kinds of attention have
dmi_status_t check_attention(const dmi_kv8_t *cache, const dmi_kv8_batch_t *batch, const dmi_kv8_heads_t *q, uint32_t n_q_heads, float scale,
                             const dmi_kv8_heads_t *out, float *lse_dev, AttendArgs &a)
{
    dmi_status_t st;
    if ((st = check_cache(cache, "cache", a.c)) != DMI_OK || (st = check_batch(batch, a.c, true, a.b)) != DMI_OK ||
        (st = check_rows(q, "q", a.b, a.q)) != DMI_OK || (st = check_rows(out, "out", a.b, a.out)) != DMI_OK ||
        (st = check_attend(n_q_heads, a.c.heads, *batch)) != DMI_OK)
        return st;
    if (q->dtype != out->dtype || (q->dtype != DMI_DTYPE_BF16 && q->dtype != DMI_DTYPE_FP16))
        return fail(DMI_ERR_INVALID_ARG, "q and out must both be BF16 or both FP16");
    if (!std::isfinite(scale)) return fail(DMI_ERR_INVALID_ARG, "scale is not finite");
    if ((uintptr_t)lse_dev % 4u) return fail(DMI_ERR_INVALID_ARG, "lse_dev must be 4-byte aligned");
    if (!same(a.q, a.out) && share(a.q, n_q_heads, a.out, n_q_heads, a.b.total_new, a.c.dim, 2u))
        return fail(DMI_ERR_INVALID_ARG, "out and q share elements and are not the same");
    a.lse = lse_dev;
    a.scale_log2 = scale * 1.44269504088896340736f;
    a.group = n_q_heads / a.c.heads;
    a.q_heads = n_q_heads;
    return DMI_OK;
}

// Query rows of a head that tokens_kernel takes in one tile: two tiles of 256 elements take more registers than there are.
uint32_t most_rows(uint32_t dim) { return dim > 128u ? 16u : kFewRows; }

// Splits of `tokens` for `units` pairs of request and head, by dmi_kv8_attend's rule: of 512 tokens while there are compute units for
// them, of 1024 (2048 for many rows) in any case.  None where a workgroup goes through them all in the time that a second launch takes to join
// parts.  Measured over listed blocks (us, one / split): 4 pairs x 2048 tokens x 64 elements 13.7 / 18.9, 96 of them 17.3 / 19.6, 128 17.6 /
// 22.6, 16 x 1536 x 128 15.4 / 18.8; 8 x 2048 x 128 17.8 / 19.1, 64 of them 23.3 / 19.5, 16 x 1536 x 256 23.4 / 19.0.
uint32_t splits_of(uint64_t units, uint64_t tokens, uint32_t rows, uint32_t dim)
{
    const uint64_t reach = rows > 16u ? 2048u : 1024u;
    uint64_t s = 1;
    if (rows <= 16u && tokens * dim <= 3u << 16) return 1u;
    if (tokens > 1024u) s = std::max<uint64_t>(1u, std::min(256u / std::max<uint64_t>(units, 1u), (tokens + 511u) / 512u));
    if (tokens > reach * s) s = (tokens + reach - 1u) / reach;
    return (uint32_t)std::min<uint64_t>(s, 64u);
}

// Wavefronts of a workgroup, `pairs` requests (or tokens) and heads: four where there is a workgroup for every compute unit so, eight where not (us,
// four / eight: listed blocks of 128 tokens x 8 heads 59 / 71, rests of 64 requests x 8 heads 24 / 28).  The heads of a request one behind the
// other on one XCD took 57.8 and 56.0 us where these calls take 56.7 and 53.8.
uint32_t waves_of(uint64_t pairs, uint32_t splits) { return pairs * splits > 256u ? 4u : 8u; }

// Whether many lists, or contexts and heads, have a wavefront each: where rounds of one on each of 1024 SIMDs end sooner so than of four, the start of
// one counted as six of its tiles of 32 tokens.  Measured (us, four wavefronts / one): lists x their tokens, heads of 128, one token a request, 1024 x 256
// 22.3 / 18.2, x 1024 56.7 / 49.7, x 4096 237 / 231, 768 x 512 25.8 / 25.0, x 1536 61.7 / 66.7; many tokens a request 13176 x 320 213 / 177, 2048 x 1536
// 108 / 103, of 256 elements 2048 x 512 110 / 80, of 64 one request's 160 tokens x 16 heads with all it has 86 / 105.  (Two took 55, 184 and 90 where one
// takes 50, 177 and 80.)  The whole call behind prefixes of 2000: 1000 requests x 8 heads of up to 100 tokens 160 / 116, 256 x 8 of 200 63 / 52, of 1000
// 115 / 113, 128 x 8 of 1000 67.6 / 68.7.
bool alone(uint64_t pairs, uint64_t tokens)
{
    const uint64_t tiles = (tokens + 31u) / 32u;
    auto cost = [&](uint64_t waves) { return (pairs * waves + 1023u) / 1024u * (6u + (tiles + waves - 1u) / waves); };
    return cost(1u) < cost(4u);
}

}  // namespace

extern "C" dmi_status_t dmi_kv8_append_rotated(const dmi_kv8_t *cache, const dmi_kv8_batch_t *batch, const dmi_kv8_heads_t *key,
                                               const dmi_kv8_heads_t *value, const dmi_kv8_rotary_t *rotary, const dmi_kv8_heads_t *q,
                                               uint32_t n_q_heads, const dmi_kv8_heads_t *q_out, void *hip_stream)
{
    RotateArgs a{};
    dmi_status_t st;
    if ((st = check_cache(cache, "cache", a.c)) != DMI_OK || (st = check_batch(batch, a.c, true, a.b)) != DMI_OK ||
        (st = check_rows(key, "key", a.b, a.x[0])) != DMI_OK || (st = check_rows(value, "value", a.b, a.x[1])) != DMI_OK)
        return st;
    if (key->dtype != value->dtype) return fail(DMI_ERR_INVALID_ARG, "key and value have different dtypes");
    if (!rotary || !rotary->freq_dev) return fail(DMI_ERR_INVALID_ARG, "rotary or its freq_dev is NULL");
    if (((uintptr_t)rotary->freq_dev | (uintptr_t)rotary->positions_dev) % 4u)
        return fail(DMI_ERR_INVALID_ARG, "freq_dev and positions_dev must be 4-byte aligned");
    if (!rotary->rotary_dim || rotary->rotary_dim % 16u || rotary->rotary_dim > a.c.dim)
        return fail(DMI_ERR_INVALID_ARG, "rotary_dim %u is not a multiple of 16 up to head_dim %u", rotary->rotary_dim, a.c.dim);
    if (rotary->pairs > 1u) return fail(DMI_ERR_INVALID_ARG, "pairs %u is neither 0 nor 1", rotary->pairs);
    if (!q != !q_out) return fail(DMI_ERR_INVALID_ARG, "q and q_out go together");
    if (q) {
        if ((st = check_rows(q, "q", a.b, a.q)) != DMI_OK || (st = check_rows(q_out, "q_out", a.b, a.q_out)) != DMI_OK) return st;
        if (q->dtype != key->dtype || q_out->dtype != key->dtype) return fail(DMI_ERR_INVALID_ARG, "q, q_out and key have different dtypes");
        if (!n_q_heads || n_q_heads > 65536u || (uint64_t)a.b.total_new * n_q_heads > kMostRows)
            return fail(DMI_ERR_INVALID_ARG, "n_q_heads %u is not in 1..65536, or their rows are more than 2^30", n_q_heads);
        const uint32_t size = dtype_size(key->dtype), n = a.b.total_new;
        if (!same(a.q, a.q_out) && share(a.q, n_q_heads, a.q_out, n_q_heads, n, a.c.dim, size))
            return fail(DMI_ERR_INVALID_ARG, "q_out and q share elements and are not the same");
        if (share(a.q_out, n_q_heads, a.x[0], a.c.heads, n, a.c.dim, size) || share(a.q_out, n_q_heads, a.x[1], a.c.heads, n, a.c.dim, size))
            return fail(DMI_ERR_INVALID_ARG, "q_out shares elements with key or value");
        a.q_heads = n_q_heads;
    }
    if (!a.b.n_reqs || !a.b.total_new || !a.b.max_new || !a.b.max_len) return DMI_OK;
    a.freq = rotary->freq_dev;
    a.positions = rotary->positions_dev;
    a.rotary = rotary->rotary_dim;
    a.neighbours = rotary->pairs != 0u;
    return launched(launch_rotate(a, key->dtype, (hipStream_t)hip_stream));
}

extern "C" dmi_status_t dmi_kv8_bound(const dmi_kv8_t *cache, const dmi_kv8_batch_t *batch, const dmi_kv8_bounds_t *bounds, void *hip_stream)
{
    BoundArgs a{};
    dmi_status_t st;
    if ((st = check_cache(cache, "cache", a.c)) != DMI_OK || (st = check_batch(batch, a.c, true, a.b)) != DMI_OK ||
        (st = check_bounds(bounds)) != DMI_OK)
        return st;
    if (!a.b.n_reqs || !a.b.total_new || !a.b.max_new || !a.b.max_len) return DMI_OK;
    a.bounds = bounds->data;
    a.bounds_block_stride = bounds->block_stride;
    a.bounds_head_stride = bounds->head_stride;
    return launched(launch_bound(a, (hipStream_t)hip_stream));
}

namespace {

// Scores of every new token and head, for each block that the longest request has; none where every block is taken
constexpr uint64_t kMostScores = 1ull << 40;

uint32_t score_stride(const dmi_kv8_t &cache, const dmi_kv8_batch_t &b) { return (b.max_len + cache.block_size - 1u) / cache.block_size; }

dmi_status_t check_select(const dmi_kv8_t &cache, const dmi_kv8_batch_t &b, uint32_t n_select)
{
    if (!n_select || n_select > kMaxLen) return fail(DMI_ERR_INVALID_ARG, "n_select %u is not in 1..%u", n_select, kMaxLen);
    if ((uint64_t)b.total_new * cache.n_heads * n_select > kMostScores ||
        (uint64_t)b.total_new * cache.n_heads * std::max(1u, score_stride(cache, b)) > kMostScores)
        return fail(DMI_ERR_INVALID_ARG, "more than 2^40 scores or listed blocks");
    return DMI_OK;
}

// (scores first, of two launches; then the words that they are ranked by)
struct SelectBytes {
    uint64_t scores, all;
};
SelectBytes select_bytes(const dmi_kv8_t &cache, const dmi_kv8_batch_t &b, uint32_t n_select)
{
    const uint32_t stride = score_stride(cache, b);
    const uint64_t items = (uint64_t)b.total_new * cache.n_heads, each = stride > n_select ? pad64(items * stride * 8u) : 0u;
    const uint64_t scores = selects_in_one(items, stride) ? 0u : each;
    return {scores, scores + each};
}

}  // namespace

extern "C" uint64_t dmi_kv8_select_workspace(const dmi_kv8_t *cache, const dmi_kv8_batch_t *batch, uint32_t n_select)
{
    if (!cache || !batch || check_shape(cache, "cache") != DMI_OK || check_counts(batch, true) != DMI_OK ||
        check_select(*cache, *batch, n_select) != DMI_OK)
        return 0;
    return select_bytes(*cache, *batch, n_select).all;
}

extern "C" dmi_status_t dmi_kv8_select(const dmi_kv8_t *cache, const dmi_kv8_batch_t *batch, const dmi_kv8_bounds_t *bounds,
                                       const dmi_kv8_heads_t *q, uint32_t n_q_heads, uint32_t n_select, uint32_t n_first, uint32_t n_recent,
                                       int32_t *blocks_dev, void *workspace, uint64_t workspace_bytes, void *hip_stream)
{
    SelectArgs a{};
    dmi_status_t st;
    if ((st = check_cache(cache, "cache", a.c)) != DMI_OK || (st = check_batch(batch, a.c, true, a.b)) != DMI_OK ||
        (st = check_bounds(bounds)) != DMI_OK || (st = check_rows(q, "q", a.b, a.q)) != DMI_OK ||
        (st = check_attend(n_q_heads, a.c.heads, *batch)) != DMI_OK || (st = check_select(*cache, *batch, n_select)) != DMI_OK)
        return st;
    if (q->dtype != DMI_DTYPE_BF16 && q->dtype != DMI_DTYPE_FP16) return fail(DMI_ERR_INVALID_ARG, "q must be BF16 or FP16");
    if (!n_recent || n_first > n_select || n_recent > n_select - n_first)
        return fail(DMI_ERR_INVALID_ARG, "n_recent %u must be positive, and n_first %u and it no more than n_select %u", n_recent, n_first, n_select);
    if ((!blocks_dev && a.b.total_new) || (uintptr_t)blocks_dev % 4u) return fail(DMI_ERR_INVALID_ARG, "blocks_dev is NULL or not 4-byte aligned");
    const SelectBytes bytes = select_bytes(*cache, *batch, n_select);
    if ((st = check_workspace(bytes.all, workspace, workspace_bytes)) != DMI_OK) return st;
    if (!a.b.n_reqs || !a.b.total_new || !a.b.max_new) return DMI_OK;
    a.bounds = bounds->data;
    a.bounds_block_stride = bounds->block_stride;
    a.bounds_head_stride = bounds->head_stride;
    a.group = n_q_heads / a.c.heads;
    a.n_select = n_select, a.n_first = n_first, a.n_recent = n_recent;
    a.stride = score_stride(*cache, *batch);
    a.scores = static_cast<f32x2 *>(workspace);
    a.keys = reinterpret_cast<uint64_t *>(static_cast<char *>(workspace) + bytes.scores);
    a.blocks = blocks_dev;
    return launched(launch_select(a, q->dtype, (hipStream_t)hip_stream));
}

namespace {

struct BlocksPlan {
    TokensPlan t;
    uint64_t parts, bytes;                      // (sums come first)
};
BlocksPlan plan_blocks(uint32_t heads, uint32_t dim, uint32_t block_size, const dmi_kv8_batch_t &b, uint32_t q_heads, uint32_t n_select)
{
    BlocksPlan p{};
    TokensPlan &t = p.t;
    const uint32_t group = q_heads / heads;
    const uint64_t blocks = std::min<uint64_t>(n_select, (b.max_len + block_size - 1u) / block_size);
    t.whole = true;
    t.tile_rows = group <= 16u ? 16u : 32u;
    t.row_tiles = 1u;
    // (the launch that joins parts has a token in each of its rows)
    t.splits = b.total_new > 65535u ? 1u : splits_of((uint64_t)b.total_new * heads, blocks * block_size, group, dim);
    t.waves = waves_of((uint64_t)b.total_new * heads, t.splits);
    if ((uint64_t)b.total_new * heads * t.splits >= 768u && alone((uint64_t)b.total_new * heads * t.splits, blocks * block_size / t.splits)) t.waves = 1u;
    t.join_blocks = t.splits > 1u ? (q_heads + 3u) / 4u : 0u;
    const uint64_t parts = t.splits > 1u ? (uint64_t)b.total_new * q_heads * t.splits : 0u;
    p.parts = pad64(parts * 8u);
    p.bytes = p.parts + pad64(parts * dim * 4u);
    return p;
}

dmi_status_t check_list(uint32_t n_q_heads, uint32_t heads, uint32_t dim, uint32_t n_select)
{
    if (n_q_heads / heads > most_rows(dim))
        return fail(DMI_ERR_INVALID_ARG, "%u query heads of %u elements read one head of the cache: more than %u", n_q_heads / heads, dim, most_rows(dim));
    if (!n_select || n_select > kMaxLen) return fail(DMI_ERR_INVALID_ARG, "n_select %u is not in 1..%u", n_select, kMaxLen);
    return DMI_OK;
}

}  // namespace

extern "C" uint64_t dmi_kv8_attend_blocks_workspace(const dmi_kv8_t *cache, const dmi_kv8_batch_t *batch, uint32_t n_q_heads, uint32_t n_select)
{
    if (!cache || !batch || check_shape(cache, "cache") != DMI_OK || check_counts(batch, true) != DMI_OK ||
        check_attend(n_q_heads, cache->n_heads, *batch) != DMI_OK || check_list(n_q_heads, cache->n_heads, cache->head_dim, n_select) != DMI_OK)
        return 0;
    return plan_blocks(cache->n_heads, cache->head_dim, cache->block_size, *batch, n_q_heads, n_select).bytes;
}

extern "C" dmi_status_t dmi_kv8_attend_blocks(const dmi_kv8_t *cache, const dmi_kv8_batch_t *batch, const int32_t *blocks_dev,
                                              uint32_t n_select, const dmi_kv8_heads_t *q, uint32_t n_q_heads, float scale,
                                              const dmi_kv8_heads_t *out, float *lse_dev, void *workspace, uint64_t workspace_bytes,
                                              void *hip_stream)
{
    AttendArgs a{};
    dmi_status_t st;
    if ((st = check_attention(cache, batch, q, n_q_heads, scale, out, lse_dev, a)) != DMI_OK ||
        (st = check_list(n_q_heads, a.c.heads, a.c.dim, n_select)) != DMI_OK)
        return st;
    if ((!blocks_dev && a.b.total_new) || (uintptr_t)blocks_dev % 4u) return fail(DMI_ERR_INVALID_ARG, "blocks_dev is NULL or not 4-byte aligned");
    const BlocksPlan plan = plan_blocks(a.c.heads, a.c.dim, a.c.bs, *batch, n_q_heads, n_select);
    if ((st = check_workspace(plan.bytes, workspace, workspace_bytes)) != DMI_OK) return st;
    if (!a.b.n_reqs || !a.b.total_new || !a.b.max_new) return DMI_OK;
    a.blocks = blocks_dev;
    a.n_select = n_select;
    TokensPlan t = plan.t;
    t.sums = static_cast<f32x2 *>(workspace);
    t.parts = reinterpret_cast<float *>(static_cast<char *>(workspace) + plan.parts);
    return launched(launch_tokens_apart(a, t, kListed, q->dtype, (hipStream_t)hip_stream));
}

namespace {

struct SharedSizes {
    SharedPlan p;
    uint64_t prefix_parts, sums, parts, bytes;  // (the prefixes' sums come first)
};
SharedSizes plan_shared(uint32_t heads, uint32_t dim, uint32_t block_size, const dmi_kv8_batch_t &b, const dmi_kv8_prefix_t &x, uint32_t q_heads)
{
    SharedSizes z{};
    SharedPlan &p = z.p;
    const uint32_t group = q_heads / heads, rows_each = dim <= 128u ? 256u : 128u, max_new = std::min(b.max_new, b.total_new);
    const uint64_t rows = (uint64_t)b.total_new * q_heads, shared = (uint64_t)max_new * group;
    const uint32_t prefix = std::min(x.max_prefix, b.max_len) / block_size * block_size;
    double once = INFINITY;                     // us that prefixes read once take
    if (x.n_groups && prefix) {
        const uint64_t all = (uint64_t)b.total_new * group;
        auto tiles_of = [&](uint32_t rows) { return std::max<uint64_t>(x.n_groups, (all + (uint64_t)x.n_groups * rows / 2u) / rows); };
        TokensPlan &t = p.prefix_few;
        t.tile_rows = all <= 16u || dim > 128u ? 16u : 32u;
        t.row_tiles = (uint32_t)((all + t.tile_rows - 1u) / t.tile_rows);
        const uint64_t few = tiles_of(t.tile_rows) * heads;
        // Few rows by tokens_kernel, many by parts_kernel.  Measured (us, the whole call, tokens / parts; 300 tokens behind the prefix; 8 heads x
        // 128, or 4 x 64 or 256): one prefix of 8000 tokens with 32 rows a head 32.6 / 33.8, with 64 33.5 / 35.4, with 128 37.4 / 38.7, with 256
        // 47.4 / 46.6, of 30000 tokens with 64 45 / 49, with 128 61 / 54; four of 2000 with 32 in all 40 / 35; 64 elements, 8000 tokens, with 128
        // 27 / 39, with 256 29 / 43; 256 elements with 64 37 / 61, with 128 40 / 52.
        p.few_rows = few <= 256u && (uint64_t)t.row_tiles * x.n_groups <= 8u * tiles_of(t.tile_rows) &&
                     (dim <= 64u || dim > 128u || (x.n_groups == 1u && all <= 64u));
        if (p.few_rows) {
            // four wavefronts with 256 tokens at least, on every compute unit
            t.whole = true;
            t.waves = 4u;
            t.by_xcd = x.n_groups * heads >= 8u;
            t.splits = p.prefix.splits = (uint32_t)std::max<uint64_t>(1u, std::min<uint64_t>(256u / few, prefix / 256u));
            once = 8.0 + 1.5 * ((prefix / 32u + t.splits * 4u - 1u) / (t.splits * 4u));
        } else {
            PartsPlan &m = p.prefix;
            m.row_tiles = (uint32_t)((all + rows_each - 1u) / rows_each);
            // As many splits as make the sum of two least: rounds of 256 workgroups, with three tiles of 64 tokens for each one's start and
            // end, 2.5 us a tile; and a part of every row written and read again, at 4 TB/s.
            const uint64_t groups = tiles_of(rows_each) * heads, tiles = (prefix + 63u) / 64u;
            for (uint32_t s = 1; s <= 64u && (s == 1u || s * 128u <= prefix); s++) {
                const double cost = (double)((groups * s + 255u) / 256u) * (double)((tiles + s - 1u) / s + 3u) * 2.5 + (double)rows * s * dim * 8.0 / 4e6;
                if (cost < once) once = cost, m.splits = s;
            }
            m.chunk = std::max(64u, ((prefix + m.splits - 1u) / m.splits + 63u) & ~63u);
            m.splits = (prefix + m.chunk - 1u) / m.chunk;
        }
    }
    p.tokens = shared <= most_rows(dim);
    p.splits = 1u;
    const uint32_t behind = b.max_len - std::min(b.max_len, p.prefix.splits ? prefix : 0u);
    if (p.tokens) {
        TokensPlan &t = p.few;
        t.whole = true;
        t.tile_rows = shared <= 16u ? 16u : 32u;
        t.row_tiles = 1u;
        t.splits = p.splits = splits_of((uint64_t)b.n_reqs * heads, behind, (uint32_t)shared, dim);
        t.waves = waves_of((uint64_t)b.n_reqs * heads, t.splits);
        // Short prefixes of few requests: each reads its group's by itself (out of the caches), in one launch.  Measured (us, read once / so; requests x
        // tokens, one prefix): 8 heads x 128, 8 x 1, 1024 21.1 / 15.0, 64 x 1, 512 22.8 / 15.6, 1024 23.4 / 20.3, 128 x 1, 512 29.5 / 27.5, 1024 32.5 / 37.1,
        // 512 x 1, 64 42.7 / 30.0, 256 44.7 / 48.2; 4 x 64, 512 x 3, 512 36.9 / 30.3, 1024 42.6 / 45.3; 8 x 256, 128 x 1, 256 45.8 / 43.1, 512 46.9 / 53.1.
        const uint64_t pairs = (uint64_t)b.n_reqs * heads;
        p.through = p.prefix.splits && pairs * prefix * dim <= 1ull << 26 && splits_of(pairs, b.max_len, (uint32_t)shared, dim) == 1u;
        if (p.through) t.through = true, t.splits = p.splits = 1u, t.waves = waves_of((uint64_t)b.n_reqs * heads, 1u);
        if (t.splits == 1u && (uint64_t)b.n_reqs * heads > 1024u && alone((uint64_t)b.n_reqs * heads, p.through ? b.max_len : behind)) t.waves = 1u;
    } else {
        PartsPlan &m = p.many;
        m.row_tiles = (uint32_t)((shared + rows_each - 1u) / rows_each);
        // Splits as for prefixes; without any, and with an unsplit prefix, no part is written.  (Requests that share less have more behind it than
        // is counted for here, and more splits of the same length.)  Measured (us, the whole call,
        // unsplit / so; 8 heads x 128, 32 query heads): 8 requests of 16 new tokens, 4000 behind prefixes of 2000, 116 / 58, 8000 behind 175 / 78; two of 64 and
        // 8000 257 / 57; one of 40 and 20000, 2 heads, 566 / 66; one head of 256 and 7 query heads, 4 x 6 and 1400 99 / 34; 4 x 256 and 2000 168 / 172.
        const uint64_t likely = m.row_tiles > 1u ? (uint64_t)b.total_new * group / rows_each + b.n_reqs / 2u + 1u : b.n_reqs;
        const uint64_t groups = std::min((uint64_t)b.n_reqs * m.row_tiles, likely) * heads;
        const uint64_t tiles = (behind + 63u) / 64u;
        const bool last = !p.few_rows && p.prefix.splits == 1u;
        double best = INFINITY;
        for (uint32_t s = 1; s <= 16u && (s == 1u || s * 128u <= behind); s++) {
            const double parts = last && s == 1u ? 0.0 : (double)rows * (s + (last ? 1u : 0u)) * dim * 8.0 / 4e6;
            const double cost = (double)((groups * s + 255u) / 256u) * (double)((tiles + s - 1u) / s + 3u) * 2.5 + parts;
            if (cost < best) best = cost, m.splits = s;
        }
        // Or each request reads its group's prefix by itself, in one launch: what prompts do with codes takes longer than reading them.  Measured (us,
        // read once / so; 8 heads x 128, 32 query heads, three groups of 32 in all): 12 tokens behind 500 44.2 / 25.7, behind 2000 52.0 / 65.4; 64 behind
        // 2000 132 / 84, behind 6000 277 / 216; 32-512 behind 500 258 / 174, behind 6000 1168 / 1022; one of 8 such, behind 6000 358 / 409.
        const double alone_cost = (double)((groups + 255u) / 256u) * (double)((b.max_len + 63u) / 64u + 3u) * 2.5;
        p.through = p.prefix.splits && alone_cost <= once + best + 6.0;
        if (p.through) m.splits = 1u;
        const uint32_t length = m.splits > 1u ? std::max((behind + m.splits - 1u) / m.splits, b.max_len / 16u) : b.max_len;
        m.chunk = std::max(64u, (length + 63u) & ~63u);
        m.splits = p.splits = std::max(1u, (b.max_len + m.chunk - 1u) / m.chunk);
    }
    // Nothing split: the sums of what is behind the prefix are where the prefix begins, and its end writes outputs (32 prompts behind 4000
    // tokens, read once, 753 us; 810 with a part of every row more to write, and two to read).
    p.last = !p.few_rows && p.prefix.splits == 1u && p.splits == 1u && !p.through;
    // Few rows behind it that nothing splits: their workgroups read its parts and write outputs (64 tokens behind 8192: 55.6 us with a
    // launch that joins, 53.4 without).
    p.few.before = p.tokens && p.splits == 1u && !p.last && !p.through;
    const uint64_t parts = p.last || p.through ? 0u : rows * p.prefix.splits;
    z.prefix_parts = pad64(parts * 8u);
    z.sums = z.prefix_parts + pad64(parts * dim * 4u);
    const uint64_t behind_parts = p.through || p.few.before ? 0u : rows * p.splits;
    z.parts = z.sums + pad64(behind_parts * 8u);
    z.bytes = rows && b.n_reqs ? z.parts + pad64(behind_parts * dim * 4u) : 0u;
    return z;
}

dmi_status_t check_prefix(const dmi_kv8_prefix_t *k)
{
    if (!k) return fail(DMI_ERR_INVALID_ARG, "prefix is NULL");
    if (k->n_groups > kMaxReqs || k->max_prefix > kMaxLen)
        return fail(DMI_ERR_INVALID_ARG, "n_groups %u or max_prefix %u is too large", k->n_groups, k->max_prefix);
    return DMI_OK;
}

}  // namespace

extern "C" uint64_t dmi_kv8_attend_shared_workspace(const dmi_kv8_t *cache, const dmi_kv8_batch_t *batch, const dmi_kv8_prefix_t *prefix,
                                                    uint32_t n_q_heads)
{
    if (!cache || !batch || check_shape(cache, "cache") != DMI_OK || check_counts(batch, true) != DMI_OK ||
        check_attend(n_q_heads, cache->n_heads, *batch) != DMI_OK || check_prefix(prefix) != DMI_OK)
        return 0;
    return plan_shared(cache->n_heads, cache->head_dim, cache->block_size, *batch, *prefix, n_q_heads).bytes;
}

extern "C" dmi_status_t dmi_kv8_attend_shared(const dmi_kv8_t *cache, const dmi_kv8_batch_t *batch, const dmi_kv8_prefix_t *prefix,
                                              const dmi_kv8_heads_t *q, uint32_t n_q_heads, float scale, const dmi_kv8_heads_t *out,
                                              float *lse_dev, void *workspace, uint64_t workspace_bytes, void *hip_stream)
{
    AttendArgs a{};
    dmi_status_t st;
    if ((st = check_attention(cache, batch, q, n_q_heads, scale, out, lse_dev, a)) != DMI_OK || (st = check_prefix(prefix)) != DMI_OK) return st;
    if (prefix->n_groups && (!prefix->group_starts_dev || !prefix->prefix_dev))
        return fail(DMI_ERR_INVALID_ARG, "group_starts_dev or prefix_dev is NULL");
    if (((uintptr_t)prefix->group_starts_dev | (uintptr_t)prefix->prefix_dev) % 4u)
        return fail(DMI_ERR_INVALID_ARG, "group_starts_dev and prefix_dev must be 4-byte aligned");
    const SharedSizes z = plan_shared(a.c.heads, a.c.dim, a.c.bs, *batch, *prefix, n_q_heads);
    if ((st = check_workspace(z.bytes, workspace, workspace_bytes)) != DMI_OK) return st;
    if (!a.b.n_reqs || !a.b.total_new || !a.b.max_new) return DMI_OK;
    SharedPlan p = z.p;
    a.n_groups = p.prefix.splits ? prefix->n_groups : 0u;
    a.max_prefix = std::min(prefix->max_prefix, a.b.max_len);
    a.group_starts = prefix->group_starts_dev;
    a.prefix = prefix->prefix_dev;
    char *const at = static_cast<char *>(workspace);
    p.prefix.sums = reinterpret_cast<f32x2 *>(at);
    p.prefix.parts = reinterpret_cast<float *>(at + z.prefix_parts);
    p.prefix_few.sums = p.prefix.sums;
    p.prefix_few.parts = p.prefix.parts;
    p.few.prefix = PrefixParts{p.prefix.splits, p.few_rows ? 0u : p.prefix.chunk, p.prefix.sums, p.prefix.parts};
    p.few.sums = p.many.sums = p.sums = reinterpret_cast<f32x2 *>(at + z.sums);
    p.few.parts = p.many.parts = p.parts = reinterpret_cast<float *>(at + z.parts);
    return launched(launch_shared(a, p, q->dtype, (hipStream_t)hip_stream));
}
