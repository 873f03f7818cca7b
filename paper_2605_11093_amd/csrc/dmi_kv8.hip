// The C entry points of the operators on the 8-bit KV cache: arguments checked, kernels' arguments made.
#include "dmi_kv8_checks.h"

#include <algorithm>
#include <cmath>

using namespace dmi;
using namespace dmi::host;
using namespace dmi::kv8;

extern "C" dmi_status_t dmi_kv8_append(const dmi_kv8_t *cache, const dmi_kv8_batch_t *batch, const dmi_kv8_heads_t *key,
                                       const dmi_kv8_heads_t *value, void *hip_stream)
{
    AppendArgs a;
    dmi_status_t st;
    if ((st = check_cache(cache, "cache", a.c)) != DMI_OK || (st = check_batch(batch, a.c, true, a.b)) != DMI_OK ||
        (st = check_rows(key, "key", a.b, a.x[0])) != DMI_OK || (st = check_rows(value, "value", a.b, a.x[1])) != DMI_OK)
        return st;
    if (key->dtype != value->dtype) return fail(DMI_ERR_INVALID_ARG, "key and value have different dtypes");
    if (!a.b.n_reqs || !a.b.total_new || !a.b.max_new || !a.b.max_len) return DMI_OK;
    a.touched = (a.b.max_new + a.c.bs - 2u) / a.c.bs + 1u;
    return launched(launch_append(a, key->dtype, (hipStream_t)hip_stream));
}

namespace {

// Which kernels attend, and what lies where in their workspace.
struct AttendPlan {
    bool tokens;
    TokensPlan t;
    PartsPlan many;
    uint64_t totals, sums, parts, bytes;        // offsets (scores come first), the whole
};

// Wavefronts of tokens_kernel that are resident at once, two on each SIMD: a step of 128 contexts (512-8192 tokens x 8 heads x 128)
// takes 190 us with them, 192 with one on each and 204 with three.
constexpr uint32_t kResident = 2048;

AttendPlan plan_attend(uint32_t block_heads, uint32_t dim, const dmi_kv8_batch_t &b, uint32_t q_heads, bool weight)
{
    AttendPlan p{};
    const uint32_t group = q_heads / block_heads, max_new = std::min(b.max_new, b.total_new);
    const uint64_t rows = (uint64_t)b.total_new * q_heads, shared = (uint64_t)max_new * group;
    if (!shared) {                              // no request has a query: weights lose their share, nothing else is there to do
        p.tokens = true;
        p.t.splits = p.t.ranges = p.t.row_tiles = 1u;
        p.t.tile_rows = 16u;
        return p;
    }
    // Up to 32 rows of queries share a head: tokens_kernel.  Measured (us, tokens / parts; 8 requests of 4000-8000 tokens and 64 of 2000-
    // 4000, 8 heads x 128): 16 rows 38 / 80 and 98 / 253, 32 rows 34 / 44 and 124 / 177, 64 rows 67 / 53 and 182 / 181.
    p.tokens = shared <= kFewRows;
    if (!p.tokens) {
        PartsPlan &m = p.many;
        const uint32_t rows_each = dim <= 128u ? 256u : 128u;
        m.row_tiles = (uint32_t)((shared + rows_each - 1u) / rows_each);
        // Workgroups run one on each of the 256 compute units: as many splits of the contexts as give the shortest sum of rounds, a
        // workgroup's start and end counted as three tiles of 64 tokens.  What splits write and the join reads is not counted: parts of
        // four long prompts behind up to 7600 tokens, 8 heads x 128, get six splits (150 MB of parts), and measure, weights included,
        // 371 us with six, 342 with one, 373 with two, 372 with three, 387 with four.
        const uint64_t bound = (uint64_t)b.n_reqs * m.row_tiles, likely = (uint64_t)b.total_new * group / rows_each + b.n_reqs / 2u + 1u;
        const uint64_t groups = std::min(bound, likely) * block_heads, len_tiles = (b.max_len + 63u) / 64u;
        uint64_t best = ~0ull;
        for (uint32_t s = 1; s <= 16u && (s == 1u || s * 512u <= b.max_len); s++) {
            const uint64_t cost = (groups * s + 255u) / 256u * (len_tiles / s + 3u);
            if (cost < best) best = cost, m.splits = s;
        }
        m.chunk = std::max(64u, ((b.max_len + m.splits - 1u) / m.splits + 63u) & ~63u);
        m.splits = std::max(1u, (b.max_len + m.chunk - 1u) / m.chunk);
        p.sums = weight ? pad64(rows * 4u) : 0u;
        p.parts = p.sums + (m.splits > 1u ? pad64(rows * m.splits * 8u) : 0u);
        p.bytes = p.parts + (m.splits > 1u ? pad64(rows * m.splits * dim * 4u) : 0u);
        return p;
    }
    TokensPlan &t = p.t;
    t.tile_rows = shared <= 16u || dim > 128u ? 16u : 32u;     // (two tiles of 256 elements take more registers than there are)
    t.row_tiles = ((uint32_t)shared + t.tile_rows - 1u) / t.tile_rows;
    // As many wavefronts as are resident at once, if there is enough for them; a request's tiles apart from others' where there is not.
    const uint32_t per = block_heads * t.row_tiles;
    const uint64_t tiles = (uint64_t)b.n_reqs * std::max(1u, (b.max_len + 31u) / 32u);
    t.ranges = (uint32_t)std::min<uint64_t>(std::max(kResident / per, 1u), std::max<uint64_t>(b.n_reqs, (tiles + 1u) / 2u));
    // Few or short contexts: one workgroup each and head, joined in LDS, and no second launch; longer ones in equal splits, of 512 tokens
    // while there are compute units for them.  Measured (us, ranges / whole): one request of 1024 tokens 17 / 12.5 (in two splits 17), of
    // 8000 34 / 17, of 32000 65 / 28; 8 of 2000-4000 28 / 23, of 4000-8000 36 / 34; 32 of 512-1024 24 / 17; 128 of them 49 / 55, of 128-256
    // 28 / 29; with 32 rows a head instead of 4, one of 8000 49 / 21, 128 of 768-1536 132 / 90.
    const uint64_t units = (uint64_t)b.n_reqs * block_heads;
    const uint32_t reach = shared > 16u ? 2048u : 1024u;       // tokens of a workgroup
    t.splits = 1;
    if (b.max_len > 1024u) t.splits = std::max(1u, (uint32_t)std::min<uint64_t>(256u / std::max<uint64_t>(units, 1u), (b.max_len + 511u) / 512u));
    if (b.max_len > reach * t.splits) t.splits = (b.max_len + reach - 1u) / reach;
    t.whole = t.row_tiles == 1u && (units * t.splits <= 512u || (t.splits == 1u && units <= 1u << 22 && (shared > 16u || b.max_len <= 256u)));
    t.join_blocks = t.whole ? t.splits > 1u : t.ranges > 1u;
    if (t.join_blocks) t.join_blocks = (uint32_t)(((uint64_t)max_new * q_heads + 3u) / 4u);
    t.score_stride = (b.max_len + 31u) & ~31u;
    const uint64_t parts = !t.join_blocks ? 0u : t.whole ? rows * t.splits : 2ull * t.ranges * per * t.tile_rows;
    p.totals = weight ? pad64(rows * t.score_stride * 4u) : 0u;
    p.sums = p.totals + (weight && !t.whole ? pad64(rows * 4u) : 0u);
    p.parts = p.sums + pad64(parts * 8u);
    p.bytes = p.parts + pad64(parts * dim * 4u);
    return p;
}

}  // namespace

extern "C" uint64_t dmi_kv8_attend_workspace(const dmi_kv8_t *cache, const dmi_kv8_batch_t *batch, uint32_t n_q_heads,
                                             int with_weight)
{
    if (!cache || !batch || check_shape(cache, "cache") != DMI_OK || check_counts(batch, true) != DMI_OK ||
        check_attend(n_q_heads, cache->n_heads, *batch) != DMI_OK)
        return 0;
    return plan_attend(cache->n_heads, cache->head_dim, *batch, n_q_heads, with_weight != 0).bytes;
}

extern "C" dmi_status_t dmi_kv8_attend(const dmi_kv8_t *cache, const dmi_kv8_batch_t *batch, const dmi_kv8_heads_t *q,
                                       uint32_t n_q_heads, float scale, const dmi_kv8_heads_t *out, float *lse_dev,
                                       const dmi_kv8_weight_t *weight, const dmi_kv8_weight_t *prior, float decay,
                                       void *workspace, uint64_t workspace_bytes, void *hip_stream)
{
    AttendArgs a{};
    dmi_status_t st;
    if ((st = check_cache(cache, "cache", a.c)) != DMI_OK || (st = check_batch(batch, a.c, true, a.b)) != DMI_OK ||
        (st = check_rows(q, "q", a.b, a.q)) != DMI_OK || (st = check_rows(out, "out", a.b, a.out)) != DMI_OK ||
        (st = check_weight(weight, "weight", a.w)) != DMI_OK || (st = check_weight(prior, "prior", a.prior)) != DMI_OK)
        return st;
    if (q->dtype != out->dtype || (q->dtype != DMI_DTYPE_BF16 && q->dtype != DMI_DTYPE_FP16))
        return fail(DMI_ERR_INVALID_ARG, "q and out must both be BF16 or both FP16");
    if ((st = check_attend(n_q_heads, a.c.heads, *batch)) != DMI_OK) return st;
    if (a.w.data && share(a.q, n_q_heads, a.out, n_q_heads, a.b.total_new, a.c.dim, 2u))
        return fail(DMI_ERR_INVALID_ARG, "out and q lie in the same memory, and weights are asked for");
    if (!std::isfinite(scale)) return fail(DMI_ERR_INVALID_ARG, "scale is not finite");
    if ((uintptr_t)lse_dev % 4u) return fail(DMI_ERR_INVALID_ARG, "lse_dev must be 4-byte aligned");
    if (a.prior.data && !a.w.data) return fail(DMI_ERR_INVALID_ARG, "prior without weight");
    if (a.prior.data && !std::isfinite(decay)) return fail(DMI_ERR_INVALID_ARG, "decay is not finite");
    const AttendPlan plan = plan_attend(a.c.heads, a.c.dim, *batch, n_q_heads, weight != nullptr);
    if ((st = check_workspace(plan.bytes, workspace, workspace_bytes)) != DMI_OK) return st;
    if (!a.b.n_reqs || (!a.b.max_new && !a.w.data)) return DMI_OK;
    a.lse = lse_dev;
    a.decay = a.prior.data ? decay : 0.0f;
    a.scale_log2 = scale * 1.44269504088896340736f;
    a.group = n_q_heads / a.c.heads;
    a.q_heads = n_q_heads;
    if (plan.tokens) {
        TokensPlan t = plan.t;
        char *const at = static_cast<char *>(workspace);
        t.scores = weight ? reinterpret_cast<float *>(at) : nullptr;
        t.totals = weight ? reinterpret_cast<float *>(at + plan.totals) : nullptr;
        t.sums = reinterpret_cast<f32x2 *>(at + plan.sums);
        t.parts = reinterpret_cast<float *>(at + plan.parts);
        return launched(launch_tokens(a, t, q->dtype, (hipStream_t)hip_stream));
    }
    PartsPlan m = plan.many;
    char *const at = static_cast<char *>(workspace);
    m.totals = weight ? reinterpret_cast<float *>(at) : nullptr;
    m.sums = reinterpret_cast<f32x2 *>(at + plan.sums);
    m.parts = reinterpret_cast<float *>(at + plan.parts);
    return launched(launch_parts(a, m, q->dtype, (hipStream_t)hip_stream));
}

extern "C" dmi_status_t dmi_kv8_evict(const dmi_kv8_t *cache, const dmi_kv8_batch_t *batch, const dmi_kv8_weight_t *weight,
                                      const dmi_kv8_t *to, const dmi_kv8_weight_t *to_weight, uint32_t keep, uint32_t recent,
                                      int32_t *positions_dev, int32_t *to_lens_dev, void *hip_stream)
{
    EvictArgs a;
    dmi_status_t st;
    if ((st = check_cache(cache, "cache", a.c)) != DMI_OK || (st = check_cache(to, "to", a.to)) != DMI_OK ||
        (st = check_batch(batch, a.c, false, a.b)) != DMI_OK || (st = check_weight(weight, "weight", a.w)) != DMI_OK ||
        (st = check_weight(to_weight, "to_weight", a.to_w)) != DMI_OK)
        return st;
    if (!a.w.data || !a.to_w.data) return fail(DMI_ERR_INVALID_ARG, "weight or to_weight is NULL");
    if (a.to.heads != a.c.heads || a.to.dim != a.c.dim || a.to.bs != a.c.bs)
        return fail(DMI_ERR_INVALID_ARG, "cache and to differ in n_heads, head_dim or block_size");
    if (a.to.n_seqs < a.c.n_seqs) return fail(DMI_ERR_INVALID_ARG, "to's block table has fewer rows than the cache's");
    if (!keep || recent > keep) return fail(DMI_ERR_INVALID_ARG, "keep %u must be positive and recent %u no more", keep, recent);
    if (keep > kMaxLen || (uint64_t)keep > (uint64_t)a.to.max_blocks * a.to.bs)
        return fail(DMI_ERR_INVALID_ARG, "keep %u is more than to's %u blocks of %u tokens, or than %u", keep, a.to.max_blocks, a.to.bs, kMaxLen);
    if (!positions_dev || !to_lens_dev || (uintptr_t)positions_dev % 4u || (uintptr_t)to_lens_dev % 4u)
        return fail(DMI_ERR_INVALID_ARG, "positions_dev or to_lens_dev is NULL or not 4-byte aligned");
    const int64_t apart = (int64_t)((uintptr_t)to_lens_dev - (uintptr_t)batch->lens_dev), length = 4ll * a.b.n_reqs;
    if (to_lens_dev == batch->lens_dev || (apart < length && -apart < length))
        return fail(DMI_ERR_INVALID_ARG, "to_lens_dev lies in lens_dev's memory");
    if (a.w.data == a.to_w.data) return fail(DMI_ERR_INVALID_ARG, "to_weight is weight");
    if (!a.b.n_reqs) return DMI_OK;
    a.b.starts = nullptr;
    a.keep = keep;
    a.recent = recent;
    a.positions = positions_dev;
    a.to_lens = to_lens_dev;
    return launched(launch_evict(a, (hipStream_t)hip_stream));
}
