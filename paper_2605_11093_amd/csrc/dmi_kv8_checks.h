// Checks of arguments that the C entry points of the operators on the 8-bit KV cache share.
#pragma once
#include "dmi_ring.h"
#include "dmi_kv8_internal.h"

#include <algorithm>
#include <cmath>

namespace dmi {
namespace kv8 {

using host::fail;
using host::dtype_size;

// A stride that moves rows by whole 16-byte units
inline bool whole(int64_t stride, uint32_t size) { return (stride * (int64_t)size) % 16 == 0; }

// Sizes that plans are made of
inline dmi_status_t check_shape(const dmi_kv8_t *k, const char *what)
{
    if (!k->block_size || k->block_size % 16u || k->block_size > kMaxBlock)
        return fail(DMI_ERR_INVALID_ARG, "%s: block_size %u is not a multiple of 16 up to %u", what, k->block_size, kMaxBlock);
    if (!k->head_dim || k->head_dim % 16u || k->head_dim > kMaxDim)
        return fail(DMI_ERR_INVALID_ARG, "%s: head_dim %u is not a multiple of 16 up to %u", what, k->head_dim, kMaxDim);
    if (!k->n_heads || k->n_heads > 1024u) return fail(DMI_ERR_INVALID_ARG, "%s: n_heads %u is not in 1..1024", what, k->n_heads);
    return DMI_OK;
}

inline dmi_status_t check_counts(const dmi_kv8_batch_t *k, bool fresh)
{
    if (k->n_reqs > kMaxReqs) return fail(DMI_ERR_INVALID_ARG, "n_reqs %u is more than %u", k->n_reqs, kMaxReqs);
    if (k->max_len > kMaxLen) return fail(DMI_ERR_INVALID_ARG, "max_len %u is more than %u", k->max_len, kMaxLen);
    if (fresh && (k->total_new > (1u << 30) || k->max_new > kMaxLen))
        return fail(DMI_ERR_INVALID_ARG, "total_new %u or max_new %u is too large", k->total_new, k->max_new);
    return DMI_OK;
}

// Kernels count query rows, and the tiles of 32 tokens of all contexts, in 31 bits; both with room to round up (and the bytes of a float
// for each row and 2^24 tokens are counted in 64).
constexpr uint64_t kMostRows = 1u << 30, kMostTiles = 1u << 30;

inline dmi_status_t check_attend(uint32_t n_q_heads, uint32_t heads, const dmi_kv8_batch_t &b)
{
    if (!n_q_heads || n_q_heads % heads || n_q_heads > 65536u)
        return fail(DMI_ERR_INVALID_ARG, "%u query heads do not share %u heads evenly", n_q_heads, heads);
    if ((uint64_t)b.total_new * n_q_heads > kMostRows)
        return fail(DMI_ERR_INVALID_ARG, "total_new %u rows of %u query heads are more than 2^30", b.total_new, n_q_heads);
    if (b.n_reqs * ((b.max_len + 31ull) / 32u) > kMostTiles)
        return fail(DMI_ERR_INVALID_ARG, "%u requests of max_len %u are more than 2^35 tokens", b.n_reqs, b.max_len);
    return DMI_OK;
}

inline dmi_status_t check_cache(const dmi_kv8_t *k, const char *what, Cache &c)
{
    if (!k) return fail(DMI_ERR_INVALID_ARG, "%s is NULL", what);
    if (!k->k || !k->v || !k->k_scale || !k->v_scale || !k->block_table_dev)
        return fail(DMI_ERR_INVALID_ARG, "%s: codes, scales or block table are NULL", what);
    if ((uintptr_t)k->k % 16u || (uintptr_t)k->v % 16u || !whole(k->block_stride, 1) || !whole(k->slot_stride, 1) ||
        !whole(k->head_stride, 1))
        return fail(DMI_ERR_INVALID_ARG, "%s: codes must be 16-byte aligned with strides that are multiples of 16", what);
    if (k->slot_stride < 0 || k->slot_stride > kMaxSlotStride)
        return fail(DMI_ERR_INVALID_ARG, "%s: slot_stride is not in 0..%lld", what, (long long)kMaxSlotStride);
    if ((uintptr_t)k->k_scale % 4u || (uintptr_t)k->v_scale % 4u || (uintptr_t)k->block_table_dev % 4u)
        return fail(DMI_ERR_INVALID_ARG, "%s: scales and block table must be 4-byte aligned", what);
    const dmi_status_t st = check_shape(k, what);
    if (st != DMI_OK) return st;
    if (!k->n_blocks || k->n_blocks > (1u << 30) || !k->n_seqs || k->n_seqs > (1u << 30) || !k->max_blocks ||
        k->max_blocks > kMaxLen || k->block_table_stride < (int64_t)k->max_blocks)
        return fail(DMI_ERR_INVALID_ARG, "%s: bad n_blocks, n_seqs, max_blocks or block_table_stride", what);
    c = Cache{{static_cast<uint8_t *>(k->k), static_cast<uint8_t *>(k->v)}, {k->k_scale, k->v_scale}, k->block_table_dev,
              k->block_stride, k->slot_stride, k->head_stride, k->scale_block_stride, k->scale_head_stride, k->block_table_stride,
              k->block_size, k->n_heads, k->head_dim, k->n_blocks, k->n_seqs, k->max_blocks, 0u};
    const uint32_t d = k->block_size / 16u;
    c.per_block = ((1u << 31) + d - 1u) / d;
    return DMI_OK;
}

inline dmi_status_t check_batch(const dmi_kv8_batch_t *k, const Cache &c, bool fresh, Batch &b)
{
    if (!k) return fail(DMI_ERR_INVALID_ARG, "batch is NULL");
    const dmi_status_t st = check_counts(k, fresh);
    if (st != DMI_OK) return st;
    if (k->n_reqs && !k->lens_dev) return fail(DMI_ERR_INVALID_ARG, "lens_dev is NULL");
    if (((uintptr_t)k->lens_dev | (uintptr_t)k->starts_dev | (uintptr_t)k->rows_dev) % 4u)
        return fail(DMI_ERR_INVALID_ARG, "lens_dev, starts_dev and rows_dev must be 4-byte aligned");
    if ((uint64_t)k->max_len > (uint64_t)c.max_blocks * c.bs)
        return fail(DMI_ERR_INVALID_ARG, "max_len %u is more than the block table's %u blocks of %u tokens", k->max_len, c.max_blocks, c.bs);
    if (!k->rows_dev && k->n_reqs > c.n_seqs)
        return fail(DMI_ERR_INVALID_ARG, "n_reqs %u is more than the block table's %u rows", k->n_reqs, c.n_seqs);
    if (fresh && !k->starts_dev && (k->total_new != k->n_reqs || k->max_new != 1u))
        return fail(DMI_ERR_INVALID_ARG, "without starts_dev there is one new token a request");
    b = Batch{k->lens_dev, k->starts_dev, k->rows_dev, k->n_reqs, k->total_new, std::min(k->max_new, k->total_new), k->max_len};
    return DMI_OK;
}

inline dmi_status_t check_rows(const dmi_kv8_heads_t *k, const char *what, const Batch &b, Rows &r)
{
    if (!k || (!k->data && b.total_new)) return fail(DMI_ERR_INVALID_ARG, "%s is NULL", what);
    const uint32_t size = dtype_size(k->dtype);
    if (size < 2u) return fail(DMI_ERR_INVALID_ARG, "%s: unsupported dtype %u", what, k->dtype);
    if ((uintptr_t)k->data % 16u || !whole(k->row_stride, size) || !whole(k->head_stride, size))
        return fail(DMI_ERR_INVALID_ARG, "%s must be 16-byte aligned with strides that are multiples of 16 bytes", what);
    r = Rows{k->data, k->row_stride, k->head_stride};
    return DMI_OK;
}

// Whether two tensors of n rows of heads (a number of heads each), `size` bytes an element, may share an element: exactly where their strides are the same, by
// the memory that they reach over where they are not.
inline bool share(const Rows &x, uint32_t x_heads, const Rows &y, uint32_t y_heads, uint32_t n, uint32_t dim, uint32_t size)
{
    typedef __int128 wide;
    struct Reach {
        wide lo, hi;
    };
    auto reach = [&](const Rows &r, uint32_t heads) {
        const wide row = (wide)r.row_stride * size * (n - 1), head = (wide)r.head_stride * size * (heads - 1), at = (wide)(uintptr_t)r.data;
        return Reach{at + std::min<wide>(row, 0) + std::min<wide>(head, 0), at + std::max<wide>(row, 0) + std::max<wide>(head, 0) + (wide)dim * size};
    };
    if (!n) return false;
    const Reach a = reach(x, x_heads), b = reach(y, y_heads);
    if (a.hi <= b.lo || b.hi <= a.lo) return false;
    if ((n > 1 && x.row_stride != y.row_stride) || (std::max(x_heads, y_heads) > 1 && x.head_stride != y.head_stride)) return true;
    const wide apart = (wide)(uintptr_t)y.data - (wide)(uintptr_t)x.data, length = (wide)dim * size;
    const wide row = n > 1 ? (wide)x.row_stride * size : 0;
    for (int64_t h = -(int64_t)x_heads + 1; h < (int64_t)y_heads; h++) {
        const wide d = apart + h * (wide)x.head_stride * size;      // one's element to the other's, of one row
        wide i = row ? -d / row : 0;                                // rows between them that come nearest: this many, or one more or less
        for (i--; ; i++) {
            const wide to = d + i * row;
            if (i > -(wide)n && i < (wide)n && to < length && -to < length) return true;
            if (i > (row ? -d / row : 0)) break;
        }
    }
    return false;
}

inline dmi_status_t check_weight(const dmi_kv8_weight_t *k, const char *what, Weight &w)
{
    w = Weight{nullptr, 0, 0};
    if (!k) return DMI_OK;
    if (!k->data || (uintptr_t)k->data % 4u) return fail(DMI_ERR_INVALID_ARG, "%s: data is NULL or not 4-byte aligned", what);
    w = Weight{k->data, k->row_stride, k->head_stride};
    return DMI_OK;
}

inline dmi_status_t launched(hipError_t e)
{
    if (e == hipErrorInvalidConfiguration) return fail(DMI_ERR_INVALID_ARG, "more work than a launch has workgroups for");
    return e == hipSuccess ? DMI_OK : fail(DMI_ERR_HIP, "launch failed: %s", hipGetErrorString(e));
}

inline dmi_status_t check_workspace(uint64_t need, const void *workspace, uint64_t bytes)
{
    if (need && (!workspace || (uintptr_t)workspace % 256u || bytes < need))
        return fail(DMI_ERR_INVALID_ARG, "workspace must be 256-byte aligned and hold %llu bytes", (unsigned long long)need);
    return DMI_OK;
}

}  // namespace kv8
}  // namespace dmi
