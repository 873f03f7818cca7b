// Attention of few query rows over the 8-bit KV cache: single tokens, and a few of them.
#include "dmi_internal.h"
#include "dmi_kv8_mfma.h"

#include <cfloat>

namespace dmi {
namespace kv8 {

// ---------------------------------------------------------------- who does what
// All contexts of a call, in tiles of 32 tokens one behind the other, are cut into p.ranges equal ranges; a wavefront takes a
// range for one head (and one tile of query rows).  A context that lies within a range is finished there; of one that goes over
// an end, every range leaves a part: in place 1 of its two where the context begins in it, in place 0 otherwise (a range holds at
// most one of either), and a second launch puts them together.  Lengths are known on the device only, so every wavefront adds
// them up for itself; equal ranges leave no wavefront idle at the end, and none starts for nothing: a step of 128 contexts of 512-8192
// tokens took 238 us with workgroups for pieces of 1024 tokens each, and takes 181 so.
//
// Few or short contexts leave too little in a range, and too many parts.  There (p.whole) a workgroup takes a request and head, its
// wavefronts equal ranges of the context; their sums meet in LDS, and nothing is left for a second launch.  p.splits workgroups share a
// longer context and leave a part each.

// A request with new tokens has a tile at least: an empty context's rows are written too.
__device__ __forceinline__ int tiles_of(const Request &q) { return q.fresh > 0 ? max(1, (q.len + 31) >> 5) : 0; }

// The tiles of requests n0 .. n0 + 63, one request a lane
__device__ __forceinline__ int lane_tiles(const AttendArgs &a, uint32_t n0)
{
    const uint32_t r = n0 + (threadIdx.x & 63u);
    return r < a.b.n_reqs ? tiles_of(request_of(a.b, a.c, (int)r)) : 0;
}

// Tiles of a range, given the tiles of all contexts
__device__ __forceinline__ int range_tiles(const TokensPlan &p, int total) { return (total + (int)p.ranges - 1) / (int)p.ranges; }

__device__ __forceinline__ int all_tiles(const AttendArgs &a)
{
    int total = 0;
    for (uint32_t n0 = 0; n0 < a.b.n_reqs; n0 += 64u) total += __builtin_amdgcn_readlane(lanes_scan(lane_tiles(a, n0)), 63);
    return total;
}

// Index of a query row's part; `at`: the row of out, where contexts are split evenly
template <bool WHOLE> __device__ __forceinline__ int64_t part_at(const AttendArgs &a, const TokensPlan &p, int range, int place, uint32_t head, uint32_t row, int64_t at)
{
    if constexpr (WHOLE) return at * p.splits + range;
    const uint32_t tile = row / p.tile_rows;
    return (((int64_t)range * 2 + place) * p.row_tiles * a.c.heads + tile * a.c.heads + head) * p.tile_rows + (row - tile * p.tile_rows);
}

// ---------------------------------------------------------------- the sums
// The transposed products, scores S^T = K Q^T and outputs O^T = V^T P^T, with 16x16x32 matrix instructions: tokens (then elements)
// are rows, query rows are columns.  A lane's registers of S^T are then the P^T operand of the second product as they are: lane
// (column c, group g) holds tokens 4g..4g+3 of each of two sixteens of tokens, and which token stands at which place of the
// product's inner dimension is free as long as V agrees.  V is read with 8 tokens x 8 elements a lane (128 elements), its bytes
// interleaved by twos and converted: column m of V^T is element 8m + j for instruction j.  No operand passes through LDS.
//
// The softmax is one pass: sums against a maximum that is raised when scores rise more than 2^kSlack above it.  P is rounded to q's
// type for its product, sums and outputs are fp32.  Bound by the cache's bytes: 128 contexts, 1.04 GB in 181 us (5.8 TB/s; reads alone
// reach 7.1 here, a copy 5.0); for few tokens by the chain of loads that a wavefront starts with (lengths, table, codes; 9 us for one
// request of 500 tokens).  Codes of K in two halves of a line are read through the caches, V's past them (all past them: 272 us
// instead of 238 at that time).
constexpr int waves_of(int dp, int nt, bool whole) { return !whole || dp * nt > 128 ? 4 : 8; }

template <typename T, int DP, int NT, bool WHOLE>
__global__ __launch_bounds__(64 * waves_of(DP, NT, WHOLE)) __attribute__((amdgpu_waves_per_eu(DP * NT <= 128 ? 2 : 1)))
void tokens_kernel(AttendArgs a, TokensPlan p)
{
    constexpr int KL = DP / 64;                 // 16-byte loads of K a lane and sixteen
    constexpr int KK = DP / 32;                 // instructions for a sixteen's scores
    constexpr int VW = DP / 64;                 // words of V a lane and token
    constexpr int NJ = DP / 16;                 // instructions for 16 query rows' outputs
    [[maybe_unused]] constexpr int NW = waves_of(DP, NT, WHOLE);

    const int lane = threadIdx.x & 63, col = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint32_t head, row_tile = 0;
    int r = 0, seg0 = 0, range = 0, first, last;        // seg0: the request's first tile; first, last: the range's tiles
    Request held{0, 0, 0, 0};                           // of this lane, where there are no more than lanes
    if constexpr (WHOLE) {
        const uint32_t pair = blockIdx.x / p.splits;
        range = (int)(blockIdx.x - pair * p.splits);
        r = (int)(pair / a.c.heads);
        head = pair % a.c.heads;
        const Request q = request_of(a.b, a.c, r);
        const int tiles = q.fresh > 0 ? tiles_of(q) : a.w.data ? (q.len + 31) >> 5 : 0;
        const int nth = range * NW + wave, of = (int)p.splits * NW;
        first = (int)((int64_t)tiles * nth / of);
        last = (int)((int64_t)tiles * (nth + 1) / of);
    } else {
        // Workgroups go to the eight XCDs in turn: the heads (and row tiles) of a range follow each other on one of them.
        const uint32_t unit = (blockIdx.x >> 3) * 4u + (uint32_t)wave, per = a.c.heads * p.row_tiles;
        range = (int)(unit / per * 8u + (blockIdx.x & 7u));
        head = unit % per % a.c.heads, row_tile = unit % per / a.c.heads;
        if (range >= (int)p.ranges) return;
        // the range's first tile, the request that it lies in
        int total, of_range;
        if (a.b.n_reqs <= 64u) {
            if ((uint32_t)lane < a.b.n_reqs) held = request_of(a.b, a.c, lane);
            const int upto = lanes_scan(tiles_of(held));
            total = __builtin_amdgcn_readlane(upto, 63);
            of_range = range_tiles(p, total);
            if (range * of_range >= total) return;
            r = __ffsll((unsigned long long)__ballot(upto > range * of_range)) - 1;
            seg0 = r ? __builtin_amdgcn_readlane(upto, r - 1) : 0;
        } else {
            total = all_tiles(a);
            of_range = range_tiles(p, total);
            if (range * of_range >= total) return;
            for (;; r += 64) {
                if (r >= (int)a.b.n_reqs) return;
                const int upto = lanes_scan(lane_tiles(a, (uint32_t)r)), sum = __builtin_amdgcn_readlane(upto, 63);
                if (seg0 + sum <= range * of_range) {
                    seg0 += sum;
                    continue;
                }
                const int in = __ffsll((unsigned long long)__ballot(seg0 + upto > range * of_range)) - 1;
                seg0 += in ? __builtin_amdgcn_readlane(upto, in - 1) : 0;
                r += in;
                break;
            }
        }
        first = range * of_range;
        last = min(first + of_range, total);
    }
    const int row0 = (int)row_tile * 16 * NT;

    // byte offsets of this lane within a sixteen; elements past the row's end are read from its start (q is 0 there, and
    // V's columns there are not written)
    uint32_t k_off[KL], v_off;
#pragma unroll
    for (int c = 0; c < KL; c++) {
        const uint32_t d = (uint32_t)(g * (DP / 4) + 16 * c);
        k_off[c] = (uint32_t)col * (uint32_t)a.c.slot_stride + (d < a.c.dim ? d : 0u);
    }
    v_off = (uint32_t)(4 * g) * (uint32_t)a.c.slot_stride + ((uint32_t)col * (DP / 16) < a.c.dim ? (uint32_t)col * (DP / 16) : 0u);

    for (; r < (int)a.b.n_reqs && (WHOLE || seg0 < last); r++) {
        const Request q = !WHOLE && a.b.n_reqs <= 64u ? request_in(held, r) : request_of(a.b, a.c, r);
        const int seg_tiles = WHOLE ? last : tiles_of(q), seg_first = seg0;
        seg0 += seg_tiles;
        const int rows = q.fresh * (int)a.group;
        if (!WHOLE && (!seg_tiles || row0 >= rows)) continue;
        // this context's tiles in this range
        const int from = max(first, seg_first) - seg_first, to = min(last, seg_first + seg_tiles) - seg_first, tiles = to - from;
        const int begin = 32 * from, end = min(q.len, 32 * to);

        // entries and scales of the sixteens of 32 tiles, one a lane, and of the 32 tiles behind them
        struct Look {
            int entry;
            float ks, vs;
        };
        auto look = [&](int tile) {
            Look l{-1, 0.0f, 0.0f};
            const int t = begin + 32 * tile + 16 * lane;
            if (t < end) {
                l.entry = entry_of(a.c, q.row, block_of(a.c, (uint32_t)t >> 4));
                if (l.entry >= 0) {
                    l.ks = *scale_at(a.c, 0, l.entry, head) * a.scale_log2;
                    l.vs = *scale_at(a.c, 1, l.entry, head);
                }
            }
            return l;
        };
        Look here = look(0), behind{-1, 0.0f, 0.0f};

        u32x4 qf[NT][KK];
        int lim[NT];                            // the last position a column's query sees
#pragma unroll
        for (int n = 0; n < NT; n++) {
            const int row = row0 + 16 * n + col;
            const QueryRow w = query_row(a, head, (uint32_t)min(row, max(rows - 1, 0)));     // (columns behind the last row: not written)
            lim[n] = row < rows ? q.len - q.fresh + w.token : q.len;
            const uint16_t *src = static_cast<const uint16_t *>(a.q.data) + (int64_t)min(q.start + w.token, (int)a.b.total_new - 1) * a.q.row_stride +
                                  (int64_t)w.head * a.q.head_stride;
#pragma unroll
            for (int k = 0; k < KK; k++) {
                const int d = g * (DP / 4) + 8 * k;
                qf[n][k] = *reinterpret_cast<const u32x4 *>(src + (d < (int)a.c.dim ? d : 0));
            }
        }
        const int all_see = q.len - q.fresh + row0 / (int)a.group;      // what every row of the tile sees

        // Where a sixteen's codes lie; one that is not there is read at the cache's first block and counts no token.
        auto place = [&](int tile, int x) {
            const int six = 2 * (tile & 31) + x, t = begin + 32 * tile + 16 * x, e = max(__builtin_amdgcn_readlane(here.entry, six), 0);
            return (int64_t)e * a.c.block_stride + (int64_t)((uint32_t)t - block_of(a.c, (uint32_t)t >> 4) * a.c.bs) * a.c.slot_stride +
                   (int64_t)head * a.c.head_stride;
        };
        u32x4 rk[2][KL];
        uint32_t rv[8][VW];
        auto fetch_k = [&](int tile) {
#pragma unroll
            for (int x = 0; x < 2; x++) {
                const Buffer k = buffer_at(a.c.code[0] + place(tile, x));
#pragma unroll
                for (int c = 0; c < KL; c++) rk[x][c] = load_b128<0>(k, k_off[c]);
            }
        };
        auto fetch_v = [&](int tile) {
#pragma unroll
            for (int x = 0; x < 2; x++) {
                const Buffer v = buffer_at(a.c.code[1] + place(tile, x));
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const uint32_t at = v_off + (uint32_t)i * (uint32_t)a.c.slot_stride;
                    if constexpr (VW == 1) rv[4 * x + i][0] = load_b32<kOnce>(v, at);
                    if constexpr (VW == 2) {
                        const u32x2 w = load_b64<kOnce>(v, at);
                        rv[4 * x + i][0] = w[0], rv[4 * x + i][1] = w[1];
                    }
                    if constexpr (VW == 4) {
                        const u32x4 w = load_b128<kOnce>(v, at);
#pragma unroll
                        for (int y = 0; y < 4; y++) rv[4 * x + i][y] = w[y];
                    }
                }
            }
        };

        float m[NT], base[NT], l[NT];
        int unit = 0;                           // outputs are sums in units of 2^unit
        f32x4 o[NT][NJ];
#pragma unroll
        for (int n = 0; n < NT; n++) {
            m[n] = -INFINITY, base[n] = 0.0f, l[n] = 0.0f;
#pragma unroll
            for (int j = 0; j < NJ; j++) o[n][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }

        const bool any_tile = !WHOLE || (tiles > 0 && rows > 0);
        if (any_tile) {
            fetch_k(0);
            fetch_v(0);
        }
        if ((int)a.c.dim < DP) {
#pragma unroll
            for (int n = 0; n < NT; n++)
#pragma unroll
                for (int k = 0; k < KK; k++)
                    if (g * (DP / 4) + 8 * k >= (int)a.c.dim) qf[n][k] = u32x4{0u, 0u, 0u, 0u};
        }
        for (int tile = 0; any_tile && tile < tiles; tile++) {
            const int t0 = begin + 32 * tile, ahead = min(tile + 1, tiles - 1);
            int count[2];
            float ks[2], vs[2];                 // vs: V's scale between 1 and 2, times 2^ve
            int ve[2];
#pragma unroll
            for (int x = 0; x < 2; x++) {
                const int six = 2 * (tile & 31) + x;
                count[x] = __builtin_amdgcn_readlane(here.entry, six) < 0 ? 0 : min(16, end - t0 - 16 * x);
                ks[x] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(here.ks), six));
                const uint32_t scale = (uint32_t)__builtin_amdgcn_readlane(__float_as_int(here.vs), six);
                vs[x] = mantissa_of(scale), ve[x] = exponent_of(scale);
            }
            if ((tile & 31) == 0 && tile + 32 < tiles) behind = look(tile + 32);
            if ((tile & 31) == 31) here = behind;
            f32x4 z[NT][2];
#pragma unroll
            for (int x = 0; x < 2; x++) {
#pragma unroll
                for (int n = 0; n < NT; n++) z[n][x] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int k = 0; k < KK; k++) {
                    const uint32_t lo = rk[x][k / 2][2 * (k % 2)], hi = rk[x][k / 2][2 * (k % 2) + 1];
                    const u32x4 f = {T::two_codes(lo, false), T::two_codes(lo, true), T::two_codes(hi, false), T::two_codes(hi, true)};
#pragma unroll
                    for (int n = 0; n < NT; n++) z[n][x] = T::mfma16(f, qf[n][k], z[n][x]);
                }
#pragma unroll
                for (int n = 0; n < NT; n++) z[n][x] *= ks[x];
            }
            fetch_k(ahead);
            const bool full = count[0] == 16 && count[1] == 16 && t0 + 31 <= all_see;
            if (!full) {
                // tokens that are not there, or not seen: no score, and no NaN out of V
#pragma unroll
                for (int x = 0; x < 2; x++)
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const bool there = 4 * g + i < count[x];
#pragma unroll
                        for (int n = 0; n < NT; n++)
                            z[n][x][i] = there && t0 + 16 * x + 4 * g + i <= lim[n] ? z[n][x][i] : -INFINITY;
#pragma unroll
                        for (int y = 0; y < VW; y++) rv[4 * x + i][y] = there ? rv[4 * x + i][y] : 0u;
                    }
            }
            if (p.scores) {
                // (-inf says that a query does not see a token: its weight is 0 then whatever the row's total, a NaN too)
#pragma unroll
                for (int n = 0; n < NT; n++) {
                    const int row = row0 + 16 * n + col;
                    if (row < rows) {
                        float *s = p.scores + ((int64_t)head * a.b.total_new * a.group + (int64_t)q.start * a.group + row) * p.score_stride + t0 + 4 * g;
#pragma unroll
                        for (int x = 0; x < 2; x++) {
                            f32x4 kept;
#pragma unroll
                            for (int i = 0; i < 4; i++)
                                kept[i] = full || (4 * g + i < count[x] && t0 + 16 * x + 4 * g + i <= lim[n]) ? fmaxf(z[n][x][i], -FLT_MAX) : -INFINITY;
                            if (t0 + 16 * x < end) *reinterpret_cast<f32x4 *>(s + 16 * x) = kept;
                        }
                    }
                }
            }
            bool rises = false;
            float top[NT];
#pragma unroll
            for (int n = 0; n < NT; n++) {
                top[n] = fmaxf(fmaxf(fmaxf(z[n][0][0], z[n][0][1]), fmaxf(z[n][0][2], z[n][0][3])),
                               fmaxf(fmaxf(z[n][1][0], z[n][1][1]), fmaxf(z[n][1][2], z[n][1][3])));
                rises |= top[n] > m[n] + kSlack;
            }
            int moves = 0;                          // the sums' unit, by so many powers of two
            if constexpr (T::kNarrow) {
                const int to = unit_for(unit, ve);
                moves = unit - to;
                unit = to;
            }
            if (moves || __ballot(rises)) {
#pragma unroll
                for (int n = 0; n < NT; n++) {
                    float t = top[n];
                    t = fmaxf(t, __shfl_xor(t, 16));
                    t = fmaxf(t, __shfl_xor(t, 32));
                    const float now = fmaxf(m[n], t);
                    const float f = now == -INFINITY ? 1.0f : exp2_of(m[n] - now);
                    m[n] = now;
                    base[n] = now == -INFINITY ? 0.0f : now;
                    l[n] *= f;
                    const float g = T::kNarrow ? __builtin_ldexpf(f, moves) : f;
#pragma unroll
                    for (int j = 0; j < NJ; j++) o[n][j] *= g;
                }
            }
            u32x4 pf[NT];
#pragma unroll
            for (int n = 0; n < NT; n++) {
                float e[2][4];
#pragma unroll
                for (int x = 0; x < 2; x++) {
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        e[x][i] = exp2_of(z[n][x][i] - base[n]);
                        l[n] += e[x][i];
                        e[x][i] *= vs[x];
                    }
                    pf[n][2 * x] = T::pack(e[x][0], e[x][1]);
                    pf[n][2 * x + 1] = T::pack(e[x][2], e[x][3]);
                }
            }
            // A NaN in V of a token that some queries do not see: their p is 0, and 0 * NaN is not.  NaNs are taken out, and
            // a product of their own counts how many of them each query sees.
            if (!full) {
                uint32_t any = 0;
#pragma unroll
                for (int i = 0; i < 8; i++)
#pragma unroll
                    for (int y = 0; y < VW; y++) any |= nan_codes(rv[i][y]);
                if (__ballot(any != 0)) {
#pragma unroll 1
                    for (int j = 0; j < NJ; j++) {
                        u32x4 bad;
#pragma unroll
                        for (int i = 0; i < 4; i++) {
                            uint32_t w[2] = {0u, 0u};
#pragma unroll
                            for (int y = 0; y < VW; y++)
#pragma unroll
                                for (int e = 0; e < 2; e++)
                                    if (y == j / 4) w[e] = nan_codes(rv[2 * i + e][y]) >> (8 * (j % 4)) & 0x80u;
                            bad[i] = (w[0] ? T::kOne : 0u) | (w[1] ? T::kOne << 16 : 0u);
                        }
#pragma unroll
                        for (int n = 0; n < NT; n++) {
                            u32x4 seen;
#pragma unroll
                            for (int i = 0; i < 4; i++) {
                                const int t = t0 + 16 * (i / 2) + 4 * g + 2 * (i % 2);
                                seen[i] = (t <= lim[n] ? T::kOne : 0u) | (t + 1 <= lim[n] ? T::kOne << 16 : 0u);
                            }
                            const f32x4 nans = T::mfma16(bad, seen, f32x4{0.0f, 0.0f, 0.0f, 0.0f});
#pragma unroll
                            for (int k = 0; k < NJ; k++)
#pragma unroll
                                for (int i = 0; i < 4; i++) o[n][k][i] += k == j && nans[i] > 0.0f ? NAN : 0.0f;
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 8; i++)
#pragma unroll
                        for (int y = 0; y < VW; y++) rv[i][y] &= ~(nan_codes(rv[i][y]) | (nan_codes(rv[i][y]) - (nan_codes(rv[i][y]) >> 7)));
                }
            }
            uint32_t two[VW][2][4];                 // bytes of two tokens in turn: [word of a token][half][pair of tokens]
#pragma unroll
            for (int y = 0; y < VW; y++)
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    two[y][0][i] = __builtin_amdgcn_perm(rv[2 * i + 1][y], rv[2 * i][y], 0x05010400u);
                    two[y][1][i] = __builtin_amdgcn_perm(rv[2 * i + 1][y], rv[2 * i][y], 0x07030602u);
                }
            fetch_v(ahead);
            const float power[2] = {power_of(ve[0] - unit), power_of(ve[1] - unit)};
#pragma unroll
            for (int j = 0; j < NJ; j++) {
                u32x4 vf;
#pragma unroll
                for (int i = 0; i < 4; i++) vf[i] = T::two_codes(two[j / 4][j / 2 % 2][i], j % 2, power[i / 2]);
#pragma unroll
                for (int n = 0; n < NT; n++) o[n][j] = T::mfma16(vf, pf[n], o[n][j]);
            }
        }

        if constexpr (WHOLE) {
            // the wavefronts' sums, relative to the largest score of all; the later half of them hand theirs to the others
            constexpr int kSlots = NW / 2;
            __shared__ f32x4 joined[kSlots][NT * NJ * 64];
            __shared__ float tops[NW][16 * NT], sums[NW][16 * NT];
#pragma unroll
            for (int n = 0; n < NT; n++) {
                l[n] += __shfl_xor(l[n], 16);
                l[n] += __shfl_xor(l[n], 32);
                if (g == 0) tops[wave][16 * n + col] = m[n];
            }
            __syncthreads();
            auto top_of = [&](int c) {
                float t = -INFINITY;
#pragma unroll
                for (int v = 0; v < NW; v++) t = fmaxf(t, tops[v][c]);
                return t;
            };
            auto total_of = [&](int c, float &sum) {    // log2 of the sum of 2^score
                sum = 0.0f;
#pragma unroll
                for (int v = 0; v < NW; v++) sum += sums[v][c];
                const float t = top_of(c);
                return t == -INFINITY && sum == 0.0f ? -INFINITY : (t == -INFINITY ? 0.0f : t) + log2_of(sum);
            };
#pragma unroll
            for (int n = 0; n < NT; n++) {
                const float t = top_of(16 * n + col), f = exp2_of(m[n] - (t == -INFINITY ? 0.0f : t));
                if (g == 0) sums[wave][16 * n + col] = l[n] * f;
#pragma unroll
                for (int j = 0; j < NJ; j++) {
                    o[n][j] *= __builtin_ldexpf(f, unit);
                    if (wave >= kSlots) joined[wave - kSlots][(n * NJ + j) * 64 + lane] = o[n][j];
                }
            }
            __syncthreads();
            if (wave < kSlots) {
#pragma unroll
                for (int n = 0; n < NT; n++)
#pragma unroll
                    for (int j = 0; j < NJ; j++) joined[wave][(n * NJ + j) * 64 + lane] += o[n][j];
            }
            __syncthreads();
            for (int u = (int)threadIdx.x; u < NT * NJ / 4 * 64; u += 64 * NW) {
                const int n = (u >> 6) / (NJ / 4), j = (u >> 6) % (NJ / 4) * 4, row = 16 * n + col;
                if (row >= rows) continue;
                f32x4 sum[4] = {};
#pragma unroll
                for (int v = 0; v < kSlots; v++)
#pragma unroll
                    for (int k = 0; k < 4; k++) sum[k] += joined[v][(n * NJ + j + k) * 64 + lane];
                float l_all;
                const float total = total_of(row, l_all), f = total == -INFINITY && l_all == 0.0f ? 0.0f : 1.0f / l_all;
                const QueryRow w = query_row(a, head, (uint32_t)row);
                if (p.splits > 1u) {
                    const int64_t part = ((int64_t)(q.start + w.token) * a.q_heads + w.head) * p.splits + range;
                    if (g == 0 && j == 0) p.sums[part] = f32x2{top_of(row), l_all};
                    float *dst = p.parts + part * a.c.dim;
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const int d = NJ * (4 * g + i) + j;
                        if (d < (int)a.c.dim) *reinterpret_cast<f32x4 *>(dst + d) = f32x4{sum[0][i], sum[1][i], sum[2][i], sum[3][i]};
                    }
                    continue;
                }
                uint16_t *dst = static_cast<uint16_t *>(a.out.data) + (int64_t)(q.start + w.token) * a.out.row_stride + (int64_t)w.head * a.out.head_stride;
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const int d = NJ * (4 * g + i) + j;
                    if (d < (int)a.c.dim)
                        *reinterpret_cast<u32x2 *>(dst + d) = u32x2{T::pack(sum[0][i] * f, sum[1][i] * f), T::pack(sum[2][i] * f, sum[3][i] * f)};
                }
                if (a.lse && g == 0 && j == 0) a.lse[(int64_t)(q.start + w.token) * a.q_heads + w.head] = total * kLn2;
            }
            if (!a.w.data || p.splits > 1u) return;
            // weights, out of the scores that the same lane wrote
            float total[NT], unused;
#pragma unroll
            for (int n = 0; n < NT; n++) {
                total[n] = total_of(16 * n + col, unused);
                if (total[n] == -INFINITY) total[n] = INFINITY;         // a row that saw nothing weighs nothing
            }
            const float *prior = a.prior.data + (int64_t)q.row * a.prior.row_stride + (int64_t)head * a.prior.head_stride;
            float *to_w = a.w.data + (int64_t)q.row * a.w.row_stride + (int64_t)head * a.w.head_stride;
            const int older = q.len - q.fresh;
            const int last_row = max(rows - 1, 0);
            for (int t0 = begin; t0 < end; t0 += 128) {
                f32x4 z[NT][8];
                if (rows) {
#pragma unroll
                    for (int n = 0; n < NT; n++)
#pragma unroll
                        for (int x = 0; x < 8; x++)
                            z[n][x] = *reinterpret_cast<const f32x4 *>(
                                p.scores + ((int64_t)head * a.b.total_new * a.group + (int64_t)q.start * a.group + min(16 * n + col, last_row)) * p.score_stride +
                                min(t0 + 16 * x, (end - 1) & ~15) + 4 * g);
                }
                float sum[32];
#pragma unroll
                for (int e = 0; e < 32; e++) {
                    sum[e] = 0.0f;
#pragma unroll
                    for (int n = 0; n < NT; n++) sum[e] += 16 * n + col < rows && z[n][e / 4][e % 4] != -INFINITY ? exp2_of(z[n][e / 4][e % 4] - total[n]) : 0.0f;
                }
                // over the columns: of two lanes each goes on with half of the tokens
                halve<8, 16>(sum, col);
                halve<4, 8>(sum, col);
                halve<2, 4>(sum, col);
                halve<1, 2>(sum, col);
                const int t = t0 + 8 * (col & ~1) + 4 * g + 2 * (col & 1);
#pragma unroll
                for (int i = 0; i < 2; i++)
                    if (t + i < end) to_w[t + i] = a.prior.data && t + i < older ? a.decay * prior[t + i] + sum[i] : sum[i];
            }
            return;
        }
#pragma unroll
        for (int n = 0; n < NT; n++) {
            l[n] += __shfl_xor(l[n], 16);
            l[n] += __shfl_xor(l[n], 32);
            const int row = row0 + 16 * n + col;
            if (row >= rows) continue;
            const QueryRow w = query_row(a, head, (uint32_t)row);
            const int64_t at = (int64_t)(q.start + w.token) * a.q_heads + w.head;
            const bool whole = tiles == seg_tiles;
            const bool empty = m[n] == -INFINITY && l[n] == 0.0f;
            const float f = __builtin_ldexpf(whole ? (empty ? 0.0f : 1.0f / l[n]) : 1.0f, unit);
            // a lane holds DP / 4 elements of its row that follow each other
            if (whole) {
                uint16_t *dst = static_cast<uint16_t *>(a.out.data) + (int64_t)(q.start + w.token) * a.out.row_stride + (int64_t)w.head * a.out.head_stride;
#pragma unroll
                for (int i = 0; i < 4; i++)
#pragma unroll
                    for (int j = 0; j < NJ; j += 4) {
                        const int d = NJ * (4 * g + i) + j;
                        if (d < (int)a.c.dim)
                            *reinterpret_cast<u32x2 *>(dst + d) = u32x2{T::pack(o[n][j][i] * f, o[n][j + 1][i] * f), T::pack(o[n][j + 2][i] * f, o[n][j + 3][i] * f)};
                    }
                if (g == 0) {
                    const float sum = empty ? -INFINITY : m[n] + log2_of(l[n]);
                    if (a.lse) a.lse[at] = sum * kLn2;
                    if (p.totals) p.totals[at] = sum;
                }
            } else {
                const int64_t part = part_at<WHOLE>(a, p, range, seg_first >= first, head, (uint32_t)row, at);
                if (g == 0) p.sums[part] = f32x2{m[n], l[n]};
                float *dst = p.parts + part * a.c.dim;
#pragma unroll
                for (int i = 0; i < 4; i++)
#pragma unroll
                    for (int j = 0; j < NJ; j += 4) {
                        const int d = NJ * (4 * g + i) + j;
                        if (d < (int)a.c.dim)
                            *reinterpret_cast<f32x4 *>(dst + d) = f32x4{o[n][j][i], o[n][j + 1][i], o[n][j + 2][i], o[n][j + 3][i]} * f;
                    }
            }
        }
    }
}

// ---------------------------------------------------------------- what ranges leave
// A request's place among the ranges: whole in one, or parts from range `from` to `to`.
struct Spread {
    int from, to;
};
template <bool WHOLE> __device__ __forceinline__ Spread spread_of(const AttendArgs &a, const TokensPlan &p, uint32_t r)
{
    if constexpr (WHOLE) return {0, (int)p.splits - 1};
    int total = 0, before = 0, own = 0;
    for (uint32_t n0 = 0; n0 < a.b.n_reqs; n0 += 64u) {
        const int tiles = lane_tiles(a, n0), upto = lanes_scan(tiles);
        if (r >= n0 && r < n0 + 64u) {
            own = __builtin_amdgcn_readlane(tiles, (int)(r - n0));
            before = total + __builtin_amdgcn_readlane(upto, (int)(r - n0)) - own;
        }
        total += __builtin_amdgcn_readlane(upto, 63);
    }
    const int size = max(1, range_tiles(p, total));
    return {before / size, (before + max(own, 1) - 1) / size};
}

// log2 of the sum of 2^score over all of a row's context; every lane of the wavefront gets it
template <bool WHOLE> __device__ __forceinline__ float total_of(const AttendArgs &a, const TokensPlan &p, const Spread &s, uint32_t head, uint32_t row, int64_t at)
{
    const int lane = threadIdx.x & 63;
    float m = -INFINITY, l = 0.0f;
    for (int i = s.from + lane; i <= s.to; i += 64) {
        const f32x2 x = p.sums[part_at<WHOLE>(a, p, i, i == s.from, head, row, at)];
        const float top = fmaxf(m, x[0]), to = top == -INFINITY ? 0.0f : top;
        l = l * exp2_of(m - to) + x[1] * exp2_of(x[0] - to);
        m = top;
    }
    float top = m;
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) top = fmaxf(top, __shfl_xor(top, k));
    const float to = top == -INFINITY ? 0.0f : top;
    l *= exp2_of(m - to);
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) l += __shfl_xor(l, k);
    return top == -INFINITY && l == 0.0f ? -INFINITY : to + log2_of(l);
}

// The first p.join_blocks workgroups of a request: outputs out of parts, a wavefront a row, eight parts a team of lanes at once.  The
// others: weights out of the scores, four tokens a thread; query rows are added in order, so no result depends on timing.  Bound by
// loads that wait for each other: 8 us behind the 181 above; 16 contexts of up to 8192 tokens with weights 8 us
// behind 32 (what waits for no total is read first; 10 with one variant for both layouts of parts).
template <typename T, bool WHOLE>
__global__ __launch_bounds__(256) void finish_kernel(AttendArgs a, TokensPlan p)
{
    __shared__ float totals[kFewRows];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Request q = request_of(a.b, a.c, (int)blockIdx.y);
    const uint32_t rows = (uint32_t)q.fresh * a.group;
    if (blockIdx.x < p.join_blocks) {
        const uint32_t n = blockIdx.x * 4u + (uint32_t)wave;
        const Spread s = spread_of<WHOLE>(a, p, blockIdx.y);
        if (n >= rows * a.c.heads || s.from == s.to) return;
        const uint32_t head = n / rows, row = n - head * rows;
        const QueryRow w = query_row(a, head, row);
        const int64_t at = (int64_t)(q.start + w.token) * a.q_heads + w.head;
        const float total = total_of<WHOLE>(a, p, s, head, row, at);
        // as many parts at a time as there are lanes for
        const int wide = (int)a.c.dim / 4, teams = 64 / wide, team = lane / wide, d = 4 * (lane - team * wide);
        f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int i0 = s.from; i0 <= s.to && team < teams; i0 += 8 * teams) {
            f32x4 x[8];
            float f[8];
#pragma unroll
            for (int k = 0; k < 8; k++) {
                const int i = i0 + k * teams + team;
                const int64_t part = part_at<WHOLE>(a, p, min(i, s.to), min(i, s.to) == s.from, head, row, at);
                x[k] = *reinterpret_cast<const f32x4 *>(p.parts + part * a.c.dim + d);
                f[k] = p.sums[part][0];
            }
#pragma unroll
            for (int k = 0; k < 8; k++) {
                if (i0 + k * teams > s.to) break;
                if (i0 + k * teams + team <= s.to) sum += x[k] * (total == -INFINITY ? 0.0f : exp2_of(f[k] - total));
            }
        }
        for (int k = 1; k < teams; k++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const float other = __shfl(sum[i], lane + k * wide);
                if (team == 0) sum[i] += other;
            }
        if (team == 0) {
            uint16_t *dst = static_cast<uint16_t *>(a.out.data) + (int64_t)(q.start + w.token) * a.out.row_stride + (int64_t)w.head * a.out.head_stride + d;
            *reinterpret_cast<u32x2 *>(dst) = u32x2{T::pack(sum[0], sum[1]), T::pack(sum[2], sum[3])};
        }
        if (a.lse && !lane) a.lse[at] = total * kLn2;
        return;
    }
    const uint32_t rest = blockIdx.x - p.join_blocks, head = rest % a.c.heads;
    const int t0 = 1024 * (int)(rest / a.c.heads), t = t0 + 4 * (int)threadIdx.x, older = q.len - q.fresh;
    if (t0 >= q.len) return;
    // what waits for no total: prior weights, and the first rows' scores
    constexpr int kFirst = 4;
    const float *scores = p.scores + ((int64_t)head * a.b.total_new * a.group + (int64_t)q.start * a.group) * p.score_stride + (t < q.len ? t : 0);
    const float *prior = a.prior.data + (int64_t)q.row * a.prior.row_stride + (int64_t)head * a.prior.head_stride;
    f32x4 z[kFirst], before = {0.0f, 0.0f, 0.0f, 0.0f};
    if (rows) {
#pragma unroll
        for (int r = 0; r < kFirst; r++) z[r] = *reinterpret_cast<const f32x4 *>(scores + (int64_t)min(r, (int)rows - 1) * p.score_stride);
    }
    if (a.prior.data) {
#pragma unroll
        for (int i = 0; i < 4; i++) before[i] = prior[max(min(t + i, older - 1), 0)];
    }
    const Spread s = spread_of<WHOLE>(a, p, blockIdx.y);
    for (int r = wave; r < (int)rows; r += 4) {
        const QueryRow w = query_row(a, head, (uint32_t)r);
        const int64_t at = (int64_t)(q.start + w.token) * a.q_heads + w.head;
        const float total = s.from == s.to ? p.totals[at] : total_of<WHOLE>(a, p, s, head, (uint32_t)r, at);
        if (!lane) totals[r] = total == -INFINITY ? INFINITY : total;       // (a row that saw nothing weighs nothing)
    }
    __syncthreads();
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
    auto add = [&](int r, const f32x4 &x) {
        const float total = totals[r];
#pragma unroll
        for (int i = 0; i < 4; i++) sum[i] += x[i] == -INFINITY ? 0.0f : exp2_of(x[i] - total);
    };
#pragma unroll
    for (int r = 0; r < kFirst; r++)
        if (r < (int)rows) add(r, z[r]);
    if (t < q.len) {
#pragma unroll 4
        for (int r = kFirst; r < (int)rows; r++) add(r, *reinterpret_cast<const f32x4 *>(scores + (int64_t)r * p.score_stride));
    }
    float *to = a.w.data + (int64_t)q.row * a.w.row_stride + (int64_t)head * a.w.head_stride;
#pragma unroll
    for (int i = 0; i < 4; i++)
        if (t + i < q.len) to[t + i] = a.prior.data && t + i < older ? a.decay * before[i] + sum[i] : sum[i];
}

template <typename T> static hipError_t tokens(const AttendArgs &a, const TokensPlan &p, hipStream_t s)
{
    const uint32_t per = a.c.heads * p.row_tiles, units = (p.ranges + 7u) / 8u * per;      // on each XCD
    const uint64_t finish_groups = p.whole && p.splits == 1u ? 0u : p.join_blocks + (a.w.data ? (a.b.max_len + 1023ull) / 1024u * a.c.heads : 0u);
    if (!launchable(finish_groups, 256)) return hipErrorInvalidConfiguration;
    const int dp = a.c.dim <= 64 ? 64 : a.c.dim <= 128 ? 128 : 256;
    auto launch = [&](auto dp_, auto nt_) {
        if (!a.b.max_new) return;               // (no queries: what they would read is not there)
        constexpr int DP = decltype(dp_)::value, NT = decltype(nt_)::value;
        if (p.whole) tokens_kernel<T, DP, NT, true><<<a.b.n_reqs * a.c.heads * p.splits, 64 * waves_of(DP, NT, true), 0, s>>>(a, p);
        else tokens_kernel<T, DP, NT, false><<<(units + 3u) / 4u * 8u, 256, 0, s>>>(a, p);
    };
    if (p.tile_rows == 16) {
        if (dp == 64) launch(Int<64>{}, Int<1>{});
        else if (dp == 128) launch(Int<128>{}, Int<1>{});
        else launch(Int<256>{}, Int<1>{});
    } else {
        if (dp == 64) launch(Int<64>{}, Int<2>{});
        else launch(Int<128>{}, Int<2>{});
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !finish_groups) return e;
    const dim3 finish((uint32_t)finish_groups, a.b.n_reqs);
    if (p.whole) finish_kernel<T, true><<<finish, 256, 0, s>>>(a, p);
    else finish_kernel<T, false><<<finish, 256, 0, s>>>(a, p);
    return hipGetLastError();
}

hipError_t launch_tokens(const AttendArgs &a, const TokensPlan &p, uint32_t dtype, hipStream_t s)
{
    return dtype == DMI_DTYPE_BF16 ? tokens<Bf16>(a, p, s) : tokens<Fp16>(a, p, s);
}

}  // namespace kv8
}  // namespace dmi
