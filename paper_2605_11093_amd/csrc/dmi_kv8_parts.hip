// Attention of many query rows over the 8-bit KV cache: prompts and parts of prompts.
#include "dmi_internal.h"
#include "dmi_kv8_mfma.h"

#include <algorithm>
#include <cfloat>

namespace dmi {
namespace kv8 {

constexpr int kTile = 64;                       // tokens that a workgroup has in LDS at a time

// What is looked up of sixteens of tokens, one a lane: entry of the block table, K's scale.
struct Look {
    int entry;
    float ks;
};
__device__ __forceinline__ Look look_up(const AttendArgs &a, const Request &q, uint32_t head, int t, int end, float scale)
{
    Look l{-1, 1.0f};
    if (t < end) {
        l.entry = entry_of(a.c, q.row, block_of(a.c, (uint32_t)t >> 4));
        if (l.entry >= 0) l.ks = *scale_at(a.c, 0, l.entry, head) * scale;
    }
    return l;
}
__device__ __forceinline__ float lane_value(float v, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane)); }

// As in tokens_kernel, S^T = K Q^T and O^T = V^T P^T with query rows as columns, here with 32x32x16 instructions, 32 query rows a
// wavefront, NW wavefronts on the same tokens.  K and V are converted once for the workgroup, on their way into LDS: K as it
// lies, V transposed, the tokens of a sixteen in the order in which the lanes' registers of S^T hold them (0-3, 8-11 for lanes
// 0-31, 4-7, 12-15 for lanes 32-63), so that an operand is 16 bytes in a row.  Both have two places in LDS: one tile is staged while
// the other is used, with one barrier a tile.
//
// Bound by neither pipe alone: a tile takes a wavefront 32 matrix instructions (1280 cycles) and some 280 vector ones (1500), 112 of
// them to stage, and the two wavefronts of a SIMD together 6000 cycles: they leave the barrier together and so want the same pipe
// at the same time; a workgroup's start and end cost as much as four tiles of its dozen.  32 ragged prompts of 128-2048 tokens, 32 query
// heads over 8: 581 to 638 us by card, 706 to 773 TFLOP/s (a large product of the library: 1250); parts of four long prompts, six splits,
// 222 to 232 us, 755 to 790 TFLOP/s.  In fp16 and with 256 elements 2 to 3 % more.  Queries and
// outputs that went between memory and the lanes without LDS cost 33 us of it.  Measured and not better (before that, at 620): one
// wavefront of 64 rows a SIMD (spills), the second four wavefronts half a tile behind the first (658), staging between the
// instructions of a product (627-671), two workgroups of four wavefronts (634), priorities (624-639), a maximum looked for only where
// sums grow (637-700), two to eight row tiles a workgroup in turn (670-818), workgroups that stay and draw row tiles (642).
template <typename T, int DP, int NW, Kind KIND = kWhole>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(NW / 4)))
void parts_kernel(AttendArgs a, PartsPlan p)
{
    constexpr bool PREFIX = KIND == kPrefix || KIND == kLast;
    constexpr int KP = DP * 2 + 16, VP = kTile * 2;             // bytes of a row in LDS; K's are padded so that rows start on other banks
    constexpr int KK = DP / 16, ND = DP / 32;
    constexpr int A = DP <= 128 ? 8 : 3;                        // operands read ahead (four, with 256 elements: 433 us for 424)
    constexpr int U = 8 / NW;                                   // eights of the tile's tokens that a wavefront stages
    constexpr int KL = DP <= 128 ? 1 : 2;                       // 16-byte loads of K a lane and eight
    constexpr int VL = DP <= 128 ? 1 : 2;                       // units of 4 tokens x 4 elements a lane and eight
    __shared__ __align__(16) uint8_t lds[2 * (kTile * KP + DP * VP)];
    // NaNs in V: the last tile, counted from 1, that had one (in an eight); a bit for each of 4 tokens
    __shared__ int nan_any[2], nan_tile[2][8];
    __shared__ __align__(4) uint8_t nan_bits[2][8][2][DP];
    // scales of sixteens: K's, log2 and inverse of what V's is between 1 and 2, of 16 tiles and the next 16
    __shared__ __align__(16) float scales[2][3][64];
    auto lk = [&](int tile) { return lds + (tile & 1) * (kTile * KP); };
    auto lv = [&](int tile) { return lds + 2 * kTile * KP + (tile & 1) * (DP * VP); };
    // V's 16-byte chunks are exchanged by row, so that neither the rows that lanes read nor those that they write (every fourth) meet
    // on a bank
    auto chunk_of = [](int row, int chunk) { return chunk ^ ((row >> 2 & 3) | ((row >> 1 ^ row >> 4) & 1) << 2); };

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
    // The row tiles of a request and head on one XCD, those that see most first: workgroups go to the eight XCDs in turn, and every eighth
    // pair of request and head belongs to each.
    const uint32_t xcd = blockIdx.x & 7u, item = (blockIdx.x >> 3) / p.splits, split = (blockIdx.x >> 3) - item * p.splits;
    const bool spread = KIND != kWhole && p.spread;             // (row tiles in turn)
    Request q{0, 0, 0, 0};
    uint32_t head = 0;
    [[maybe_unused]] int unit_at = 0;           // the request, or group
    [[maybe_unused]] uint32_t skipped = 0;      // kRest: blocks in front
    [[maybe_unused]] uint32_t front = 0;        // kThrough: blocks that are read through front_row
    [[maybe_unused]] int front_row = 0;
    int row0 = -1;
    const uint32_t units = PREFIX ? a.n_groups : a.b.n_reqs;
    if (p.counted) {
        // as many workgroups as all requests' rows make: their tiles are counted here
        for (uint32_t n0 = 0, before = 0; n0 < units; n0 += 64u) {
            const uint32_t r = n0 + (uint32_t)lane;
            Request own{0, 0, 0, 0};
            if (r < units) own = PREFIX ? group_rows(a, (int)r) : request_of(a.b, a.c, (int)r);
            const int row_tiles = (own.fresh * (int)a.group + 32 * NW - 1) / (32 * NW);
            const uint32_t pairs = spread ? a.c.heads : ((r + 1u) * a.c.heads + 7u - xcd) / 8u - (r * a.c.heads + 7u - xcd) / 8u;
            const int upto = lanes_scan(row_tiles * (int)pairs), place = (int)((spread ? 8u * item + xcd : item) - before);
            const uint64_t behind = __ballot(upto > place);
            if (!behind) {
                before += (uint32_t)__builtin_amdgcn_readlane(upto, 63);
                continue;
            }
            const int in = __ffsll((unsigned long long)behind) - 1, of = __builtin_amdgcn_readlane(row_tiles, in);
            const int nth = place - (in ? __builtin_amdgcn_readlane(upto, in - 1) : 0), which = nth / of;
            const uint32_t first = (n0 + (uint32_t)in) * a.c.heads;
            q = request_in(own, in);
            unit_at = (int)n0 + in;
            head = spread ? (uint32_t)which : ((xcd - first) & 7u) + 8u * (uint32_t)which;
            row0 = (of - 1 - (nth - which * of)) * 32 * NW;
            break;
        }
    } else {
        // as many for every request as the one with most rows has
        const uint32_t pair = item / p.row_tiles * 8u + xcd, r = pair / a.c.heads;
        if (r >= units) return;
        head = pair - r * a.c.heads;
        q = PREFIX ? group_rows(a, (int)r) : request_of(a.b, a.c, (int)r);
        unit_at = (int)r;
        row0 = (int)(p.row_tiles - 1u - item % p.row_tiles) * 32 * NW;
        if (row0 >= q.fresh * (int)a.group) return;
    }
    if (row0 < 0) return;
    const int rows = q.fresh * (int)a.group;
    if constexpr (PREFIX) q.len = group_tokens(a, unit_at, q.row);
    if constexpr (KIND == kRest) {
        const int shared = shared_tokens(a, unit_at, q);
        q.len -= shared;
        skipped = block_of(a.c, (uint32_t)shared >> 4);
    }
    if constexpr (KIND == kThrough) front = block_of(a.c, (uint32_t)shared_tokens(a, unit_at, q, front_row) >> 4);
    const int older = PREFIX ? q.len - 1 : q.len - q.fresh, last_row = min(row0 + 32 * NW, rows) - 1;
    // tokens that the workgroup's last row sees (of a prefix all rows see all)
    const int seen = PREFIX ? q.len : older + last_row / (int)a.group + 1;
    const int begin = (int)(split * p.chunk), end = min(seen, begin + (int)p.chunk), tiles = max(0, (end - begin + kTile - 1) / kTile);
    if (split && tiles == 0) return;                            // (what reads the parts counts the same way)

    // the wavefront's query rows; a negative scale goes into their sign
    const uint32_t flip = a.scale_log2 < 0.0f ? 0x80008000u : 0u;
    const float scale = fabsf(a.scale_log2);
    const int wave_row = row0 + wave * 32, row = wave_row + col;
    const QueryRow w = query_row(a, head, (uint32_t)row);
    const int lim = row < rows ? older + (PREFIX ? 0 : w.token) : -1;      // the last position that the column's query sees
    // Read by whole rows, and given to the lanes that take them through LDS (rows of its own for each wavefront; outputs go the same way)
    constexpr int kRow = 2 * DP, kChunks = DP / 8, kRows = 64 / kChunks;       // bytes; 16s of them; rows of a load
    static_assert(NW * 32 * kRow <= 2 * (kTile * KP + DP * VP));
    uint8_t *const own = lds + wave * 32 * kRow;
    auto in_row = [&](int r, int chunk) { return own + r * kRow + 16 * (chunk ^ (r & (kChunks - 1))); };
    u32x4 qf[KK];
    {
        // (loads that depend on nothing: each in a branch of its own would wait for itself)
        const QueryRow v = query_row(a, head, (uint32_t)min(row, rows - 1));
        const int64_t src = (int64_t)(q.start + v.token) * a.q.row_stride + (int64_t)v.head * a.q.head_stride;
        const int chunk = lane % kChunks;
#pragma unroll
        for (int k = 0; k < KK; k++) {
            const int r = k * kRows + lane / kChunks;
            const int64_t from = (int64_t)(uint32_t)__shfl((int)(uint32_t)src, r) | (int64_t)__shfl((int)(src >> 32), r) << 32;
            qf[k] = *reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(a.q.data) + from + (8 * chunk < (int)a.c.dim ? 8 * chunk : 0));
        }
    }
    // what the first and the last of them see
    const int least = wave_row + 32 <= rows ? older + (PREFIX ? 0 : wave_row / (int)a.group) : -1;
    const int most = wave_row < rows ? older + (PREFIX ? 0 : min(wave_row + 31, rows - 1) / (int)a.group) : -1;

    // ---- staging
    struct KCodes {
        u32x4 w[U][KL];
    };
    struct VCodes {
        uint32_t w[U][VL][4];
        int there[U];                           // tokens of the sixteen
        float power[U];                         // what codes are converted times
    };
    uint32_t k_off[KL], v_off[VL];              // this lane's offsets in a sixteen: 8 lanes a token of K (4 if it has 64 elements)
#pragma unroll
    for (int c = 0; c < KL; c++) {
        const uint32_t d = DP == 64 ? 16u * (lane & 3) : 128u * c + 16u * (lane & 7);
        k_off[c] = (DP == 64 ? (lane >> 2 & 7) : lane >> 3) * (uint32_t)a.c.slot_stride + (d < a.c.dim ? d : 0u);
    }
#pragma unroll
    for (int c = 0; c < VL; c++) {
        const uint32_t unit = lane + 64 * c, d = 4 * (unit % (DP / 4));
        v_off[c] = 8u * (unit / (DP / 4) & 1u) * (uint32_t)a.c.slot_stride + (d < a.c.dim ? d : 0u);
    }
    // Where sixteens lie, from the first code on: a batch's 64, one a lane (the cache's first, if there is no entry)
    struct Places {
        uint32_t lo, hi;
        int e;                                  // exponent of V's scale
        uint64_t there;                         // which of them the cache has
        uint64_t far;                           // fp16: whose scale lies outside of the unit's reach
    };
    int unit = 0;                               // of the sums over V: see unit_for
    // a batch of 16 tiles is looked up, and its scales go into LDS (every wavefront writes the same; what is not there is masked, and
    // weighs nothing); what is done in between does not wait for the scales
    auto look = [&](int batch, auto between) {
        const int t = begin + 1024 * batch + 16 * lane;
        const uint32_t block = block_of(a.c, (uint32_t)t >> 4);
        const uint32_t column = KIND == kRest ? block + skipped : block;
        const int raw = a.c.table[(int64_t)(KIND == kThrough && block < front ? front_row : q.row) * a.c.table_stride + min(column, a.c.max_blocks - 1u)];
        const bool there = t < end && column < a.c.max_blocks && (uint32_t)raw < a.c.n_blocks;
        const int entry = there ? raw : 0;
        const int64_t at = (int64_t)entry * a.c.block_stride + (int64_t)((uint32_t)t - block * a.c.bs) * a.c.slot_stride + (int64_t)head * a.c.head_stride;
        Places l{(uint32_t)at, (uint32_t)(at >> 32), 0, __ballot(there), 0};
        const float ks = *scale_at(a.c, 0, entry, head), vs = *scale_at(a.c, 1, entry, head);
        between(l);
        l.e = there ? exponent_of(__float_as_uint(vs)) : -126;
        if constexpr (T::kNarrow) l.far = __ballot(outside(l.e, unit));
        const float m = mantissa_of(__float_as_uint(vs));
        scales[batch & 1][0][lane] = there ? fmaxf(ks * scale, FLT_MIN) : 1.0f;     // (-inf times 0 would be no mask)
        scales[batch & 1][1][lane] = there ? log2_of(m) : -INFINITY;
        scales[batch & 1][2][lane] = there ? 1.0f / m : 0.0f;
        return l;
    };
    auto fetch = [&](int tile, const Places &p, KCodes &k, VCodes &v) {
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int eight = wave + NW * u, six = (4 * tile + (eight >> 1)) & 63;
            const uint64_t at = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)p.hi, six) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)p.lo, six);
            const Buffer bk = buffer_at(a.c.code[0] + at), bv = buffer_at(a.c.code[1] + at);
            v.there[u] = p.there >> six & 1u ? min(16, end - begin - kTile * tile - 16 * (eight >> 1)) : 0;
#pragma unroll
            for (int c = 0; c < KL; c++) k.w[u][c] = load_b128<0>(bk, k_off[c] + ((eight & 1) ? 8u * (uint32_t)a.c.slot_stride : 0u));
#pragma unroll
            for (int c = 0; c < VL; c++)
#pragma unroll
                for (int i = 0; i < 4; i++)
                    v.w[u][c][i] = load_b32<0>(bv, v_off[c] + ((eight & 1) ? 4u * (uint32_t)a.c.slot_stride : 0u) + (uint32_t)i * (uint32_t)a.c.slot_stride);
        }
    };
    auto place_k = [&](const KCodes &r, int tile) {
#pragma unroll
        for (int u = 0; u < U; u++)
#pragma unroll
            for (int c = 0; c < KL; c++) {
                const int d = DP == 64 ? 16 * (lane & 3) : 128 * c + 16 * (lane & 7), token = 8 * (wave + NW * u) + (DP == 64 ? lane >> 2 : lane >> 3);
                uint8_t *const to = lk(tile) + token * KP + 2 * d;
                const u32x4 k = r.w[u][c];
                if (DP > 64 || lane < 32) {
                    *reinterpret_cast<u32x4 *>(to) = u32x4{T::two_codes(k[0], false), T::two_codes(k[0], true), T::two_codes(k[1], false), T::two_codes(k[1], true)};
                    *reinterpret_cast<u32x4 *>(to + 16) = u32x4{T::two_codes(k[2], false), T::two_codes(k[2], true), T::two_codes(k[3], false), T::two_codes(k[3], true)};
                }
            }
    };
    // What V's codes are converted times, in the unit of the tile; which of the batch's scales lie outside of its reach
    auto powers = [&](int tile, int exponents, uint64_t far, VCodes &v) {
        auto exponent_in = [&](int x) { return __builtin_amdgcn_readlane(exponents, (4 * tile + x) & 63); };
        if constexpr (T::kNarrow) {
            if (far >> (4 * tile & 63) & 15u) {
                unit = unit_for(unit, {exponent_in(0), exponent_in(1), exponent_in(2), exponent_in(3)});
                far = __ballot(outside(exponents, unit));
            }
        }
#pragma unroll
        for (int u = 0; u < U; u++) v.power[u] = power_of(exponent_in((wave + NW * u) >> 1) - unit);
        return far;
    };
    // V's codes as they come: nothing where there is no token, and 0 in a NaN's place (the queries that see it are given it apart)
    auto clean_v = [&](VCodes &r, int tile) {
        const int buf = tile & 1;
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int eight = wave + NW * u;
            uint32_t any = 0;
            if (r.there[u] < 16) {
                asm volatile("");               // (a branch that most tiles skip)
#pragma unroll
                for (int c = 0; c < VL; c++)
#pragma unroll
                    for (int i = 0; i < 4; i++)
                        r.w[u][c][i] = 4 * (eight & 1) + 8 * ((lane + 64 * c) / (DP / 4) & 1) + i < r.there[u] ? r.w[u][c][i] : 0u;
            }
#pragma unroll
            for (int c = 0; c < VL; c++)
#pragma unroll
                for (int i = 0; i < 4; i++) any |= nan_codes(r.w[u][c][i]);
            if (__ballot(any != 0)) {
                if (lane == 0) nan_any[buf] = nan_tile[buf][eight] = tile + 1;
#pragma unroll
                for (int c = 0; c < VL; c++) {
                    const int unit = lane + 64 * c, d = 4 * (unit % (DP / 4));
                    uint32_t bits = 0;
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const uint32_t top = nan_codes(r.w[u][c][i]);
                        bits |= top >> (7 - i);
                        r.w[u][c][i] &= ~(top | (top - (top >> 7)));
                    }
                    if (DP > 64 || lane < 32) *reinterpret_cast<uint32_t *>(&nan_bits[buf][eight][unit / (DP / 4) & 1][d]) = bits;
                }
            }
        }
    };
    auto place_v = [&](const VCodes &r, int tile) {
        uint8_t *const to_v = lv(tile);
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int eight = wave + NW * u;
#pragma unroll
            for (int c = 0; c < VL; c++) {
                const int unit = lane + 64 * c, d = 4 * (unit % (DP / 4)), quad = unit / (DP / 4) & 1;
                const uint32_t *v = r.w[u][c];
                u32x2 e[4];
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    const uint32_t lo = __builtin_amdgcn_perm(v[2 * i + 1], v[2 * i], 0x05010400u);
                    const uint32_t hi = __builtin_amdgcn_perm(v[2 * i + 1], v[2 * i], 0x07030602u);
                    e[0][i] = T::two_codes(lo, false, r.power[u]), e[1][i] = T::two_codes(lo, true, r.power[u]);
                    e[2][i] = T::two_codes(hi, false, r.power[u]), e[3][i] = T::two_codes(hi, true, r.power[u]);
                }
                if (DP > 64 || lane < 32) {
#pragma unroll
                    for (int i = 0; i < 4; i++) *reinterpret_cast<u32x2 *>(to_v + (d + i) * VP + 16 * chunk_of(d + i, eight) + 8 * quad) = e[i];
                }
            }
        }
    };

    // ---- operands out of LDS: two 32s' scores in turn (neither waits for itself); elements 32d.. of a sixteen's V
    auto k_part = [&](int tile, int i) { return *reinterpret_cast<const u32x4 *>(lk(tile) + (32 * (i % 2) + col) * KP + 32 * (i / 2) + 16 * half); };
    auto v_part = [&](int tile, int i) {
        return *reinterpret_cast<const u32x4 *>(lv(tile) + (32 * (i % ND) + col) * VP + 16 * chunk_of(col, 2 * (i / ND) + half));
    };

    float m = -INFINITY, base = 0.0f, l = 0.0f;
    int ref = 0;                                // outputs are sums in units of 2^ref
    f32x16 o[ND];
#pragma unroll
    for (int d = 0; d < ND; d++)
#pragma unroll
        for (int i = 0; i < 16; i++) o[d][i] = 0.0f;
    // a NaN in V reaches the queries that see it, and no others
    auto give_nans = [&](int tile) {
#pragma unroll 1
        for (int e8 = 0; e8 < 8; e8++) {
            if (nan_tile[tile & 1][e8] != tile + 1) continue;
            uint32_t sees[2] = {0u, 0u};
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (begin + kTile * tile + 16 * (e8 >> 1) + 4 * (e8 & 1) + (i & 3) + 8 * (i >> 2) <= lim) sees[i >> 2] |= 0x01010101u << (i & 3);
#pragma unroll
            for (int d = 0; d < ND; d++)
#pragma unroll
                for (int y = 0; y < 4; y++) {
                    const int e = 32 * d + 8 * y + 4 * half;
                    const uint32_t bits = (*reinterpret_cast<const uint32_t *>(&nan_bits[tile & 1][e8][0][e]) & sees[0]) |
                                          (*reinterpret_cast<const uint32_t *>(&nan_bits[tile & 1][e8][1][e]) & sees[1]);
#pragma unroll
                    for (int i = 0; i < 4; i++) o[d][4 * y + i] += bits >> (8 * i) & 0xFFu ? NAN : 0.0f;
                }
        }
    };
    if (tiles) {
        if (threadIdx.x < 16) nan_tile[threadIdx.x >> 3][threadIdx.x & 7] = nan_any[threadIdx.x & 1] = 0;
        KCodes kc;
        VCodes vc;
        Places now = look(0, [&](const Places &l) { fetch(0, l, kc, vc); }), next = now;
#pragma unroll
        for (int k = 0; k < KK; k++) *reinterpret_cast<u32x4 *>(in_row(k * kRows + lane / kChunks, lane % kChunks)) = qf[k];
        lds_handover();
#pragma unroll
        for (int k = 0; k < KK; k++) qf[k] = *reinterpret_cast<const u32x4 *>(in_row(col, 2 * k + half));
        lds_barrier();                          // (the NaN flags are cleared, and the rows read)
#pragma unroll
        for (int k = 0; k < KK; k++)
#pragma unroll
            for (int i = 0; i < 4; i++) qf[k][i] = 16 * k + 8 * half < (int)a.c.dim ? qf[k][i] ^ flip : 0u;
        now.far = powers(0, now.e, now.far, vc);
        clean_v(vc, 0);
        place_v(vc, 0);
        place_k(kc, 0);
        if constexpr (KIND == kLast) {              // goes on from the sums of what is behind the prefix
            const int64_t part = (int64_t)(q.start + min(w.token, q.fresh - 1)) * a.q_heads + w.head;
            const f32x2 x = p.sums[part];
            const float *const from = p.parts + part * a.c.dim;
            m = row < rows ? x[0] : -INFINITY;
            base = m == -INFINITY ? 0.0f : m;
            l = row < rows && !half ? x[1] : 0.0f;
#pragma unroll
            for (int d = 0; d < ND; d++)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const int e = 32 * d + 2 * i + 4 * half;
                    const f32x4 y = *reinterpret_cast<const f32x4 *>(from + (e < (int)a.c.dim ? e : 0));
#pragma unroll
                    for (int k = 0; k < 4; k++) o[d][i + k] = row < rows ? y[k] : 0.0f;
                }
        }
#pragma unroll 1
        for (int tile = 0; tile < tiles; tile++) {
            const int t0 = begin + kTile * tile;
            if ((tile & 15) == 0 && tile) now = next;
            if (((tile + 1) & 15) == 0) next = look((tile + 1) >> 4, [](const Places &) {});
            fetch(tile + 1, ((tile + 1) & 15) == 0 ? next : now, kc, vc);
            lds_barrier();                      // the tile is in LDS
            if (t0 <= most) {
                const bool nans = nan_any[tile & 1] == tile + 1;
                // Operands are read from LDS well ahead of the instructions that take them, V's first ones while K's last are
                // used (left to itself the compiler reads one or two ahead, and every instruction waits for most of a trip to LDS).
                f32x16 z[2];
                u32x4 kf[A], vf[A];
#pragma unroll
                for (int i = 0; i < A; i++) kf[i] = k_part(tile, i);
#pragma unroll
                for (int s = 0; s < 2; s++)
#pragma unroll
                    for (int i = 0; i < 16; i++) z[s][i] = 0.0f;
#pragma unroll
                for (int i = 0; i < 2 * KK; i++) {
                    z[i % 2] = T::mfma32(kf[i % A], qf[i / 2], z[i % 2]);
                    if (i + A < 2 * KK) kf[i % A] = k_part(tile, i + A);
                    else vf[i + A - 2 * KK] = v_part(tile, i + A - 2 * KK);
                }
                f32x4 ks = *reinterpret_cast<const f32x4 *>(&scales[tile >> 4 & 1][0][4 * (tile & 15)]);
                f32x4 lift = *reinterpret_cast<const f32x4 *>(&scales[tile >> 4 & 1][1][4 * (tile & 15)]);
                f32x4 inv = *reinterpret_cast<const f32x4 *>(&scales[tile >> 4 & 1][2][4 * (tile & 15)]);
                __builtin_amdgcn_sched_group_barrier(0x100, A, 0);
#pragma unroll
                for (int i = 0; i < 2 * KK; i++) {
                    __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                }
                const uint32_t there = (uint32_t)(now.there >> (4 * (tile & 15))) & 15u;
                if (there != 15u || t0 + kTile - 1 > least) {
                    asm volatile("");           // (a branch that most tiles skip, not selects in all of them)
#pragma unroll
                    for (int s = 0; s < 2; s++)
#pragma unroll
                        for (int i = 0; i < 16; i++)
                            z[s][i] = (there >> (2 * s + (i >> 3)) & 1u) && t0 + 32 * s + 8 * (i >> 2) + 4 * half + (i & 3) <= lim ? z[s][i] : -INFINITY;
                }
                // (the middle of three with +inf is the larger of two, and takes products' results without a step to quiet NaNs first)
                float top = -INFINITY;
#pragma unroll
                for (int x = 0; x < 4; x++) {
                    float t = -INFINITY;
#pragma unroll
                    for (int i = 0; i < 8; i++) t = __builtin_amdgcn_fmed3f(t, z[x >> 1][8 * (x & 1) + i], INFINITY);
                    top = fmaxf(top, t * ks[x]);
                }
                if constexpr (T::kNarrow) {
                    if (unit != ref) {          // the sums in the tile's unit
#pragma unroll
                        for (int d = 0; d < ND; d++)
#pragma unroll
                            for (int i = 0; i < 16; i++) o[d][i] = __builtin_ldexpf(o[d][i], ref - unit);
                        ref = unit;
                    }
                }
                if (__ballot(top > m + kSlack)) {       // the sums against a higher maximum
                    const float to = fmaxf(m, fmaxf(top, __shfl_xor(top, 32)));
                    const float f = to == -INFINITY ? 1.0f : exp2_of(m - to);
                    m = to;
                    base = to == -INFINITY ? 0.0f : to;
                    l *= f;
#pragma unroll
                    for (int d = 0; d < ND; d++) o[d] *= f;
                }
                // p, times V's scale between 1 and 2 (in the exponent; what is summed is divided by it again)
                u32x4 pf[4];
#pragma unroll
                for (int x = 0; x < 4; x++) {
                    const float off = lift[x] - base;
                    float e[8], sum[2] = {0.0f, 0.0f};
#pragma unroll
                    for (int i = 0; i < 8; i++) {
                        e[i] = exp2_of(__builtin_fmaf(z[x >> 1][8 * (x & 1) + i], ks[x], off));
                        sum[i & 1] += e[i];
                    }
                    l = __builtin_fmaf(sum[0] + sum[1], inv[x], l);
#pragma unroll
                    for (int i = 0; i < 4; i++) pf[x][i] = T::pack(e[2 * i], e[2 * i + 1]);
                }
#pragma unroll
                for (int i = 0; i < 4 * ND; i++) {
                    o[i % ND] = T::mfma32(vf[i % A], pf[i / ND], o[i % ND]);
                    if (i + A < 4 * ND) vf[i % A] = v_part(tile, i + A);
                }
                if (nans) give_nans(tile);
            }
            const bool other = ((tile + 1) & 15) == 0;          // (a batch is not looked at again behind its last tile)
            now.far = powers(tile + 1, other ? next.e : now.e, other ? next.far : now.far, vc);
            if (other) next.far = now.far;
            clean_v(vc, tile + 1);
            place_v(vc, tile + 1);
            place_k(kc, tile + 1);
        }
    }

    // Rows of requests that share nothing are joined elsewhere, and rows of no request are none.  (No return for them: without a way around
    // the loop the compiler runs out of registers.)
    [[maybe_unused]] uint32_t written_rows = 0;
    if constexpr (KIND == kLast) {
        bool shares = tiles > 0 && row < rows;
        if (shares) {
            const int token = q.start + w.token;
            int r = token;
            if (a.b.starts) {                   // the last request whose rows begin at or in front of it
                r = 0;
                for (int n = (int)a.b.n_reqs; n > 1;) {
                    const int step = n >> 1;
                    if (a.b.starts[r + step] <= token) r += step, n -= step;
                    else n = step;
                }
            }
            const Request of = request_of(a.b, a.c, r);
            shares = token >= of.start && token < of.start + of.fresh && of.len - of.fresh >= q.len;
        }
        written_rows = (uint32_t)__ballot(shares);
    }
    l += __shfl_xor(l, 32);
    const int64_t at = (int64_t)(q.start + w.token) * a.q_heads + w.head;
    const bool empty = m == -INFINITY && l == 0.0f;
    if (KIND == kLast || KIND == kThrough || (KIND == kWhole && p.splits == 1)) {
        // Rows are put together in LDS, so that a store writes whole ones: as the lanes hold them it would write 16 bytes here and there.
        const float f = __builtin_ldexpf(empty ? 0.0f : 1.0f / l, ref);
        const int64_t dst = (int64_t)(q.start + w.token) * a.out.row_stride + (int64_t)w.head * a.out.head_stride;
        lds_barrier();                          // (the tiles are done with)
#pragma unroll
        for (int d = 0; d < ND; d++)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                *reinterpret_cast<u32x2 *>(in_row(col, 4 * d + i / 4) + 8 * half) =
                    u32x2{T::pack(o[d][i] * f, o[d][i + 1] * f), T::pack(o[d][i + 2] * f, o[d][i + 3] * f)};
        lds_handover();
#pragma unroll
        for (int j = 0; j < 32; j += kRows) {
            const int r = j + lane / kChunks, chunk = lane % kChunks;
            const u32x4 x = *reinterpret_cast<const u32x4 *>(in_row(r, chunk));
            const int64_t to = (int64_t)(uint32_t)__shfl((int)(uint32_t)dst, r) | (int64_t)__shfl((int)(dst >> 32), r) << 32;
            if ((KIND == kLast ? (bool)(written_rows >> r & 1u) : wave_row + r < rows) && 8 * chunk < (int)a.c.dim)
                *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(a.out.data) + to + 8 * chunk) = x;
        }
        if ((KIND == kLast ? (bool)(written_rows >> col & 1u) : row < rows) && half == 0) {
            const float sum = empty ? -INFINITY : m + log2_of(l);
            if (a.lse) a.lse[at] = sum * kLn2;
            if (p.totals) p.totals[at] = sum;
        }
    } else {
        const float unit = power_of(ref);
        if (row < rows && half == 0) p.sums[at * p.splits + split] = f32x2{m, l};
        const int64_t part = at * p.splits + split;
        lds_barrier();                          // (the tiles are done with)
#pragma unroll
        for (int h = 0; h < 2; h++) {           // halves of a row in fp32
#pragma unroll
            for (int d = 0; d < ND / 2; d++)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const f32x16 &x = o[h * (ND / 2) + d];
                    *reinterpret_cast<f32x4 *>(in_row(col, 8 * d + i / 2 + half)) = f32x4{x[i], x[i + 1], x[i + 2], x[i + 3]} * unit;
                }
            lds_handover();
#pragma unroll
            for (int j = 0; j < 32; j += kRows) {
                const int r = j + lane / kChunks, e = h * (DP / 2) + 4 * (lane % kChunks);
                const f32x4 x = *reinterpret_cast<const f32x4 *>(in_row(r, lane % kChunks));
                const int64_t to = (int64_t)(uint32_t)__shfl((int)(uint32_t)part, r) | (int64_t)__shfl((int)(part >> 32), r) << 32;
                if (wave_row + r < rows && e < (int)a.c.dim) *reinterpret_cast<f32x4 *>(p.parts + to * a.c.dim + e) = x;
            }
            lds_handover();
        }
    }
}

// Outputs out of the parts that splits of the contexts left: a row by as many lanes as take four elements each of it, in one pass with
// the running maximum (and then another row, where a request has more than a launch has workgroups for).  Bound by memory and its
// latency: 48000 rows of 128 elements out of six parts, 150 MB, 25 us.
template <typename T>
__global__ __launch_bounds__(256) void join_parts_kernel(AttendArgs a, PartsPlan p, uint32_t tile_rows)
{
    const Request q = request_of(a.b, a.c, (int)blockIdx.y);
    const uint32_t wide = a.c.dim / 4u, each = 256u / wide, rows = (uint32_t)q.fresh * a.group, lane = threadIdx.x % wide;
    if (threadIdx.x >= each * wide) return;
    for (uint32_t n = blockIdx.x * each + threadIdx.x / wide; n < rows * a.c.heads; n += gridDim.x * each) {
        const uint32_t head = n / rows, row = n - head * rows;
        const QueryRow w = query_row(a, head, row);
        const int64_t at = (int64_t)(q.start + w.token) * a.q_heads + w.head;
        // splits that the row's workgroup had work in
        const uint32_t last_row = min((row / tile_rows + 1u) * tile_rows, rows) - 1u;
        const int seen = q.len - q.fresh + (int)(last_row / a.group) + 1, splits = max(1, (seen + (int)p.chunk - 1) / (int)p.chunk);
        const f32x2 *sums = p.sums + at * p.splits;
        const float *parts = p.parts + at * p.splits * a.c.dim + 4u * lane;
        float m = -INFINITY, l = 0.0f;
        f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
        for (int s = 0; s < splits; s++) {
            const f32x2 x = sums[s];
            const f32x4 part = *reinterpret_cast<const f32x4 *>(parts + (int64_t)s * a.c.dim);
            const float top = fmaxf(m, x[0]), to = top == -INFINITY ? 0.0f : top, f = exp2_of(m - to), g = exp2_of(x[0] - to);
            l = l * f + x[1] * g;
            o = o * f + part * g;
            m = top;
        }
        const bool empty = m == -INFINITY && l == 0.0f;
        o *= empty ? 0.0f : 1.0f / l;
        uint16_t *dst = static_cast<uint16_t *>(a.out.data) + (int64_t)(q.start + w.token) * a.out.row_stride + (int64_t)w.head * a.out.head_stride + 4u * lane;
        *reinterpret_cast<u32x2 *>(dst) = u32x2{T::pack(o[0], o[1]), T::pack(o[2], o[3])};
        if (!lane) {
            const float total = empty ? -INFINITY : m + log2_of(l);
            if (a.lse) a.lse[at] = total * kLn2;
            if (p.totals) p.totals[at] = total;
        }
    }
}

// A product's N matrix instructions and 48 vector ones in turn
template <int N> __device__ __forceinline__ void interleave()
{
#pragma unroll
    for (int k = 0; k < N; k++) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x402, 48 / N, 0);
    }
}

// Weights: 256 tokens a workgroup, 64 a wavefront, whose K stays in registers; the query rows that see them pass through LDS 64 at
// a time (32 of 256 elements).  Scores once more (their rows' totals were not known before), p summed over the rows in fp32, in an
// order that timing does not change.  A row of queries is a column of the product: a lane adds up its column's rows in turn, and lanes
// are joined once at the end.  Half of attention's operations, and an exp2 for each score: bound by the vector instructions (three a
// score, exp2 at half rate) that run between the matrix ones: four long prompts' parts, 343 million scores, 88 GFLOP in 104 to 110 us by card (172 us
// with 32 rows a step and nothing read ahead, 130 with the two one after the other, 121 with 160 lane exchanges at the end).
template <typename T, int DP>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(DP <= 128 ? 2 : 1))) void weights_kernel(AttendArgs a, PartsPlan p)
{
    constexpr int QP = DP * 2 + 16, KK = DP / 16, QT = DP <= 128 ? 64 : 32;
    constexpr int TR = 256 / QT, QL = DP / (8 * TR);            // threads a query row, loads of 8 elements each of them
    __shared__ __align__(16) uint8_t lq[2][QT * QP];
    __shared__ float lt[2][QT];
    __shared__ int ll[2][QT];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
    const uint32_t head = blockIdx.x % a.c.heads;
    const Request q = request_of(a.b, a.c, (int)blockIdx.y);
    const int block0 = (int)(blockIdx.x / a.c.heads) * 256, t0 = block0 + 64 * wave;
    if (block0 >= q.len) return;
    const int older = q.len - q.fresh, rows = q.fresh * (int)a.group;
    const int first_row = max(0, block0 - older) * (int)a.group, tiles = (rows - first_row + QT - 1) / QT;

    u32x4 rq[QL];
    float rt = -INFINITY;
    int rl = -1;
    const int per_token = (int)a.group, step_token = QT / per_token, step_head = QT - step_token * per_token;
    int next = first_row + (int)(threadIdx.x / TR), token = next / per_token, head_of = next - token * per_token;
    auto fetch = [&]() {                        // of the rows that follow
        const int at = min(token, q.fresh - 1);
        const uint32_t q_head = head * a.group + (uint32_t)head_of;
        const uint16_t *src = static_cast<const uint16_t *>(a.q.data) + (int64_t)(q.start + at) * a.q.row_stride + (int64_t)q_head * a.q.head_stride;
#pragma unroll
        for (int c = 0; c < QL; c++) {
            const int d = 8 * TR * c + 8 * (int)(threadIdx.x % TR);
            rq[c] = *reinterpret_cast<const u32x4 *>(src + (d < (int)a.c.dim ? d : 0));
        }
        rt = p.totals[(int64_t)(q.start + at) * a.q_heads + q_head];
        rl = token < q.fresh ? older + token : -1;
        token += step_token, head_of += step_head;
        if (head_of >= per_token) head_of -= per_token, token++;
    };
    auto place = [&](int buf) {
        if ((int)a.c.dim < DP) {
#pragma unroll
            for (int c = 0; c < QL; c++)
#pragma unroll
                for (int i = 0; i < 4; i++) rq[c][i] = 8 * TR * c + 8 * (int)(threadIdx.x % TR) < (int)a.c.dim ? rq[c][i] : 0u;
        }
#pragma unroll
        for (int c = 0; c < QL; c++)
            *reinterpret_cast<u32x4 *>(lq[buf] + (threadIdx.x / TR) * QP + 16 * TR * c + 16 * (threadIdx.x % TR)) = rq[c];
        if ((threadIdx.x % TR) == 0) {          // a row that saw nothing, or is none, weighs nothing
            lt[buf][threadIdx.x / TR] = rt == -INFINITY || rl < 0 ? INFINITY : rt;
            ll[buf][threadIdx.x / TR] = rl;
        }
    };
    if (tiles > 0) fetch();

    // K of the wavefront's tokens: two 32s, their sixteens' scales
    const Look l = look_up(a, q, head, t0 + 16 * lane, lane < 4 ? q.len : 0, a.scale_log2);
    u32x4 kf[2][KK];
    float ks[4];
#pragma unroll
    for (int x = 0; x < 4; x++) ks[x] = lane_value(l.ks, x);
#pragma unroll
    for (int s = 0; s < 2; s++) {
        const int t = t0 + 32 * s + col, e0 = __builtin_amdgcn_readlane(l.entry, 2 * s), e1 = __builtin_amdgcn_readlane(l.entry, 2 * s + 1);
        const int e = col < 16 ? e0 : e1;
        const uint32_t b = block_of(a.c, (uint32_t)t >> 4);
        const uint8_t *k = code_at(a.c, 0, max(e, 0), (uint32_t)t - b * a.c.bs, head);
        u32x2 w[KK];
#pragma unroll
        for (int i = 0; i < KK; i++) w[i] = *reinterpret_cast<const u32x2 *>(k + (16 * i + 8 * half < (int)a.c.dim ? 16 * i + 8 * half : 0));
#pragma unroll
        for (int i = 0; i < KK; i++) kf[s][i] = u32x4{T::two_codes(w[i][0], false), T::two_codes(w[i][0], true), T::two_codes(w[i][1], false), T::two_codes(w[i][1], true)};
    }

    float w[2][16];
#pragma unroll
    for (int s = 0; s < 2; s++)
#pragma unroll
        for (int i = 0; i < 16; i++) w[s][i] = 0.0f;
    if (tiles > 0) place(0);
    constexpr int A = DP <= 128 ? (KK < 8 ? KK : 8) : 4;          // operands read ahead
    auto operand = [&](int buf, int h, int k) { return *reinterpret_cast<const u32x4 *>(lq[buf] + (32 * h + col) * QP + 16 * half + 32 * k); };
    // rows that do not see all of the workgroup's tokens (those behind the context are not written)
    const int seen = max(0, min(block0 + 255, q.len - 1) - older) * per_token - first_row;      // rows in front of the first that does
    const int masked = min(tiles, (max(seen, 0) + QT - 1) / QT);
#pragma unroll 1
    for (int tile = 0; tile < masked; tile++) {
        const int buf = tile & 1;
        if (tile + 1 < tiles) fetch();
        lds_barrier();
#pragma unroll 1
        for (int h = 0; h < QT / 32; h++) {
            u32x4 f[A];
#pragma unroll
            for (int k = 0; k < A; k++) f[k] = operand(buf, h, k);
            const float total = lt[buf][32 * h + col];
            const int lim = ll[buf][32 * h + col];
            f32x16 z[2];
#pragma unroll
            for (int s = 0; s < 2; s++)
#pragma unroll
                for (int i = 0; i < 16; i++) z[s][i] = 0.0f;
#pragma unroll
            for (int k = 0; k < KK; k++) {
#pragma unroll
                for (int s = 0; s < 2; s++) z[s] = T::mfma32(kf[s][k], f[k % A], z[s]);
                if (k + A < KK) f[k % A] = operand(buf, h, k + A);
            }
#pragma unroll
            for (int s = 0; s < 2; s++)
#pragma unroll
                for (int i = 0; i < 16; i++) {
                    const float e = exp2_of(z[s][i] * ks[2 * s + (i >> 3)] - total);
                    w[s][i] += t0 + 32 * s + 8 * (i >> 2) + 4 * half + (i & 3) <= lim ? e : 0.0f;
                }
        }
        if (tile + 1 < tiles) place(buf ^ 1);
    }
    // The others: one 32 of tokens is weighed while the products of the other run.
    if (masked < tiles) {
        int buf = masked & 1, h = 0;
        if (masked + 1 < tiles) fetch();
        lds_barrier();
        u32x4 f[KK];
#pragma unroll
        for (int k = 0; k < KK; k++) f[k] = operand(buf, 0, k);
        float total = lt[buf][col];
        f32x16 z0, z1;
        auto zero = [](f32x16 &z) {
#pragma unroll
            for (int i = 0; i < 16; i++) z[i] = 0.0f;
        };
        zero(z0);
#pragma unroll
        for (int k = 0; k < KK; k++) z0 = T::mfma32(kf[0][k], f[k], z0);
        int left = tiles - masked - 1;          // tiles behind this one
#pragma unroll 1
        for (int n = (left + 1) * (QT / 32) - 1; n > 0; n--) {
            if (++h == QT / 32) {
                place(buf ^ 1);
                lds_barrier();
                if (left > 1) fetch();
                left--, buf ^= 1, h = 0;
            }
            const float next_total = lt[buf][32 * h + col];
            zero(z1);
#pragma unroll
            for (int k = 0; k < KK; k++) {
                z1 = T::mfma32(kf[1][k], f[k], z1);
                f[k] = operand(buf, h, k);
            }
#pragma unroll
            for (int i = 0; i < 16; i++) w[0][i] += exp2_of(__builtin_fmaf(z0[i], ks[i >> 3], -total));
            interleave<KK>();
            zero(z0);
#pragma unroll
            for (int k = 0; k < KK; k++) z0 = T::mfma32(kf[0][k], f[k], z0);
#pragma unroll
            for (int i = 0; i < 16; i++) w[1][i] += exp2_of(__builtin_fmaf(z1[i], ks[2 + (i >> 3)], -total));
            interleave<KK>();
            total = next_total;
        }
        zero(z1);
#pragma unroll
        for (int k = 0; k < KK; k++) z1 = T::mfma32(kf[1][k], f[k], z1);
#pragma unroll
        for (int i = 0; i < 16; i++) {
            w[0][i] += exp2_of(__builtin_fmaf(z0[i], ks[i >> 3], -total));
            w[1][i] += exp2_of(__builtin_fmaf(z1[i], ks[2 + (i >> 3)], -total));
        }
    }
#pragma unroll
    for (int s = 0; s < 2; s++) {
        halve<16, 8>(w[s], col);
        halve<8, 4>(w[s], col);
        halve<4, 2>(w[s], col);
        halve<2, 1>(w[s], col);
        float x = w[s][0] + __shfl_xor(w[s][0], 1);
        const int i = col >> 1, t = t0 + 32 * s + 8 * (i >> 2) + 4 * half + (i & 3);
        const int e0 = __builtin_amdgcn_readlane(l.entry, 2 * s), e1 = __builtin_amdgcn_readlane(l.entry, 2 * s + 1);
        if ((i >> 3 ? e1 : e0) < 0) x = 0.0f;
        if (!(col & 1) && t < q.len) {
            if (a.prior.data && t < older)
                x += a.decay * a.prior.data[(int64_t)q.row * a.prior.row_stride + (int64_t)head * a.prior.head_stride + t];
            a.w.data[(int64_t)q.row * a.w.row_stride + (int64_t)head * a.w.head_stride + t] = x;
        }
    }
}

// Workgroups of a launch, of `waves` wavefronts each, and how they find their rows (p.counted, p.spread)
static uint64_t groups_of(const AttendArgs &a, PartsPlan &p, Kind kind, uint32_t waves)
{
    // Row tiles of an XCD at most: as many as the longest request makes, for each pair; as many as all rows make, and one for each request.
    // Where the second is less the kernel counts for itself: a workgroup that finds nothing to do has waited for a compute unit of its own.
    // Measured (us, first / second): one prompt of 8192 tokens among 63 single ones 2163 / 1387, one of 512 among 255 1031 / 284, 32 ragged
    // prompts 609 / 603; where all requests are alike counting costs some 0.7 us for every 64 of them, and is not done.
    const uint64_t units = kind == kPrefix || kind == kLast ? a.n_groups : a.b.n_reqs;
    const uint64_t by_pairs = (units * a.c.heads + 7u) / 8u * p.row_tiles;
    const uint64_t by_rows = ((uint64_t)a.b.total_new * a.group / (32u * waves) + units) * ((a.c.heads + 7u) / 8u);
    // Few pairs, of a group and a head or of a request, that eight do not divide: XCDs without any, or with one more than others; their row tiles
    // go to the XCDs in turn.  (Us, by pairs / so; requests x tokens,
    // heads, query heads each, prefixes: 59 x 370, 1 x 256, 1, one of 7000 2057 / 359; 85 x 174, 1 x 128, 2, three of 8000 460 / 151; 32 x 300, 4 x 128, 4, one
    // of 4000 844 / 491; 64 x 32, 12 x 128, 4, one of 4000 376 / 304; 32 x 100, 10 x 128, 4, six 461 / 458.)
    const uint64_t pairs = units * a.c.heads;
    p.spread = kind != kWhole && pairs % 8u && pairs < 64u;
    p.counted = p.spread || by_pairs > by_rows;
    const uint64_t all = std::min(((uint64_t)a.b.total_new * a.group / (32u * waves) + units) * a.c.heads, pairs * p.row_tiles);
    return (p.spread ? (all + 7u) / 8u : p.counted ? by_rows : by_pairs) * p.splits * 8u;
}
static uint32_t parts_waves(const AttendArgs &a) { return a.c.dim <= 128u ? 8u : 4u; }
static bool parts_fit(const AttendArgs &a, PartsPlan p, Kind kind) { return launchable(groups_of(a, p, kind, parts_waves(a)), 64u * parts_waves(a)); }

template <typename T, int DP, int NW, Kind KIND> static hipError_t parts(const AttendArgs &a, PartsPlan p, hipStream_t s)
{
    const uint64_t groups = groups_of(a, p, KIND, NW);
    const uint64_t weight_groups = a.w.data ? (a.b.max_len + 255ull) / 256u * a.c.heads : 0u;
    if (!launchable(groups, 64u * NW) || !launchable(weight_groups, 256)) return hipErrorInvalidConfiguration;
    parts_kernel<T, DP, NW, KIND><<<(uint32_t)groups, 64 * NW, 0, s>>>(a, p);
    hipError_t e = hipGetLastError();
    if constexpr (KIND != kWhole) return e;
    if (e == hipSuccess && p.splits > 1u) {
        const uint32_t each = 256u / (a.c.dim / 4u);
        join_parts_kernel<T><<<dim3(std::min((a.b.max_new * a.q_heads + each - 1u) / each, 1u << 20), a.b.n_reqs), 256, 0, s>>>(a, p, 32u * NW);
        e = hipGetLastError();
    }
    if (e == hipSuccess && weight_groups) {
        weights_kernel<T, DP><<<dim3((uint32_t)weight_groups, a.b.n_reqs), 256, 0, s>>>(a, p);
        e = hipGetLastError();
    }
    return e;
}

template <typename T, Kind KIND> static hipError_t parts_of(const AttendArgs &a, const PartsPlan &p, hipStream_t s)
{
    return a.c.dim <= 64 ? parts<T, 64, 8, KIND>(a, p, s) : a.c.dim <= 128 ? parts<T, 128, 8, KIND>(a, p, s) : parts<T, 256, 4, KIND>(a, p, s);
}

hipError_t launch_parts(const AttendArgs &a, const PartsPlan &p, uint32_t dtype, hipStream_t s)
{
    return dtype == DMI_DTYPE_BF16 ? parts_of<Bf16, kWhole>(a, p, s) : parts_of<Fp16, kWhole>(a, p, s);
}

hipError_t launch_parts_apart(const AttendArgs &a, const PartsPlan &p, Kind kind, uint32_t dtype, hipStream_t s)
{
    if (kind == kLast) return dtype == DMI_DTYPE_BF16 ? parts_of<Bf16, kLast>(a, p, s) : parts_of<Fp16, kLast>(a, p, s);
    if (kind == kThrough) return dtype == DMI_DTYPE_BF16 ? parts_of<Bf16, kThrough>(a, p, s) : parts_of<Fp16, kThrough>(a, p, s);
    if (kind == kPrefix) return dtype == DMI_DTYPE_BF16 ? parts_of<Bf16, kPrefix>(a, p, s) : parts_of<Fp16, kPrefix>(a, p, s);
    return dtype == DMI_DTYPE_BF16 ? parts_of<Bf16, kRest>(a, p, s) : parts_of<Fp16, kRest>(a, p, s);
}

// ---------------------------------------------------------------- contexts behind shared prefixes
// Prefixes that groups share: 32 prompts, 8516 tokens of 32 query heads behind one of 4000, 581 GFLOP, read by each (kThrough) 670 to 770 us by card;
// read once 700 (kLast), and 88 for their own tokens in front.  64 single tokens behind 8192, 256 rows a head in 26 splits 22 us: 5 until the first
// tile, 2.4 each of five, 7 to write 27 MB of parts.
//
// Outputs out of the parts of prefixes and of what is behind them (p.last: of requests that share nothing, the others' are written already):
// see join_parts_kernel.
template <typename T>
__global__ __launch_bounds__(256) void join_shared_kernel(AttendArgs a, SharedPlan p)
{
    const Request q = request_of(a.b, a.c, (int)blockIdx.y);
    const uint32_t wide = a.c.dim / 4u, each = 256u / wide, rows = (uint32_t)q.fresh * a.group, lane = threadIdx.x % wide;
    const int shared = shared_tokens(a, (int)blockIdx.y, q);
    if (p.last && shared) return;
    if (threadIdx.x >= each * wide) return;
    const int before = p.few_rows ? (shared ? (int)p.prefix.splits : 0) : p.prefix.chunk ? min((shared + (int)p.prefix.chunk - 1) / (int)p.prefix.chunk, (int)p.prefix.splits) : 0;
    for (uint32_t n = blockIdx.x * each + threadIdx.x / wide; n < rows * a.c.heads; n += gridDim.x * each) {
        const uint32_t head = n / rows, row = n - head * rows;
        const QueryRow w = query_row(a, head, row);
        const int64_t at = (int64_t)(q.start + w.token) * a.q_heads + w.head;
        float m = -INFINITY, l = 0.0f;
        f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
        auto add = [&](const f32x2 *sums, const float *parts, int count) {
            parts += 4u * lane;
#pragma unroll 4
            for (int s = 0; s < count; s++) {
                const f32x2 x = sums[s];
                const f32x4 part = *reinterpret_cast<const f32x4 *>(parts + (int64_t)s * a.c.dim);
                const float top = fmaxf(m, x[0]), to = top == -INFINITY ? 0.0f : top, f = exp2_of(m - to), g = exp2_of(x[0] - to);
                l = l * f + x[1] * g;
                o = o * f + part * g;
                m = top;
            }
        };
        add(p.prefix.sums + at * p.prefix.splits, p.prefix.parts + at * p.prefix.splits * a.c.dim, before);
        int behind = (int)p.splits;
        if (!p.tokens) {                        // splits that the row's workgroup had work in, as in join_parts_kernel
            const uint32_t tile_rows = a.c.dim <= 128u ? 256u : 128u, last_row = min((row / tile_rows + 1u) * tile_rows, rows) - 1u;
            behind = max(1, (q.len - shared - q.fresh + (int)(last_row / a.group) + (int)p.many.chunk) / (int)p.many.chunk);
        }
        add(p.sums + at * p.splits, p.parts + at * p.splits * a.c.dim, behind);
        const bool empty = m == -INFINITY && l == 0.0f;
        o *= empty ? 0.0f : 1.0f / l;
        uint16_t *dst = static_cast<uint16_t *>(a.out.data) + (int64_t)(q.start + w.token) * a.out.row_stride + (int64_t)w.head * a.out.head_stride + 4u * lane;
        *reinterpret_cast<u32x2 *>(dst) = u32x2{T::pack(o[0], o[1]), T::pack(o[2], o[3])};
        if (!lane && a.lse) a.lse[at] = empty ? -INFINITY : (m + log2_of(l)) * kLn2;
    }
}

hipError_t launch_shared(const AttendArgs &a, const SharedPlan &p, uint32_t dtype, hipStream_t s)
{
    const Kind rest = p.tokens || !p.through ? kRest : kThrough;
    const bool first = a.n_groups && !p.last && !p.through;
    if ((first && !(p.few_rows ? tokens_apart_fit(a, p.prefix_few, kPrefix) : parts_fit(a, p.prefix, kPrefix))) ||
        !(p.tokens ? tokens_apart_fit(a, p.few, kRest) : parts_fit(a, p.many, rest)) || (p.last && !parts_fit(a, p.prefix, kLast)))
        return hipErrorInvalidConfiguration;
    hipError_t e = hipSuccess;
    if (first) {
        e = p.few_rows ? launch_tokens_apart(a, p.prefix_few, kPrefix, dtype, s) : launch_parts_apart(a, p.prefix, kPrefix, dtype, s);
        if (e != hipSuccess) return e;
    }
    e = p.tokens ? launch_tokens_apart(a, p.few, kRest, dtype, s) : launch_parts_apart(a, p.many, rest, dtype, s);
    if (e != hipSuccess) return e;
    if (p.through || (p.tokens && p.few.before)) return hipSuccess;
    if (p.last) {
        PartsPlan prefix = p.prefix;
        prefix.sums = p.sums, prefix.parts = p.parts;
        if ((e = launch_parts_apart(a, prefix, kLast, dtype, s)) != hipSuccess) return e;
    }
    const uint32_t each = 256u / (a.c.dim / 4u);
    const dim3 grid(std::min((a.b.max_new * a.q_heads + each - 1u) / each, p.last ? 64u : 1u << 20), a.b.n_reqs);
    if (dtype == DMI_DTYPE_BF16) join_shared_kernel<Bf16><<<grid, 256, 0, s>>>(a, p);
    else join_shared_kernel<Fp16><<<grid, 256, 0, s>>>(a, p);
    return hipGetLastError();
}

}  // namespace kv8
}  // namespace dmi
