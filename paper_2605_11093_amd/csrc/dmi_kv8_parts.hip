// Attention of many query rows over the 8-bit KV cache: prompts and parts of prompts.
#include "dmi_internal.h"
#include "dmi_kv8_mfma.h"

namespace dmi {
namespace kv8 {

constexpr int kTile = 64;                       // tokens that a workgroup has in LDS at a time

// What is looked up of sixteens of tokens, one a lane: entry of the block table, scales.
struct Look {
    int entry;
    float ks, vs;
};
__device__ __forceinline__ Look look_up(const AttendArgs &a, const Request &q, uint32_t head, int t, int end)
{
    Look l{-1, 0.0f, 0.0f};
    if (t < end) {
        l.entry = entry_of(a.c, q.row, block_of(a.c, (uint32_t)t >> 4));
        if (l.entry >= 0) {
            l.ks = *scale_at(a.c, 0, l.entry, head);
            l.vs = *scale_at(a.c, 1, l.entry, head);
        }
    }
    return l;
}
__device__ __forceinline__ float lane_value(float v, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane)); }

// As in tokens_kernel, S^T = K Q^T and O^T = V^T P^T with query rows as columns, here with 32x32x16 instructions, 32 * NQ query
// rows a wavefront, four wavefronts on the same tokens.  K and V are converted once for the workgroup, on their way into LDS: K as
// it lies, V transposed, the tokens of a sixteen in the order in which the lanes' registers of S^T hold them (0-3, 8-11 for
// lanes 0-31, 4-7, 12-15 for lanes 32-63), so that an operand is 16 bytes in a row.
template <typename T, int DP, int NQ>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1)))
void parts_kernel(AttendArgs a, PartsPlan p)
{
    constexpr int KP = DP * 2 + 16, VP = kTile * 2 + 16;        // bytes of a row in LDS, padded so that rows start on other banks
    constexpr int KK = DP / 16, ND = DP / 32;
    constexpr int KL = DP / 64;                                 // 16-byte loads of K a thread
    constexpr int VU = (DP / 2 + 63) / 64;                      // units of 8 tokens x 4 elements a thread
    __shared__ __align__(16) uint8_t lds[2 * (kTile * KP + DP * VP)];
    __shared__ int nan_tile[2];                                 // the last tile in either half with a NaN in V, counted from 1
    auto lk = [&](int buf) { return lds + buf * kTile * KP; };
    auto lv = [&](int buf) { return lds + 2 * kTile * KP + buf * DP * VP; };

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
    // the row tiles of a request and head on one XCD, those that see most first
    const uint32_t seq = blockIdx.x >> 3, pair = seq / (p.row_tiles * p.splits) * 8u + (blockIdx.x & 7u), in = seq % (p.row_tiles * p.splits);
    if (pair >= a.b.n_reqs * a.c.heads) return;
    const uint32_t head = pair % a.c.heads, split = in % p.splits, row_tile = p.row_tiles - 1u - in / p.splits;
    const Request q = request_of(a.b, a.c, (int)(pair / a.c.heads));
    const int rows = q.fresh * (int)a.group, row0 = (int)row_tile * 128 * NQ;
    if (row0 >= rows) return;
    const int older = q.len - q.fresh, last_row = min(row0 + 128 * NQ, rows) - 1;
    const int seen = older + last_row / (int)a.group + 1;       // tokens that the workgroup's last row sees
    const int begin = (int)(split * p.chunk), end = min(seen, begin + (int)p.chunk), tiles = max(0, (end - begin + kTile - 1) / kTile);
    if (split && tiles == 0) return;                            // (what reads the parts counts the same way)

    // the wavefront's query rows; a negative scale goes into their sign
    u32x4 qf[NQ][KK];
    int lim[NQ];
    const uint32_t flip = a.scale_log2 < 0.0f ? 0x80008000u : 0u;
    const float scale = fabsf(a.scale_log2);
    const int wave_row = row0 + wave * 32 * NQ;
#pragma unroll
    for (int n = 0; n < NQ; n++) {
        const int row = wave_row + 32 * n + col;
        const QueryRow w = query_row(a, head, (uint32_t)row);
        lim[n] = row < rows ? older + w.token : -1;
        const uint16_t *src = static_cast<const uint16_t *>(a.q.data) + (int64_t)(q.start + w.token) * a.q.row_stride + (int64_t)w.head * a.q.head_stride;
#pragma unroll
        for (int k = 0; k < KK; k++) {
            const int d = 16 * k + 8 * half;
            qf[n][k] = u32x4{0u, 0u, 0u, 0u};
            if (row < rows && d < (int)a.c.dim) {
                qf[n][k] = *reinterpret_cast<const u32x4 *>(src + d);
#pragma unroll
                for (int i = 0; i < 4; i++) qf[n][k][i] ^= flip;
            }
        }
    }
    // what the first and the last of them see
    const int least = wave_row < rows ? older + wave_row / (int)a.group : -1;
    const int most = wave_row < rows ? older + min(wave_row + 32 * NQ - 1, rows - 1) / (int)a.group : -1;
    const bool ragged = wave_row + 32 * NQ > rows;              // (columns past the rows see nothing)

    // A wavefront stages a sixteen of the tile's four.
    u32x4 rk[KL];
    uint32_t rv[VU][8];
    Look here{-1, 0.0f, 0.0f}, stage{-1, 0.0f, 0.0f};
    auto fetch = [&](int tile) {
        const int t = begin + kTile * tile + 16 * wave, six = (4 * tile + wave) & 63;
        const int entry = __builtin_amdgcn_readlane(stage.entry, six);
        const int64_t at = (int64_t)max(entry, 0) * a.c.block_stride +
                           (int64_t)((uint32_t)t - block_of(a.c, (uint32_t)t >> 4) * a.c.bs) * a.c.slot_stride + (int64_t)head * a.c.head_stride;
        const Buffer k = buffer_at(a.c.code[0] + at), v = buffer_at(a.c.code[1] + at);
        const int there = entry < 0 ? 0 : min(16, end - t);
#pragma unroll
        for (int c = 0; c < KL; c++) {
            const uint32_t d = 64u * c + 16u * (lane & 3);
            rk[c] = load_b128<0>(k, (uint32_t)(lane >> 2) * (uint32_t)a.c.slot_stride + (d < a.c.dim ? d : 0u));
        }
#pragma unroll
        for (int u = 0; u < VU; u++) {
            const int unit = lane + 64 * u, h = unit / (DP / 4) & 1, d = 4 * (unit % (DP / 4));
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const int token = 4 * h + (i & 3) + 8 * (i >> 2);
                rv[u][i] = load_b32<0>(v, (uint32_t)token * (uint32_t)a.c.slot_stride + (d < (int)a.c.dim ? (uint32_t)d : 0u));
                rv[u][i] = token < there ? rv[u][i] : 0u;
            }
        }
    };
    auto place = [&](int tile) {
        const int buf = tile & 1;
#pragma unroll
        for (int c = 0; c < KL; c++) {
            uint8_t *to = lk(buf) + (16 * wave + (lane >> 2)) * KP + 2 * (64 * c + 16 * (lane & 3));
            const u32x4 lo = {T::two_codes(rk[c][0], false), T::two_codes(rk[c][0], true), T::two_codes(rk[c][1], false), T::two_codes(rk[c][1], true)};
            const u32x4 hi = {T::two_codes(rk[c][2], false), T::two_codes(rk[c][2], true), T::two_codes(rk[c][3], false), T::two_codes(rk[c][3], true)};
            *reinterpret_cast<u32x4 *>(to) = lo;
            *reinterpret_cast<u32x4 *>(to + 16) = hi;
        }
        uint32_t any = 0;
#pragma unroll
        for (int u = 0; u < VU; u++) {
            const int unit = lane + 64 * u, h = unit / (DP / 4) & 1, d = 4 * (unit % (DP / 4));
            if (unit < DP / 2) {
                u32x4 e[4];
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    any |= nan_codes(rv[u][2 * i]) | nan_codes(rv[u][2 * i + 1]);
                    const uint32_t lo = __builtin_amdgcn_perm(rv[u][2 * i + 1], rv[u][2 * i], 0x05010400u);
                    const uint32_t hi = __builtin_amdgcn_perm(rv[u][2 * i + 1], rv[u][2 * i], 0x07030602u);
                    e[0][i] = T::two_codes(lo, false), e[1][i] = T::two_codes(lo, true);
                    e[2][i] = T::two_codes(hi, false), e[3][i] = T::two_codes(hi, true);
                }
#pragma unroll
                for (int i = 0; i < 4; i++) *reinterpret_cast<u32x4 *>(lv(buf) + (d + i) * VP + 32 * wave + 16 * h) = e[i];
            }
        }
        if (__ballot(any != 0) && lane == 0) nan_tile[buf] = tile + 1;
    };

    float m[NQ], base[NQ], l[NQ], v_ref = T::kNarrow ? 0.0f : 1.0f;
    f32x16 o[NQ][ND];
#pragma unroll
    for (int n = 0; n < NQ; n++) {
        m[n] = -INFINITY, base[n] = 0.0f, l[n] = 0.0f;
#pragma unroll
        for (int d = 0; d < ND; d++)
#pragma unroll
            for (int i = 0; i < 16; i++) o[n][d][i] = 0.0f;
    }

    if (threadIdx.x < 2) nan_tile[threadIdx.x] = 0;
    if (tiles) {
        stage = look_up(a, q, head, begin + 16 * lane, end);
        here = stage;
        fetch(0);
    }
    __syncthreads();
    if (tiles) place(0);
    for (int tile = 0; tile < tiles; tile++) {
        const int buf = tile & 1, t0 = begin + kTile * tile;
        if (tile && (tile & 15) == 0) here = stage;
        if (tile + 1 < tiles) {
            if (((tile + 1) & 15) == 0) stage = look_up(a, q, head, begin + kTile * (tile + 1) + 16 * lane, end);
            fetch(tile + 1);
        }
        __syncthreads();                        // this tile is in LDS
        if (t0 <= most) {
#pragma unroll
            for (int sub = 0; sub < 2; sub++) {
                const int t = t0 + 32 * sub;
                if (t > most) break;
                float ks[2], vs[2];
                bool there = true;
#pragma unroll
                for (int x = 0; x < 2; x++) {
                    const int six = (4 * tile + 2 * sub + x) & 63;
                    ks[x] = lane_value(here.ks, six) * scale;
                    vs[x] = lane_value(here.vs, six);
                    there = there && __builtin_amdgcn_readlane(here.entry, six) >= 0;
                }
                f32x16 z[NQ];
#pragma unroll
                for (int n = 0; n < NQ; n++)
#pragma unroll
                    for (int i = 0; i < 16; i++) z[n][i] = 0.0f;
#pragma unroll
                for (int k = 0; k < KK; k++) {
                    const u32x4 f = *reinterpret_cast<const u32x4 *>(lk(buf) + (32 * sub + col) * KP + 32 * k + 16 * half);
#pragma unroll
                    for (int n = 0; n < NQ; n++) z[n] = T::mfma32(f, qf[n][k], z[n]);
                }
                const bool full = there && t + 31 <= least && !ragged;
                if (!full) {
#pragma unroll
                    for (int i = 0; i < 16; i++) {
                        const int at = t + 8 * (i >> 2) + 4 * half + (i & 3);
                        const bool is = __builtin_amdgcn_readlane(here.entry, (4 * tile + 2 * sub + (i >> 3)) & 63) >= 0;
#pragma unroll
                        for (int n = 0; n < NQ; n++) z[n][i] = is && at <= lim[n] ? z[n][i] : -INFINITY;
                    }
                }
                bool rises = false;
                float top[NQ];
#pragma unroll
                for (int n = 0; n < NQ; n++) {
                    float x[2];
#pragma unroll
                    for (int y = 0; y < 2; y++)
                        x[y] = fmaxf(fmaxf(fmaxf(z[n][8 * y], z[n][8 * y + 1]), fmaxf(z[n][8 * y + 2], z[n][8 * y + 3])),
                                     fmaxf(fmaxf(z[n][8 * y + 4], z[n][8 * y + 5]), fmaxf(z[n][8 * y + 6], z[n][8 * y + 7])));
                    // (-inf stays -inf, also where a scale is 0)
                    top[n] = fmaxf(full || x[0] != -INFINITY ? x[0] * ks[0] : x[0], full || x[1] != -INFINITY ? x[1] * ks[1] : x[1]);
                    rises |= top[n] > m[n] + kSlack;
                }
                if (__ballot(rises)) {
#pragma unroll
                    for (int n = 0; n < NQ; n++) {
                        const float now = fmaxf(m[n], fmaxf(top[n], __shfl_xor(top[n], 32)));
                        const float f = now == -INFINITY ? 1.0f : exp2_of(m[n] - now);
                        m[n] = now;
                        base[n] = now == -INFINITY ? 0.0f : now;
                        l[n] *= f;
#pragma unroll
                        for (int d = 0; d < ND; d++) o[n][d] *= f;
                    }
                }
                if constexpr (T::kNarrow) {     // V's scale relative to the largest yet, to stay within fp16's range
                    const float largest = fmaxf(vs[0], vs[1]);
                    if (largest > v_ref) {
                        const float f = v_ref / largest;
#pragma unroll
                        for (int n = 0; n < NQ; n++)
#pragma unroll
                            for (int d = 0; d < ND; d++) o[n][d] *= f;
                        v_ref = largest;
                    }
                    const float inv = v_ref > 0.0f ? 1.0f / v_ref : 0.0f;
                    vs[0] *= inv, vs[1] *= inv;
                }
                u32x4 pf[NQ][2];
#pragma unroll
                for (int n = 0; n < NQ; n++)
#pragma unroll
                    for (int x = 0; x < 2; x++) {
                        float e[8];
#pragma unroll
                        for (int i = 0; i < 8; i++) {
                            const float s = z[n][8 * x + i];
                            e[i] = exp2_of(full ? s * ks[x] - base[n] : s == -INFINITY ? s : s * ks[x] - base[n]);
                            l[n] += e[i];
                            e[i] *= vs[x];
                        }
#pragma unroll
                        for (int i = 0; i < 4; i++) pf[n][x][i] = T::pack(e[2 * i], e[2 * i + 1]);
                    }
                const bool mixed = !full && nan_tile[buf] == tile + 1;
#pragma unroll
                for (int d = 0; d < ND; d++)
#pragma unroll
                    for (int x = 0; x < 2; x++) {
                        u32x4 f = *reinterpret_cast<const u32x4 *>(lv(buf) + (32 * d + col) * VP + 64 * sub + 32 * x + 16 * half);
                        if (mixed) {            // a NaN in V reaches the queries that see it, and 0 * NaN no other
                            u32x4 bad;
#pragma unroll
                            for (int i = 0; i < 4; i++) {
                                const bool lo = (f[i] & 0x7FFFu) > T::kInf, hi = (f[i] >> 16 & 0x7FFFu) > T::kInf;
                                bad[i] = (lo ? T::kOne : 0u) | (hi ? T::kOne << 16 : 0u);
                                f[i] &= (lo ? 0u : 0xFFFFu) | (hi ? 0u : 0xFFFF0000u);
                            }
#pragma unroll
                            for (int n = 0; n < NQ; n++) {
                                u32x4 sees;
#pragma unroll
                                for (int i = 0; i < 4; i++) {
                                    const int at = t + 16 * x + 4 * half + 8 * (i >> 1) + 2 * (i & 1);
                                    sees[i] = (at <= lim[n] ? T::kOne : 0u) | (at + 1 <= lim[n] ? T::kOne << 16 : 0u);
                                }
                                f32x16 nans;
#pragma unroll
                                for (int i = 0; i < 16; i++) nans[i] = 0.0f;
                                nans = T::mfma32(bad, sees, nans);
#pragma unroll
                                for (int i = 0; i < 16; i++) o[n][d][i] += nans[i] > 0.0f ? NAN : 0.0f;
                            }
                        }
#pragma unroll
                        for (int n = 0; n < NQ; n++) o[n][d] = T::mfma32(f, pf[n][x], o[n][d]);
                    }
            }
        }
        if (tile + 1 < tiles) place(tile + 1);
    }

#pragma unroll
    for (int n = 0; n < NQ; n++) {
        l[n] += __shfl_xor(l[n], 32);
        const int row = wave_row + 32 * n + col;
        if (row >= rows) continue;
        const QueryRow w = query_row(a, head, (uint32_t)row);
        const int64_t at = (int64_t)(q.start + w.token) * a.q_heads + w.head;
        const bool empty = m[n] == -INFINITY && l[n] == 0.0f;
        if (p.splits == 1) {
            const float f = (empty ? 0.0f : 1.0f / l[n]) * v_ref;
            uint16_t *dst = static_cast<uint16_t *>(a.out.data) + (int64_t)(q.start + w.token) * a.out.row_stride + (int64_t)w.head * a.out.head_stride;
#pragma unroll
            for (int d = 0; d < ND; d++)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const int e = 32 * d + 2 * i + 4 * half;
                    if (e < (int)a.c.dim)
                        *reinterpret_cast<u32x2 *>(dst + e) = u32x2{T::pack(o[n][d][i] * f, o[n][d][i + 1] * f), T::pack(o[n][d][i + 2] * f, o[n][d][i + 3] * f)};
                }
            if (half == 0) {
                const float sum = empty ? -INFINITY : m[n] + log2_of(l[n]);
                if (a.lse) a.lse[at] = sum * kLn2;
                if (p.totals) p.totals[at] = sum;
            }
        } else {
            if (half == 0) p.sums[at * p.splits + split] = f32x2{m[n], l[n]};
            float *dst = p.parts + (at * p.splits + split) * a.c.dim;
#pragma unroll
            for (int d = 0; d < ND; d++)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const int e = 32 * d + 2 * i + 4 * half;
                    if (e < (int)a.c.dim) *reinterpret_cast<f32x4 *>(dst + e) = f32x4{o[n][d][i], o[n][d][i + 1], o[n][d][i + 2], o[n][d][i + 3]} * v_ref;
                }
        }
    }
}

// Outputs out of the parts that splits of the contexts left, a wavefront a row.
template <typename T>
__global__ __launch_bounds__(256) void join_parts_kernel(AttendArgs a, PartsPlan p, uint32_t tile_rows)
{
    const int lane = threadIdx.x & 63;
    const Request q = request_of(a.b, a.c, (int)blockIdx.y);
    const uint32_t n = blockIdx.x * 4u + (threadIdx.x >> 6), rows = (uint32_t)q.fresh * a.group;
    if (n >= rows * a.c.heads) return;
    const uint32_t head = n / rows, row = n - head * rows;
    const QueryRow w = query_row(a, head, row);
    const int64_t at = (int64_t)(q.start + w.token) * a.q_heads + w.head;
    // splits that the row's workgroup had work in
    const uint32_t last_row = min((row / tile_rows + 1u) * tile_rows, rows) - 1u;
    const int seen = q.len - q.fresh + (int)(last_row / a.group) + 1, splits = max(1, (seen + (int)p.chunk - 1) / (int)p.chunk);
    const f32x2 *sums = p.sums + at * p.splits;
    float top = -INFINITY, sum = 0.0f;
    for (int s = 0; s < splits; s++) top = fmaxf(top, sums[s][0]);
    const float to = top == -INFINITY ? 0.0f : top;
    for (int s = 0; s < splits; s++) sum += sums[s][1] * exp2_of(sums[s][0] - to);
    const float total = top == -INFINITY && sum == 0.0f ? -INFINITY : to + log2_of(sum);
    const int d = 4 * lane;
    if (d < (int)a.c.dim) {
        f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int s = 0; s < splits; s++) {
            const float f = total == -INFINITY ? 0.0f : exp2_of(sums[s][0] - total);
            o += *reinterpret_cast<const f32x4 *>(p.parts + (at * p.splits + s) * a.c.dim + d) * f;
        }
        uint16_t *dst = static_cast<uint16_t *>(a.out.data) + (int64_t)(q.start + w.token) * a.out.row_stride + (int64_t)w.head * a.out.head_stride + d;
        *reinterpret_cast<u32x2 *>(dst) = u32x2{T::pack(o[0], o[1]), T::pack(o[2], o[3])};
    }
    if (!lane) {
        if (a.lse) a.lse[at] = total * kLn2;
        if (p.totals) p.totals[at] = total;
    }
}

// Weights: 256 tokens a workgroup, 64 a wavefront, whose K stays in registers; the query rows that see them pass through LDS 32 at
// a time.  Scores once more (their rows' totals were not known before), p summed over the rows in fp32, in order.
template <typename T, int DP>
__global__ __launch_bounds__(256) void weights_kernel(AttendArgs a, PartsPlan p)
{
    constexpr int QP = DP * 2 + 16, KK = DP / 16;
    __shared__ __align__(16) uint8_t lq[2][32 * QP];
    __shared__ float lt[2][32];
    __shared__ int ll[2][32];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
    const uint32_t head = blockIdx.x % a.c.heads;
    const Request q = request_of(a.b, a.c, (int)blockIdx.y);
    const int block0 = (int)(blockIdx.x / a.c.heads) * 256, t0 = block0 + 64 * wave;
    if (block0 >= q.len) return;
    const int older = q.len - q.fresh, rows = q.fresh * (int)a.group;
    const int first_row = max(0, block0 - older) * (int)a.group, tiles = (rows - first_row + 31) / 32;

    // K of the wavefront's tokens: two 32s, their sixteens' scales
    const Look l = look_up(a, q, head, t0 + 16 * lane, lane < 4 ? q.len : 0);
    u32x4 kf[2][KK];
    float ks[4];
#pragma unroll
    for (int x = 0; x < 4; x++) ks[x] = lane_value(l.ks, x) * a.scale_log2;
#pragma unroll
    for (int s = 0; s < 2; s++) {
        const int t = t0 + 32 * s + col, e0 = __builtin_amdgcn_readlane(l.entry, 2 * s), e1 = __builtin_amdgcn_readlane(l.entry, 2 * s + 1);
        const int e = col < 16 ? e0 : e1;
        const uint32_t b = block_of(a.c, (uint32_t)t >> 4);
        const uint8_t *k = code_at(a.c, 0, max(e, 0), (uint32_t)t - b * a.c.bs, head);
#pragma unroll
        for (int i = 0; i < KK; i++) {
            const int d = 16 * i + 8 * half;
            u32x2 w = {0u, 0u};
            if (d < (int)a.c.dim) w = *reinterpret_cast<const u32x2 *>(k + d);
            kf[s][i] = u32x4{T::two_codes(w[0], false), T::two_codes(w[0], true), T::two_codes(w[1], false), T::two_codes(w[1], true)};
        }
    }

    // 8 threads a query row
    u32x4 rq[DP / 64];
    float rt = -INFINITY;
    int rl = -1;
    auto fetch = [&](int tile) {
        const int row = first_row + 32 * tile + (int)(threadIdx.x >> 3);
        rt = -INFINITY, rl = -1;
#pragma unroll
        for (int c = 0; c < DP / 64; c++) rq[c] = u32x4{0u, 0u, 0u, 0u};
        if (row < rows) {
            const QueryRow w = query_row(a, head, (uint32_t)row);
            const uint16_t *src = static_cast<const uint16_t *>(a.q.data) + (int64_t)(q.start + w.token) * a.q.row_stride + (int64_t)w.head * a.q.head_stride;
#pragma unroll
            for (int c = 0; c < DP / 64; c++) {
                const int d = 64 * c + 8 * (int)(threadIdx.x & 7);
                if (d < (int)a.c.dim) rq[c] = *reinterpret_cast<const u32x4 *>(src + d);
            }
            rt = p.totals[(int64_t)(q.start + w.token) * a.q_heads + w.head];
            rl = rt == -INFINITY ? -1 : older + w.token;
        }
    };
    auto place = [&](int buf) {
#pragma unroll
        for (int c = 0; c < DP / 64; c++)
            *reinterpret_cast<u32x4 *>(lq[buf] + (threadIdx.x >> 3) * QP + 2 * (64 * c + 8 * (threadIdx.x & 7))) = rq[c];
        if ((threadIdx.x & 7) == 0) lt[buf][threadIdx.x >> 3] = rt, ll[buf][threadIdx.x >> 3] = rl;
    };
    float w[2][16];
#pragma unroll
    for (int s = 0; s < 2; s++)
#pragma unroll
        for (int i = 0; i < 16; i++) w[s][i] = 0.0f;
    if (tiles > 0) {
        fetch(0);
        place(0);
    }
    for (int tile = 0; tile < tiles; tile++) {
        const int buf = tile & 1;
        if (tile + 1 < tiles) fetch(tile + 1);
        __syncthreads();
        f32x16 z[2];
#pragma unroll
        for (int s = 0; s < 2; s++)
#pragma unroll
            for (int i = 0; i < 16; i++) z[s][i] = 0.0f;
#pragma unroll
        for (int k = 0; k < KK; k++) {
            const u32x4 f = *reinterpret_cast<const u32x4 *>(lq[buf] + col * QP + 32 * k + 16 * half);
#pragma unroll
            for (int s = 0; s < 2; s++) z[s] = T::mfma32(kf[s][k], f, z[s]);
        }
        const float total = lt[buf][col];
        const int lim = ll[buf][col];
        const bool full = __ballot(lim < t0 + 63) == 0;
#pragma unroll
        for (int s = 0; s < 2; s++)
#pragma unroll
            for (int i = 0; i < 16; i++) {
                const float e = exp2_of(z[s][i] * ks[2 * s + (i >> 3)] - total);
                w[s][i] += full || t0 + 32 * s + 8 * (i >> 2) + 4 * half + (i & 3) <= lim ? e : 0.0f;
            }
        if (tile + 1 < tiles) place(buf ^ 1);
    }
#pragma unroll
    for (int s = 0; s < 2; s++)
#pragma unroll
        for (int i = 0; i < 16; i++) {
            float x = w[s][i];
#pragma unroll
            for (int k = 1; k < 32; k <<= 1) x += __shfl_xor(x, k);
            const int t = t0 + 32 * s + 8 * (i >> 2) + 4 * half + (i & 3);
            if (__builtin_amdgcn_readlane(l.entry, 2 * s + (i >> 3)) < 0) x = 0.0f;
            if (col == i && t < q.len) {
                if (a.prior.data && t < older)
                    x += a.decay * a.prior.data[(int64_t)q.row * a.prior.row_stride + (int64_t)head * a.prior.head_stride + t];
                a.w.data[(int64_t)q.row * a.w.row_stride + (int64_t)head * a.w.head_stride + t] = x;
            }
        }
}

template <typename T, int DP, int NQ> static hipError_t parts(const AttendArgs &a, const PartsPlan &p, hipStream_t s)
{
    const uint32_t pairs = (a.b.n_reqs * a.c.heads + 7u) / 8u;
    parts_kernel<T, DP, NQ><<<dim3(pairs * p.row_tiles * p.splits * 8u), 256, 0, s>>>(a, p);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && p.splits > 1u) {
        join_parts_kernel<T><<<dim3((a.b.max_new * a.q_heads + 3u) / 4u, a.b.n_reqs), 256, 0, s>>>(a, p, 128u * NQ);
        e = hipGetLastError();
    }
    if (e == hipSuccess && a.w.data) {
        weights_kernel<T, DP><<<dim3((a.b.max_len + 255u) / 256u * a.c.heads, a.b.n_reqs), 256, 0, s>>>(a, p);
        e = hipGetLastError();
    }
    return e;
}

template <typename T> static hipError_t parts_of(const AttendArgs &a, const PartsPlan &p, hipStream_t s)
{
    return a.c.dim <= 64 ? parts<T, 64, 2>(a, p, s) : a.c.dim <= 128 ? parts<T, 128, 2>(a, p, s) : parts<T, 256, 1>(a, p, s);
}

hipError_t launch_parts(const AttendArgs &a, const PartsPlan &p, uint32_t dtype, hipStream_t s)
{
    return dtype == DMI_DTYPE_BF16 ? parts_of<Bf16>(a, p, s) : parts_of<Fp16>(a, p, s);
}

}  // namespace kv8
}  // namespace dmi
