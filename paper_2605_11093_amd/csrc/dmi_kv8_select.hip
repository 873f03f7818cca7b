// Kernels that choose, for each new token and head of the 8-bit KV cache, the blocks that can hold the largest scores.
#include "dmi_internal.h"
#include "dmi_kv8_mfma.h"

#include <algorithm>

namespace dmi {
namespace kv8 {

// Blocks that a token chooses from by score, between those that it takes anyway; none where it takes all that it sees.
struct Choice {
    uint32_t seen;                              // blocks that the token sees
    uint32_t lo, hi;
};
__device__ __forceinline__ Choice choice_of(const SelectArgs &a, const Request &q)
{
    const uint32_t seen = q.len > 0 ? block_of(a.c, (uint32_t)(q.len - 1) >> 4) + 1u : 0u;
    if (seen <= a.n_select) return {seen, 0u, 0u};
    return {seen, a.n_first, seen - a.n_recent};
}

// Scores in an order of unsigned numbers: NaN as -inf, -0 as 0.
__device__ __forceinline__ uint64_t order_of(double x)
{
    if (x != x) x = -INFINITY;
    const uint64_t u = __builtin_bit_cast(uint64_t, x + 0.0);
    return u >> 63 ? ~u : u | 1ull << 63;
}
__device__ __forceinline__ uint32_t order_of(float x)
{
    const uint32_t u = __float_as_uint(x);
    return u >> 31 ? ~u : u | 1u << 31;
}
__device__ __forceinline__ float float_of(uint32_t order) { return __uint_as_float(order >> 31 ? order & 0x7FFFFFFFu : ~order); }

// Largest of what 16 lanes have
__device__ __forceinline__ float largest_of_16(float x)
{
    auto turned = [](float v, auto n) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x120 + decltype(n)::value, 0xF, 0xF, false)); };
    x = fmaxf(x, turned(x, Int<8>{}));
    x = fmaxf(x, turned(x, Int<4>{}));
    x = fmaxf(x, turned(x, Int<2>{}));
    return fmaxf(x, turned(x, Int<1>{}));
}

// Largest of what `each` neighbours have, 1 to 16 (a power of two)
__device__ __forceinline__ float largest_of(float x, uint32_t each)
{
    auto other = [](float v, auto how) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(how)::value, 0xF, 0xF, false)); };
    if (each > 1u) x = fmaxf(x, other(x, Int<0xB1>{}));         // the one beside it
    if (each > 2u) x = fmaxf(x, other(x, Int<0x4E>{}));         // two further
    if (each > 4u) x = fmaxf(x, other(x, Int<0x141>{}));        // eight, mirrored
    if (each > 8u) x = fmaxf(x, other(x, Int<0x140>{}));        // sixteen
    return x;
}

// ---------------------------------------------------------------- scores, nearly
// The larger of q x least and q x largest is one product with the one or the other, by q's sign: a score is the product of a row (q where
// it is negative; q where it is positive) with a column (least; largest), and matrix instructions take it, 16 blocks x 16 query rows at a
// time.  Every product is exact in fp32; their sum is off by no more than 2 dim + 16 roundings (of one unit in the last place, whatever
// the instruction's order and rounding) of 448 sum |q|, the most that the terms' magnitudes add up to, and by what numbers of q below
// the normal ones make, should they count as 0.  What lies nearer than twice that to the score at which the selection ends is looked at
// again in 64 bits.
//
// A wavefront asks for the bounds of its next 16 blocks before it uses those of the last.
template <typename T, int DP> struct Scorer {
    static constexpr int KL = DP / 64, KK = DP / 32;
    const SelectArgs &a;
    const Request &q;
    uint32_t token, head;
    int lane, col, g;
    u32x4 below[KK], above[KK];                 // q where it is negative, positive
    float off;                                  // how far a score may be off, before K's scale

    __device__ __forceinline__ Scorer(const SelectArgs &a_, const Request &q_, uint32_t token_, uint32_t head_)
        : a(a_), q(q_), token(token_), head(head_), lane(threadIdx.x & 63), col(lane & 15), g(lane >> 4), off(0.0f) {}

    // A column's query row, of token t; how far its scores may be off
    __device__ __forceinline__ float column(uint32_t t, uint32_t row)
    {
        const uint16_t *const src = static_cast<const uint16_t *>(a.q.data) + (int64_t)t * a.q.row_stride + (int64_t)(head * a.group + row) * a.q.head_stride;
        float sum = 0.0f, faint = 0.0f;
#pragma unroll
        for (int k = 0; k < KK; k++) {
            const uint32_t d = (uint32_t)(g * (DP / 4) + 8 * k);
            const u32x4 w = *reinterpret_cast<const u32x4 *>(src + (d < a.c.dim ? d : 0u));
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const uint32_t v = d < a.c.dim ? w[i] : 0u, sign = (v >> 15 & 0x00010001u) * 0xFFFFu;
                below[k][i] = v & sign, above[k][i] = v & ~sign;
#pragma unroll
                for (int y = 0; y < 2; y++) {
                    const float size = fabsf(T::number((uint16_t)(v >> 16 * y)));
                    sum += size;
                    if (!(v >> 16 * y & T::kExponent)) faint += size;
                }
            }
        }
        sum += __shfl_xor(sum, 16), faint += __shfl_xor(faint, 16);
        sum += __shfl_xor(sum, 32), faint += __shfl_xor(faint, 32);
        // (of nothing but zeros every score is 0 or no number, and that is exact)
        return sum == 0.0f ? 0.0f : sum > 0x1p-90f && sum < 0x1p+100f ? 448.0f * ((float)(2 * DP + 16) * 0x1p-23f * sum + 1.001f * faint) : INFINITY;
    }
    __device__ __forceinline__ void rows(uint32_t row0) { off = fmaxf(off, largest_of_16(column(token, min(row0 + (uint32_t)col, a.group - 1u)))); }
    struct Tile {
        u32x4 low[KL], high[KL];
        float scale;
    };
    // 16 blocks' bounds, and for the lanes with col < 4 K's scale of block 4 g + col (0 where there is none).  entry(i): where block i lies
    template <typename Entry> __device__ __forceinline__ Tile fetch(const Entry &entry) const
    {
        Tile x;
        const int mine = entry((uint32_t)(4 * g + (col & 3)));
        x.scale = *scale_at(a.c, 0, max(mine, 0), head);
        const uint8_t *const at = a.bounds + (int64_t)max(entry((uint32_t)col), 0) * a.bounds_block_stride + (int64_t)head * a.bounds_head_stride;
#pragma unroll
        for (int c = 0; c < KL; c++) {
            const uint32_t d = (uint32_t)(g * (DP / 4) + 16 * c), from = d < a.c.dim ? d : 0u;
            x.low[c] = *reinterpret_cast<const u32x4 *>(at + from);
            x.high[c] = *reinterpret_cast<const u32x4 *>(at + a.c.dim + from);
        }
        if (mine < 0) x.scale = 0.0f;
        return x;
    }
    // Scores of blocks 4 g + 0..3 by the column's row
    __device__ __forceinline__ f32x4 products(const Tile &x) const
    {
        f32x4 z = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < KK; k++) {
            const u32x4 &l = x.low[k / 2], &h = x.high[k / 2];
            const uint32_t l0 = l[2 * (k % 2)], l1 = l[2 * (k % 2) + 1], h0 = h[2 * (k % 2)], h1 = h[2 * (k % 2) + 1];
            z = T::mfma16(u32x4{T::two_codes(l0, false), T::two_codes(l0, true), T::two_codes(l1, false), T::two_codes(l1, true)}, below[k], z);
            z = T::mfma16(u32x4{T::two_codes(h0, false), T::two_codes(h0, true), T::two_codes(h1, false), T::two_codes(h1, true)}, above[k], z);
        }
        return z;
    }
    // The largest score of block 4 g + (col & 3) by these rows (rows behind the group's last are that one again).  INFINITY says that one is
    // no number.
    __device__ __forceinline__ float of(const Tile &x) const
    {
        const f32x4 z = products(x);
        float best = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const float v = largest_of_16(z[i] == z[i] ? z[i] : INFINITY);
            if ((col & 3) == i) best = v;
        }
        return best;
    }
};
// A block's score as it counts: none where there is no block (scale 0), or no number
__device__ __forceinline__ float counted(float best, float scale)
{
    const float v = best * scale;
    return scale != 0.0f && fabsf(v) < INFINITY ? v + 0.0f : -INFINITY;
}
// How far that may be off, `wide` before K's scale.  A scale that takes a number out of fp32's range says nothing about it: it is looked at in 64
// bits, and as long as scores are not exact there is an error, however small (one that fp32 has no number for counted as none).
__device__ __forceinline__ float off_of(float wide, float best, float scale)
{
    if (fabsf(best) < INFINITY && fabsf(best * scale) == INFINITY) return INFINITY;
    return scale != 0.0f && wide > 0.0f ? fmaxf(wide * scale, 0x1p-126f) : 0.0f;
}

// A score in 64 bits, as an unsigned number in their order: a wavefront's work, 16 lanes a query row.
template <typename T> __device__ __forceinline__ uint64_t exact_order(const SelectArgs &a, const Request &q, uint32_t token, uint32_t head, uint32_t block)
{
    const uint32_t lane = threadIdx.x & 63u;
    const int entry = entry_of(a.c, q.row, block);
    if (entry < 0) return order_of((double)-INFINITY);
    const uint8_t *const at = a.bounds + (int64_t)entry * a.bounds_block_stride + (int64_t)head * a.bounds_head_stride;
    const double scale = *scale_at(a.c, 0, entry, head);
    double best = -INFINITY;
    bool bad = false;
    for (uint32_t r0 = 0; r0 < a.group; r0 += 4u) {
        const uint32_t r = min(r0 + (lane >> 4), a.group - 1u);
        const uint16_t *const src = static_cast<const uint16_t *>(a.q.data) + (int64_t)token * a.q.row_stride + (int64_t)(head * a.group + r) * a.q.head_stride;
        double sum = 0.0;
        for (uint32_t d = 8u * (lane & 15u); d < a.c.dim; d += 128u) {
            const u32x4 v = *reinterpret_cast<const u32x4 *>(src + d);
            const u32x2 l = *reinterpret_cast<const u32x2 *>(at + d), h = *reinterpret_cast<const u32x2 *>(at + a.c.dim + d);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const double x = T::number((uint16_t)(v[i / 2] >> 16 * (i % 2)));
                const f32x2 l2 = i & 2 ? __builtin_amdgcn_cvt_pk_f32_fp8((int)l[i / 4], true) : __builtin_amdgcn_cvt_pk_f32_fp8((int)l[i / 4], false);
                const f32x2 h2 = i & 2 ? __builtin_amdgcn_cvt_pk_f32_fp8((int)h[i / 4], true) : __builtin_amdgcn_cvt_pk_f32_fp8((int)h[i / 4], false);
                const double least = x * (double)l2[i & 1], most = x * (double)h2[i & 1];
                sum += least != least || most != most ? NAN : fmax(least, most);
            }
        }
        auto turned = [](double v, auto n) {
            const uint64_t w = __builtin_bit_cast(uint64_t, v);
            const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)w, 0x120 + decltype(n)::value, 0xF, 0xF, false);
            const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(w >> 32), 0x120 + decltype(n)::value, 0xF, 0xF, false);
            return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
        };
        sum += turned(sum, Int<8>{});
        sum += turned(sum, Int<4>{});
        sum += turned(sum, Int<2>{});
        sum += turned(sum, Int<1>{});
        bad |= sum != sum;
        best = sum > best ? sum : best;
    }
#pragma unroll
    for (int m = 16; m < 64; m <<= 1) {
        const double other = __shfl_xor(best, m);
        best = other > best ? other : best;
    }
    return order_of(__ballot(bad) ? (double)-INFINITY : best * scale);
}

// ---------------------------------------------------------------- which blocks
constexpr uint32_t kScoreThreads = 256, kBlocksAtOnce = kScoreThreads / 2;      // blocks of a workgroup
constexpr uint32_t kPickBins = 2048;
constexpr uint32_t kClose = 256;                                // blocks near the border that are ranked in LDS

struct PickShared {
    uint32_t hist[kPickBins];
    uint32_t wave_n[16][2], found[3], count[3];
    float wave_x[16][3];
    uint32_t close[kClose];
    uint64_t order[kClose];
    uint32_t off[16];                           // several tokens: how far their scores may be off, as numbers of fp32
};

// The bin that holds the rank-th of those counted, from the largest bin down: found = bin, rank in it, how many it has.
template <uint32_t N> __device__ __forceinline__ void find_bin(PickShared &s, uint32_t rank)
{
    constexpr uint32_t kEach = kPickBins / N;
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6;
    __syncthreads();
    uint32_t n[kEach], sum = 0;
#pragma unroll
    for (uint32_t i = 0; i < kEach; i++) sum += n[i] = s.hist[kPickBins - 1u - kEach * tid - i];
    uint32_t before = (uint32_t)lanes_scan((int)sum);
    if (lane == 63u) s.wave_n[wave][0] = before;
    __syncthreads();
    before -= sum;
#pragma unroll
    for (uint32_t v = 0; v < N / 64u; v++)
        if (v < wave) before += s.wave_n[v][0];
#pragma unroll
    for (uint32_t i = 0; i < kEach; i++) {
        if (before < rank && rank <= before + n[i]) {
            s.found[0] = kPickBins - 1u - kEach * tid - i;
            s.found[1] = rank - before;
            s.found[2] = n[i];
        }
        before += n[i];
    }
    __syncthreads();
}

// Of `count` unsigned numbers that key(i) gives, those that begin with `prefix` (their bits from `shift` on) hold the want-th largest: `rank`-th
// of them, `same` in all.  Digit by digit, from the top and, unless all bits are asked for, only as far as it takes to tell it from the others.
template <uint32_t N, typename U, typename Key>
__device__ __forceinline__ void find_rank(PickShared &s, uint32_t count, uint32_t want, bool all_bits, const Key &key, U &prefix, int &shift, uint32_t &rank)
{
    const uint32_t tid = threadIdx.x;
    prefix = 0;
    rank = want;
    shift = 8 * (int)sizeof(U);
    while (shift > 0) {
        const int bits = min(11, shift), above = shift;
        shift -= bits;
        for (uint32_t i = tid; i < kPickBins; i += N) s.hist[i] = 0;
        __syncthreads();
        for (uint32_t i = tid; i < count; i += N) {
            const U k = key(i);
            if (above == 8 * (int)sizeof(U) || k >> above == prefix) atomicAdd(&s.hist[(uint32_t)(k >> shift) & ((1u << bits) - 1u)], 1u);
        }
        find_bin<N>(s, rank);
        prefix = prefix << bits | s.found[0];
        rank = s.found[1];
        if (!all_bits && s.found[2] == rank) break;
    }
}

// Numbers lo + i of those i < count that are more (which(i) > 0), or among the first `rank` that are equal (0), in order.  A thread has
// neighbours, so that one look over all threads' counts is enough.
template <uint32_t N, typename Which> __device__ __forceinline__ void write_in_order(PickShared &s, uint32_t count, uint32_t lo, uint32_t rank, const Which &which, int32_t *to)
{
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6, each = (count + N - 1u) / N;
    const uint32_t from = min(tid * each, count), end = min(from + each, count);
    uint32_t more = 0, same = 0;
    for (uint32_t i = from; i < end; i++) {
        const int w = which(i);
        more += w > 0, same += w == 0;
    }
    uint32_t m = (uint32_t)lanes_scan((int)more), e = (uint32_t)lanes_scan((int)same);
    __syncthreads();
    if (lane == 63u) s.wave_n[wave][0] = m, s.wave_n[wave][1] = e;
    __syncthreads();
    m -= more, e -= same;
#pragma unroll
    for (uint32_t v = 0; v < N / 64u; v++)
        if (v < wave) m += s.wave_n[v][0], e += s.wave_n[v][1];
    for (uint32_t i = from; i < end; i++) {
        const int w = which(i);
        if (w > 0 || (w == 0 && e < rank)) to[m + min(e, rank)] = (int32_t)(lo + i);
        m += w > 0, e += w == 0;
    }
}

// (two wavefronts a SIMD with 256 elements, four with fewer)
template <typename T, int DP> __global__ __launch_bounds__(kScoreThreads) __attribute__((amdgpu_waves_per_eu(DP <= 128 ? 4 : 2))) void score_kernel(SelectArgs a)
{
    const uint32_t per = (a.stride + kBlocksAtOnce - 1u) / kBlocksAtOnce, item = blockIdx.x / per, chunk = blockIdx.x - item * per;
    const uint32_t token = item / a.c.heads, head = item - token * a.c.heads, lane = threadIdx.x & 63u;
    const Request q = token_of(a.b, a.c, (int)token);
    const Choice x = choice_of(a, q);
    const uint32_t block0 = x.lo + kBlocksAtOnce * chunk + 32u * (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (q.fresh <= 0 || block0 >= x.hi) return;
    Scorer<T, DP> scorer(a, q, token, head);
    const int own = block0 + (lane & 31u) < x.hi ? entry_of(a.c, q.row, block0 + (lane & 31u)) : -1;
    typename Scorer<T, DP>::Tile tile[2];
#pragma unroll
    for (uint32_t y = 0; y < 2u; y++) tile[y] = scorer.fetch([&](uint32_t i) { return __shfl(own, (int)(16u * y + i)); });
    float s[2] = {-INFINITY, -INFINITY};
    for (uint32_t row0 = 0; row0 < a.group; row0 += 16u) {
        scorer.rows(row0);
#pragma unroll
        for (int y = 0; y < 2; y++) s[y] = fmaxf(s[y], scorer.of(tile[y]));
    }
#pragma unroll
    for (uint32_t y = 0; y < 2u; y++) {
        const uint32_t block = block0 + 16u * y + 4u * (uint32_t)scorer.g + (uint32_t)scorer.col;
        if (scorer.col < 4 && block < x.hi) a.scores[(int64_t)item * a.stride + block] = f32x2{counted(s[y], tile[y].scale), off_of(scorer.off, s[y], tile[y].scale)};
    }
}

// The choice out of scores, in LDS or in memory; off, most and least as the thread has seen them
template <typename T, uint32_t N>
__device__ __forceinline__ void choose(PickShared &s, const SelectArgs &a, const Request &q, uint32_t token, uint32_t head, const Choice &x, float *own,
                                       bool in_lds, float off, float most, float least)
{
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = (uint32_t)__builtin_amdgcn_readfirstlane(tid >> 6), item = token * a.c.heads + head;
    const uint32_t want = a.n_select - a.n_first - a.n_recent, count = x.hi - x.lo;
    int32_t *const to = a.blocks + (int64_t)item * a.n_select;
    f32x2 *const left = a.scores + (int64_t)item * a.stride + x.lo;
#pragma unroll
    for (int m = 32; m; m >>= 1) off = fmaxf(off, __shfl_xor(off, m)), most = fmaxf(most, __shfl_xor(most, m)), least = fminf(least, __shfl_xor(least, m));
    if (!lane) s.wave_x[wave][0] = off, s.wave_x[wave][1] = most, s.wave_x[wave][2] = least;
    __syncthreads();
#pragma unroll
    for (uint32_t v = 0; v < N / 64u; v++) off = fmaxf(off, s.wave_x[v][0]), most = fmaxf(most, s.wave_x[v][1]), least = fminf(least, s.wave_x[v][2]);
    auto score = [&](uint32_t i) { return in_lds ? own[i] : left[i][0]; };
    // A step of the range: equal numbers share one, larger ones have none that is lower
    const float steps = (float)(kPickBins - 1u) / fmaxf(most - least, 0x1p-100f);
    auto step_of = [&](float v) { return (uint32_t)fminf(fmaxf((v - least) * steps, 0.0f), (float)(kPickBins - 1u)); };
    for (uint32_t i = tid; i < count; i += N) atomicAdd(&s.hist[step_of(score(i))], 1u);
    find_bin<N>(s, want);
    const uint32_t bin = s.found[0], in_bin = s.found[2];
    uint32_t rank = s.found[1];
    if (in_bin <= kClose) {
        for (uint32_t i = tid; i < count; i += N) {
            const float v = score(i);
            if (step_of(v) == bin) s.close[atomicAdd(&s.count[2], 1u)] = order_of(v);
        }
        __syncthreads();
        if (tid < in_bin) {
            uint32_t more = 0, same = 0;
            for (uint32_t i = 0; i < in_bin; i++) more += s.close[i] > s.close[tid], same += s.close[i] == s.close[tid];
            if (more < rank && rank <= more + same) s.found[0] = s.close[tid];
        }
        __syncthreads();
    } else {
        uint32_t border;
        int shift;
        __syncthreads();
        find_rank<N, uint32_t>(s, count, want, true, [&](uint32_t i) { return order_of(score(i)); }, border, shift, rank);
        __syncthreads();
        if (!tid) s.found[0] = border;
        __syncthreads();
    }
    const float t = float_of(s.found[0]);       // the want-th largest
    // what is nearer to the want-th than both may be off together (and numbers so small that fp32 runs out below them are all near)
    const float off2 = off > 0.0f && off < 0x1p-80f ? INFINITY : 2.001f * off;
    auto side = [&](float v) { return v == t ? 0 : v > t ? (v - t > off2 ? 1 : 0) : (t - v > off2 ? -1 : 0); };      // 0: near
    uint32_t surely = 0;
    for (uint32_t i = tid; i < count; i += N) {
        const int w = side(score(i));
        surely += w > 0;
        if (w == 0) {
            const uint32_t at = atomicAdd(&s.count[1], 1u);
            if (at < kClose) s.close[at] = i;
        }
    }
#pragma unroll
    for (int m = 32; m; m >>= 1) surely += (uint32_t)__shfl_xor((int)surely, m);
    if (!lane) atomicAdd(&s.count[0], surely);
    __syncthreads();
    const uint32_t close = s.count[1], need = want - s.count[0];
    if (close == need || off2 == 0.0f || (t == -INFINITY && off2 < INFINITY)) {
        // all of those (where scores are exact, or the want-th has none: as many as are wanted, the lowest first)
        write_in_order<N>(s, count, x.lo, need, [&](uint32_t i) { return side(score(i)); }, to + a.n_first);
        return;
    }
    if (close <= kClose) {
        // ranked in 64 bits, equal ones by their number
        for (uint32_t i = wave; i < close; i += N / 64u) {
            const uint64_t o = exact_order<T>(a, q, token, head, x.lo + s.close[i]);
            if (!lane) s.order[i] = o;
        }
        __syncthreads();
        if (tid < close) {
            const uint64_t o = s.order[tid];
            const uint32_t mine = s.close[tid];
            uint32_t before = 0;
            for (uint32_t i = 0; i < close; i++) before += s.order[i] > o || (s.order[i] == o && s.close[i] < mine);
            const float v = before < need ? INFINITY : -INFINITY;
            if (in_lds) own[mine] = v;
            else left[mine][0] = v;
        }
        __threadfence_block();
        __syncthreads();
        write_in_order<N>(s, count, x.lo, 0u, [&](uint32_t i) { const float v = score(i); return v == INFINITY ? 1 : v == -INFINITY ? -1 : side(v) > 0 ? 1 : -1; }, to + a.n_first);
        return;
    }
    // more than there is room for: those near in 64 bits through memory, what is sure at either end
    uint64_t *const keys = a.keys + (int64_t)item * a.stride + x.lo;
    for (uint32_t i = wave; i < count; i += N / 64u) {
        const int w = side(score(i));
        const uint64_t o = w > 0 ? ~0ull : w < 0 ? 0ull : exact_order<T>(a, q, token, head, x.lo + i);
        if (!lane) keys[i] = o;
    }
    __threadfence_block();
    __syncthreads();
    uint64_t prefix;
    int shift;
    find_rank<N, uint64_t>(s, count, want, false, [&](uint32_t i) { return keys[i]; }, prefix, shift, rank);
    write_in_order<N>(s, count, x.lo, rank, [&](uint32_t i) { const uint64_t k = keys[i] >> shift; return k > prefix ? 1 : k == prefix ? 0 : -1; }, to + a.n_first);
}

// N threads per new token and head.  Scores in fp32 (made here, FUSED; else score_kernel has left them in memory), of which LDS holds as many
// as it has room for; which of 2048 even steps between the least and the largest the want-th largest lies in, and which it is of those;
// what lies nearer to it than the scores' error once more in 64 bits; then the blocks in order.  Which blocks are taken hangs on no rounding
// but of the 64 bits, and on no order of sums.
//
// 128 tokens over 512-8192 tokens in blocks of 16, 8 heads x 128: 74 MB of bounds in 27 us.  4.5 go by until the lengths are there, 18 to the
// last score (4.1 TB/s, in pieces of 256 bytes from all over; the arithmetic takes 5 beside that), 5 from there on.  Scores in 64 bits throughout
// took 47 us and 8 for the choice (the queries came out of LDS), digits of 11 bits for the choice 8 us more than even steps do, 512 threads 32.
// Four contexts of 60000-120000 tokens, 4 heads x 64: scores 6.8 us, choice 14.5, of which 64 bits 4 (three loads that wait for each other).
template <typename T, int DP, bool FUSED, uint32_t N>
__global__ __launch_bounds__(N) __attribute__((amdgpu_waves_per_eu(DP <= 128 ? 4 : 2))) void pick_kernel(SelectArgs a)
{
    __shared__ PickShared s;
    extern __shared__ float own[];              // scores
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = (uint32_t)__builtin_amdgcn_readfirstlane(tid >> 6);
    // Workgroups go to the eight XCDs in turn: with FUSED the heads of a token follow each other on one of them, whose scales of a block
    // lie in one line (128 tokens 27.8 us, 29.2 without).
    uint32_t token, head;
    if constexpr (FUSED) {
        const uint32_t nth = blockIdx.x >> 3;
        token = nth / a.c.heads, head = nth - token * a.c.heads;
        token = 8u * token + (blockIdx.x & 7u);
        if (token >= a.b.total_new) return;
    } else {
        token = blockIdx.x / a.c.heads, head = blockIdx.x - token * a.c.heads;
    }
    const uint32_t item = token * a.c.heads + head;
    const Request q = token_of(a.b, a.c, (int)token);
    if (q.fresh <= 0) return;                   // no request's
    const Choice x = choice_of(a, q);
    int32_t *const to = a.blocks + (int64_t)item * a.n_select;
    if (x.seen <= a.n_select) {
        for (uint32_t i = tid; i < a.n_select; i += N) to[i] = i < x.seen ? (int32_t)i : -1;
        return;
    }
    const uint32_t want = a.n_select - a.n_first - a.n_recent, count = x.hi - x.lo;
    for (uint32_t i = tid; i < a.n_first; i += N) to[i] = (int32_t)i;
    for (uint32_t i = tid; i < a.n_recent; i += N) to[a.n_first + want + i] = (int32_t)(x.hi + i);
    if (!want) return;
    f32x2 *const left = a.scores + (int64_t)item * a.stride + x.lo;
    const bool in_lds = FUSED || a.stride <= kMostInLds;
    for (uint32_t i = tid; i < kPickBins; i += N) s.hist[i] = 0;
    if (tid < 3u) s.count[tid] = 0;
    // how far the scores may be off, the least and the largest of them
    float off = 0.0f, least = INFINITY, most = -INFINITY;
    auto look = [&](float v) { most = fmaxf(most, v), least = fminf(least, v == -INFINITY ? INFINITY : v); };
    if constexpr (FUSED) {
        Scorer<T, DP> scorer(a, q, token, head);
        // where all blocks lie first, in the scores' places
        for (uint32_t i = tid; i < count; i += N) own[i] = __int_as_float(entry_of(a.c, q.row, x.lo + i));
        for (uint32_t row0 = 0; row0 < a.group; row0 += 16u) {
            scorer.rows(row0);
            if (!row0) __syncthreads();
            uint32_t base = 16u * wave;
            if (base >= count) break;
            auto entries = [&](uint32_t from) {
                return [&, from](uint32_t i) {
                    i += from;
                    return i >= count ? -1 : row0 ? entry_of(a.c, q.row, x.lo + i) : __float_as_int(own[i]);
                };
            };
            auto tile = scorer.fetch(entries(base));
            for (;;) {
                const auto here = tile;
                const uint32_t next = base + N / 4u;
                if (next < count) tile = scorer.fetch(entries(next));
                float v = scorer.of(here);
                const uint32_t i = base + 4u * (uint32_t)scorer.g + (uint32_t)scorer.col;
                if (scorer.col < 4 && i < count) {
                    if (row0) v = fmaxf(v, own[i]);
                    if (row0 + 16u >= a.group) off = fmaxf(off, off_of(scorer.off, v, here.scale)), v = counted(v, here.scale), look(v);
                    own[i] = v;
                }
                if (next >= count) break;
                base = next;
            }
        }
    } else {
        constexpr uint32_t kAhead = 8;
        for (uint32_t i0 = tid; i0 < count; i0 += kAhead * N) {
            f32x2 v[kAhead];
#pragma unroll
            for (uint32_t k = 0; k < kAhead; k++) v[k] = left[min(i0 + k * N, count - 1u)];
#pragma unroll
            for (uint32_t k = 0; k < kAhead; k++) {
                off = fmaxf(off, v[k][1]);
                look(v[k][0]);
                if (in_lds && i0 + k * N < count) own[i0 + k * N] = v[k][0];
            }
        }
    }
    choose<T, N>(s, a, q, token, head, x, own, in_lds, off, most, least);
}

// Several tokens of a request at a time, one pass over the bounds for all of them: the columns of the products are rows of 16 / each tokens, their
// scores lie in LDS one token's behind the other's, and the choices follow each other.
template <typename T, int DP, uint32_t N>
__global__ __launch_bounds__(N) __attribute__((amdgpu_waves_per_eu(DP <= 64 ? 4 : DP <= 128 ? 3 : 2))) void pick_several_kernel(SelectArgs a)
{
    __shared__ PickShared s;
    extern __shared__ float scores[];
    const uint32_t tid = threadIdx.x, wave = (uint32_t)__builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t nth = blockIdx.x / a.c.heads, head = blockIdx.x - nth * a.c.heads, first = nth * a.several;
    const uint32_t last = min(first + a.several, a.b.total_new), want = a.n_select - a.n_first - a.n_recent, lo = a.n_first;
    const uint32_t each = a.group <= 1u ? 1u : 2u << (31 - __builtin_clz(a.group - 1u));
    for (uint32_t t0 = first; t0 < last;) {
        const Request r = request_with(a.b, a.c, (int)t0);
        const int before = (int)t0 - r.start;
        if (before < 0 || before >= r.fresh) {                  // no request's
            t0++;
            continue;
        }
        const uint32_t n = min(last - t0, (uint32_t)(r.fresh - before));
        auto nth_of = [&](uint32_t y) { return Request{r.row, min(r.len, max(0, r.len - r.fresh + before + (int)y + 1)), (int)(t0 + y), 1}; };
        auto count_of = [&](uint32_t y) {
            const Choice x = choice_of(a, nth_of(y));
            return x.hi - x.lo;
        };
        __syncthreads();
        if (tid < 16u) s.off[tid] = 0;
        const uint32_t most_blocks = want ? count_of(n - 1u) : 0u;
        if (most_blocks) {
            Scorer<T, DP> scorer(a, r, t0, head);
            for (uint32_t i = tid; i < most_blocks; i += N) scores[i] = __int_as_float(entry_of(a.c, r.row, lo + i));
            const uint32_t own = (uint32_t)scorer.col / each, row = (uint32_t)scorer.col & (each - 1u);
            const float wide = largest_of(scorer.column(t0 + min(own, n - 1u), min(row, a.group - 1u)), each);
            const uint32_t count = own < n ? count_of(min(own, n - 1u)) : 0u;
            float *const to = scores + own * a.stride;
            __syncthreads();
            uint32_t base = 16u * wave;
            auto entries = [&](uint32_t from) {
                return [&, from](uint32_t i) { return i + from >= most_blocks ? -1 : __float_as_int(scores[i + from]); };
            };
            if (base < most_blocks) {
                auto tile = scorer.fetch(entries(base));
                float off = 0.0f;
                for (;;) {
                    const auto here = tile;
                    const uint32_t next = base + N / 4u;
                    if (next < most_blocks) tile = scorer.fetch(entries(next));
                    const f32x4 z = scorer.products(here);
                    float v[4];
#pragma unroll
                    for (int i = 0; i < 4; i++) v[i] = largest_of(z[i] == z[i] ? z[i] : INFINITY, each);
                    const uint32_t block = base + 4u * (uint32_t)scorer.g;
                    if (each >= 4u) {           // one of four lanes' blocks
                        const float w = row & 2u ? row & 1u ? v[3] : v[2] : row & 1u ? v[1] : v[0];
                        if (row < 4u && block + row < count) to[block + row] = counted(w, here.scale), off = fmaxf(off, off_of(wide, w, here.scale));
                    } else {
                        const int x = __float_as_int(here.scale);
                        const float scale[4] = {__int_as_float(__builtin_amdgcn_update_dpp(0, x, 0x00, 0xF, 0xF, false)),
                                                __int_as_float(__builtin_amdgcn_update_dpp(0, x, 0x55, 0xF, 0xF, false)),
                                                __int_as_float(__builtin_amdgcn_update_dpp(0, x, 0xAA, 0xF, 0xF, false)),
                                                __int_as_float(__builtin_amdgcn_update_dpp(0, x, 0xFF, 0xF, 0xF, false))};
#pragma unroll
                        for (uint32_t i = 0; i < 4u; i++)
                            if ((i & (each - 1u)) == row && block + i < count) to[block + i] = counted(v[i], scale[i]), off = fmaxf(off, off_of(wide, v[i], scale[i]));
                    }
                    if (next >= most_blocks) break;
                    base = next;
                }
                if (own < n) atomicMax(&s.off[own], __float_as_uint(off));
            }
        }
        for (uint32_t y = 0; y < n; y++) {
            const Request q = nth_of(y);
            const Choice x = choice_of(a, q);
            int32_t *const to = a.blocks + ((int64_t)(t0 + y) * a.c.heads + head) * a.n_select;
            if (x.seen <= a.n_select) {
                for (uint32_t i = tid; i < a.n_select; i += N) to[i] = i < x.seen ? (int32_t)i : -1;
                continue;
            }
            for (uint32_t i = tid; i < a.n_first; i += N) to[i] = (int32_t)i;
            for (uint32_t i = tid; i < a.n_recent; i += N) to[a.n_first + want + i] = (int32_t)(x.hi + i);
            if (!want) continue;
            __syncthreads();
            for (uint32_t i = tid; i < kPickBins; i += N) s.hist[i] = 0;
            if (tid < 3u) s.count[tid] = 0;
            float *const own = scores + y * a.stride;
            float least = INFINITY, most = -INFINITY;
            for (uint32_t i = tid; i < x.hi - x.lo; i += N) {
                const float v = own[i];
                most = fmaxf(most, v), least = fminf(least, v == -INFINITY ? INFINITY : v);
            }
            choose<T, N>(s, a, q, t0 + y, head, x, own, true, __uint_as_float(s.off[y]), most, least);
        }
        t0 += n;
    }
}

template <typename T, int DP> static hipError_t select(SelectArgs a, hipStream_t s)
{
    constexpr uint32_t kMany = DP <= 128 ? 1024 : 512;
    const uint64_t items = (uint64_t)a.b.total_new * a.c.heads, per = (a.stride + kBlocksAtOnce - 1u) / kBlocksAtOnce;
    const bool fused = selects_in_one(items, a.stride);
    // Many tokens of few requests: four of a request at a time (two, where eight query heads leave room for no more), while there are four workgroups for
    // every compute unit (two over many blocks, one of 256 elements) and their scores take no more LDS than leaves two (heads of 64: three) resident.
    // Measured (us, one at a time / so; requests x tokens x heads, query heads each, blocks): heads of 128, 1 x 512 x 8, 4, 1875 252 / 158, 4 x 256 x 8, 4,
    // 500 111 / 93, 1 x 2048 x 8, 8, 625 393 / 336, 4 x 190 x 16, 1, 3125 1214 / 673, 4 x 64 x 8, 4, 312 38 / 35, 1375 105 / 64, 6250 423 / 306; of 64, 4 x 190 x
    // 16, 4, 3200 776 / 490, 16 x 64 x 8, 1, 250 85 / 61, 4 x 40 x 8, 1, 1375 60 / 48; of 256, 16 x 64 x 8, 2, 250 222 / 135, 4 x 58 x 8, 4, 206 59 / 44, 3125
    // 422 / 221.  Fewer blocks, two at a time: 5 x 154 x 4, 7, 102 22 / 29, 4 x 172 x 8, 7, 283 75 / 79.  Fewer tokens: 2048 and heads of 128 with 62 blocks 28 / 34, 1600, two at a time, with 312 34 / 41, with 1625 110 / 105: one at a time.  Eight
    // took 140 where four take 111 (16 x 64 x 8, 1, 1000) and 54 where they take 61.
    a.several = 1u;
    if (fused && a.b.starts && a.group <= 8u && a.stride > a.n_select) {
        const uint64_t least = DP > 128 ? 256u : a.stride >= 300u ? 512u : 1024u;
        uint32_t several = a.group <= 4u ? 4u : 2u;
        while (several > 1u && (several * a.stride * 4u > (DP <= 64 ? 32768u : 53248u) || (uint64_t)several * a.b.n_reqs > a.b.total_new)) several /= 2u;
        if (items / several >= least && a.stride >= (several == 4u ? 48u : DP <= 128 ? 400u : 128u)) a.several = several;
    }
    const uint32_t lds = a.stride > a.n_select && a.stride <= kMostInLds ? a.stride * 4u : 0u;
    if (a.several > 1u) {
        const uint64_t groups = ((uint64_t)a.b.total_new + a.several - 1u) / a.several * a.c.heads;
        if (!launchable(groups, 256)) return hipErrorInvalidConfiguration;
        pick_several_kernel<T, DP, 256><<<(uint32_t)groups, 256, a.several * a.stride * 4u, s>>>(a);
        return hipGetLastError();
    }
    if (fused) {
        // Workgroups of eight wavefronts while all of them are resident, of four beyond (us, four / eight: 256, 500 18 / 16, 512, 500 22 / 22, 1024 of
        // up to 512 27 / 32).
        const uint64_t groups = ((uint64_t)a.b.total_new + 7u) / 8u * 8u * a.c.heads;
        if (!launchable(groups, items <= 512u ? 512 : 256)) return hipErrorInvalidConfiguration;
        if (items <= 512u) pick_kernel<T, DP, true, 512><<<(uint32_t)groups, 512, lds, s>>>(a);
        else pick_kernel<T, DP, true, 256><<<(uint32_t)groups, 256, lds, s>>>(a);
        return hipGetLastError();
    }
    if (!launchable(items, kMany) || (a.stride > a.n_select && !launchable(items * per, kScoreThreads))) return hipErrorInvalidConfiguration;
    if (a.stride > a.n_select) {
        score_kernel<T, DP><<<(uint32_t)(items * per), kScoreThreads, 0, s>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    pick_kernel<T, DP, false, kMany><<<(uint32_t)items, kMany, lds, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_select(const SelectArgs &a, uint32_t dtype, hipStream_t s)
{
    auto by_dim = [&](auto type) {
        typedef decltype(type) T;
        return a.c.dim <= 64 ? select<T, 64>(a, s) : a.c.dim <= 128 ? select<T, 128>(a, s) : select<T, 256>(a, s);
    };
    return dtype == DMI_DTYPE_BF16 ? by_dim(Bf16{}) : by_dim(Fp16{});
}

}  // namespace kv8
}  // namespace dmi
