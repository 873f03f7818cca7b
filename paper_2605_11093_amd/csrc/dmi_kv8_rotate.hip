// Kernels that write new tokens into the 8-bit KV cache with their positions' rotation, and the bounds of the blocks they reach.
#include "dmi_internal.h"
#include "dmi_kv8_long.h"
#include "dmi_kv8_rows.h"

#include <algorithm>

namespace dmi {
namespace kv8 {

// ---------------------------------------------------------------- which block
// The nth of the blocks that new tokens reach: of request `r`, or of all requests one behind the other (r < 0).
struct Reached {
    Request q;
    int block, lo, hi;                          // lo, hi: positions of its new tokens; lo >= hi: there is none
};
__device__ __forceinline__ Reached reached_by(const Batch &b, const Cache &c, int r, uint32_t nth)
{
    const uint32_t lane = threadIdx.x & 63u;
    Reached x{{0, 0, 0, 0}, 0, 0, 0};
    if (r < 0) {
        for (uint32_t n0 = 0;; n0 += 64u) {
            if (n0 >= b.n_reqs) return x;
            Request own{0, 0, 0, 0};
            if (n0 + lane < b.n_reqs) own = request_of(b, c, (int)(n0 + lane));
            const int begin = max(own.len - own.fresh, 0);
            const int reached = own.len > begin ? (int)(block_of(c, (uint32_t)(own.len - 1) >> 4) - block_of(c, (uint32_t)begin >> 4)) + 1 : 0;
            const int upto = lanes_scan(reached);
            const uint64_t behind = __ballot(upto > (int)nth);
            if (!behind) {
                nth -= (uint32_t)__builtin_amdgcn_readlane(upto, 63);
                continue;
            }
            const int in = __ffsll((unsigned long long)behind) - 1;
            if (in) nth -= (uint32_t)__builtin_amdgcn_readlane(upto, in - 1);
            x.q = request_in(own, in);
            break;
        }
    } else {
        x.q = request_of(b, c, r);
    }
    const int from = max(x.q.len - x.q.fresh, 0);
    x.block = (int)(block_of(c, (uint32_t)from >> 4) + nth);
    x.lo = max(from, (int)((uint32_t)x.block * c.bs));
    x.hi = min(x.q.len, (int)(((uint32_t)x.block + 1u) * c.bs));
    return x;
}

// How many of them a launch is made for, for every request or for all; the rule is launch_append's (a prompt of 8192 tokens among 63 single
// ones, for every request / counted: rotated 62.9 / 48.1 us, bounds 9.0 / 8.6).
struct Reach {
    uint64_t blocks;
    uint32_t reqs;
    bool counted;
};
static Reach reach_of(const Cache &c, const Batch &b)
{
    const uint32_t touched = (b.max_new + c.bs - 2u) / c.bs + 1u;
    const uint64_t all = (uint64_t)b.total_new / c.bs + 2u * (uint64_t)b.n_reqs;
    const bool counted = (uint64_t)touched * b.n_reqs > 2u * all;
    return {counted ? all : touched, counted ? 1u : b.n_reqs, counted};
}

// ---------------------------------------------------------------- append, rotated
// Sixteen elements of a row: two eights that are rotated together (the one is the pairs' x and the other their y where pairs are halves
// of the row apart; both neighbours where they are neighbours).
struct Place {
    uint32_t a, b;                              // the eights' first elements
    int pair;                                   // the first of eight pairs, -1: not rotated
};
__device__ __forceinline__ Place place_of(uint32_t sixteen, uint32_t rotary, bool neighbours)
{
    const uint32_t d = 16u * sixteen;
    if (d >= rotary) return {d, d + 8u, -1};
    if (neighbours) return {d, d + 8u, (int)(8u * sixteen)};
    return {8u * sixteen, 8u * sixteen + rotary / 2u, (int)(8u * sixteen)};
}

// Eight pairs turned, in F: fp64 for K and for queries in fp32, whose codes and elements then hang on no order of operations, fp32 for
// queries of 16 bits.
template <typename F, bool NEIGHBOURS> __device__ __forceinline__ void turn(float (&x)[16], const float *cos, const float *sin)
{
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
        const f32x4 c = *reinterpret_cast<const f32x4 *>(cos + i), s = *reinterpret_cast<const f32x4 *>(sin + i);
#pragma unroll
        for (int k = 0; k < 4; k++) {
            float &p = NEIGHBOURS ? x[2 * (i + k)] : x[i + k], &r = NEIGHBOURS ? x[2 * (i + k) + 1] : x[8 + i + k];
            const F u = p, v = r;
            p = (float)(u * (F)c[k] - v * (F)s[k]), r = (float)(u * (F)s[k] + v * (F)c[k]);
            if constexpr (sizeof(F) == 8) __builtin_amdgcn_sched_barrier(0);       // (all pairs at once would take all registers)
        }
    }
}

template <typename T> __device__ __forceinline__ void store8(T *p, const float *x);
template <> __device__ __forceinline__ void store8<Bf16Bits>(Bf16Bits *p, const float *x)
{
    typedef __bf16 two __attribute__((ext_vector_type(2)));
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; i++) w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x[2 * i], x[2 * i + 1]}), two));
    *reinterpret_cast<u32x4 *>(p) = w;
}
template <> __device__ __forceinline__ void store8<_Float16>(_Float16 *p, const float *x)
{
    typedef _Float16 two __attribute__((ext_vector_type(2)));
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; i++) w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x[2 * i], x[2 * i + 1]}), two));
    *reinterpret_cast<u32x4 *>(p) = w;
}
template <> __device__ __forceinline__ void store8<float>(float *p, const float *x)
{
    *reinterpret_cast<f32x4 *>(p) = f32x4{x[0], x[1], x[2], x[3]};
    *reinterpret_cast<f32x4 *>(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
}

template <typename T> constexpr uint32_t kAheadOf = sizeof(T) == 4 ? 2 : 4;     // sixteens of queries that are asked for before the first is used
constexpr uint32_t kTableBytes = 32768;         // cosines and sines in LDS: as many tokens as there is room for

// A workgroup per block that new tokens reach and a.each of its items: K of a head, V of a head, queries of a.q_each tokens (which lie in one
// piece).  Cosines and sines of the block's tokens are computed into LDS, in 64 bits (angles of far positions have no others), and every
// item takes them from there: once where those of all tokens fit in kTableBytes, else a part of the tokens at a time, again for every four items and
// each of their two passes (16 prompts of 1024 tokens, 369 MB: 4 heads x 256, blocks of 32 108 us, of 64 157; 8 x 128, of 64 106, of 128 155, of 1024 448).
// A wavefront has an item at a time, a lane the same sixteen of every few rows.  As in append_kernel the scale of K
// and V wants the largest of all the block's new elements first; what a lane can hold of them it does.
//
// Bound by memory where there is much: 32 prompts, 38014 tokens, K and V of 8 heads x 128 and queries of 32 in bf16, 857 MB in 180 us (4.8 TB/s;
// a copy reaches 5.2); single tokens by the chain of lengths, table, cosines, rows: 7.3 us.  Measured and not better for the prompts: one
// sixteen of queries under way at a time 268, four wavefronts a SIMD (spills) 362, three sixteens of K or V held 205, queries by head 186.
template <typename T, bool NEIGHBOURS>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(3))) void rotate_kernel(RotateArgs a)
{
    extern __shared__ __align__(16) float table[];
    constexpr int kHeld = 2;                    // sixteens of K or V a lane keeps
    constexpr uint32_t kAhead = kAheadOf<T>;
    const uint32_t lane = threadIdx.x & 63u, wave = (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Reached x = reached_by(a.b, a.c, a.counted ? -1 : (int)blockIdx.y, blockIdx.x / a.groups);
    if (x.lo >= x.hi) return;
    const uint32_t half = a.rotary / 2u, per_row = a.c.dim / 16u, stored = 2u * a.c.heads;
    const uint32_t items = stored + (a.q_heads ? (a.tokens + a.q_each - 1u) / a.q_each : 0u);
    const uint32_t first_item = blockIdx.x % a.groups * a.each, last_item = min(first_item + a.each, items);
    const int first = x.q.len - x.q.fresh;      // the first new token's place
    const int entry = entry_of(a.c, x.q.row, (uint32_t)x.block);
    const uint32_t slot0 = (uint32_t)x.lo - (uint32_t)x.block * a.c.bs;
    float *const cosines = table, *const sines = table + a.tokens * half;
    // this lane's row among those of a step, its sixteen of it
    const uint32_t of_step = 64u / per_row, row = lane / per_row, sixteen = lane - row * per_row;
    const Place rotated = place_of(sixteen, a.rotary, NEIGHBOURS), as_is = place_of(sixteen, 0u, NEIGHBOURS);

    struct Raw {
        Eight<T> a, b;
        __device__ __forceinline__ void load(const T *row, const Place &p) { a.load(row + p.a), b.load(row + p.b); }
        __device__ __forceinline__ void numbers(float (&v)[16]) const
        {
            a.numbers(*reinterpret_cast<float(*)[8]>(&v[0]));
            b.numbers(*reinterpret_cast<float(*)[8]>(&v[8]));
        }
    };
    auto fill = [&](int lo, int tokens) {
        for (uint32_t u = threadIdx.x; u < (uint32_t)tokens * half; u += 256u) {
            const uint32_t t = u / half, i = u - t * half;
            const int nth = x.q.start + lo - first + (int)t, at = a.positions ? a.positions[nth] : lo + (int)t;
            const double angle = (double)at * (double)a.freq[i];
            // less whole turns, whose length in two parts
            const double turns = __builtin_rint(angle * 0.15915494309189533577);
            const double rest = __builtin_fma(-turns, 2.4492935982947064e-16, __builtin_fma(-turns, 6.283185307179586477, angle));
            double s, c;
            sincospi(rest * 0.31830988618379067154, &s, &c);
            cosines[t * half + i] = (float)c;
            sines[t * half + i] = (float)s;
        }
    };

    const int tokens = x.hi - x.lo, chunk = (int)a.tokens;
    const bool one = tokens <= chunk;           // all cosines fit in LDS at once
    if (one) {
        fill(x.lo, tokens);
        __syncthreads();
    }
    for (uint32_t base = first_item; base < last_item; base += 4u) {
        const uint32_t item = base + wave;
        const bool mine = item < last_item, store = mine && item < stored && entry >= 0, turns_q = mine && item >= stored;
        const uint32_t kv = item & 1u, head = (item >> 1) % a.c.heads;
        const T *const src = static_cast<const T *>(a.x[kv].data) + (int64_t)(x.q.start + x.lo - first) * a.x[kv].row_stride + (int64_t)head * a.x[kv].head_stride;
        float *const scale_p = scale_at(a.c, (int)kv, max(entry, 0), head);
        const float had = store && slot0 ? *scale_p : 0.0f;
        const Place p = kv ? as_is : rotated;
        float held[kHeld][16];
        uint32_t largest = 0;
        float s = 0.0f, inv = 0.0f;
        bool exact = false;
        // twice over the tokens for K and V, the second time with their scale
        for (int pass = 0; pass < (one && !store ? 1 : 2); pass++) {
            for (int lo = 0; lo < tokens; lo += chunk) {
                const uint32_t here = (uint32_t)min(chunk, tokens - lo);
                if (!one) {
                    __syncthreads();            // (the cosines of the last chunk have been used)
                    fill(x.lo + lo, (int)here);
                    __syncthreads();
                }
                auto ask = [&](uint32_t t, Raw &r) { r.load(src + (int64_t)(lo + (int)t) * a.x[kv].row_stride, p); };
                auto have = [&](uint32_t t, const Raw &r, float (&v)[16]) {
                    r.numbers(v);
                    if (!kv && p.pair >= 0) turn<double, NEIGHBOURS>(v, cosines + t * half + (uint32_t)p.pair, sines + t * half + (uint32_t)p.pair);
                };
                auto look = [&](const float (&v)[16]) {
#pragma unroll
                    for (int i = 0; i < 16; i++) {
                        const uint32_t m = __float_as_uint(v[i]) & 0x7FFFFFFFu;
                        largest = max(largest, m < 0x7F800000u ? m : 0u);
                    }
                };
                auto put = [&](uint32_t t, const float (&v)[16]) {
                    float y[16];
#pragma unroll
                    for (int i = 0; i < 16; i++) y[i] = v[i] * inv;
                    if (!exact) {
#pragma unroll
                            for (int i = 0; i < 16; i++) {
                            y[i] = v[i] / s;
                            __builtin_amdgcn_sched_barrier(0);
                        }
                    }
                    uint8_t *const to = code_at(a.c, (int)kv, entry, slot0 + (uint32_t)lo + t, head);
                    *reinterpret_cast<u32x2 *>(to + p.a) = u32x2{to_codes(y[0], y[1], y[2], y[3]), to_codes(y[4], y[5], y[6], y[7])};
                    *reinterpret_cast<u32x2 *>(to + p.b) = u32x2{to_codes(y[8], y[9], y[10], y[11]), to_codes(y[12], y[13], y[14], y[15])};
                };
                if (store && row < of_step) {
                    if (one && pass == 0) {
                        Raw raw[kHeld];
#pragma unroll
                        for (uint32_t i = 0; i < kHeld; i++) ask(min(row + i * of_step, here - 1u), raw[i]);
#pragma unroll
                        for (uint32_t i = 0; i < kHeld; i++) {
                            have(min(row + i * of_step, here - 1u), raw[i], held[i]);
                            look(held[i]);      // (behind the last token that one again)
                        }
                    } else if (one) {
#pragma unroll
                        for (uint32_t i = 0; i < kHeld; i++)
                            if (row + i * of_step < here) put(row + i * of_step, held[i]);
                    }
                    for (uint32_t t = row + (one ? of_step * kHeld : 0u); t < here; t += of_step) {
                        Raw r;
                        float v[16];
                        ask(t, r);
                        have(t, r, v);
                        if (pass == 0) look(v);
                        else put(t, v);
                    }
                } else if (turns_q && pass == 0 && row < of_step) {
                    const uint32_t token0 = (item - stored) * a.q_each, rows = token0 < here ? min(a.q_each, here - token0) * a.q_heads : 0u;
                    const int64_t at0 = x.q.start + x.lo - first + lo;
                    auto locate = [&](uint32_t r, uint32_t &t, uint32_t &h) {
                        t = a.q_heads == 1u ? r : __umulhi(r, a.q_part);
                        h = r - t * a.q_heads;
                        t += token0;
                    };
                    for (uint32_t r0 = row; r0 < rows; r0 += kAhead * of_step) {
                        Raw raw[kAhead];
#pragma unroll
                        for (uint32_t i = 0; i < kAhead; i++) {
                            uint32_t t, h;
                            locate(min(r0 + i * of_step, rows - 1u), t, h);
                            raw[i].load(static_cast<const T *>(a.q.data) + (at0 + t) * a.q.row_stride + (int64_t)h * a.q.head_stride, rotated);
                        }
#pragma unroll
                        for (uint32_t i = 0; i < kAhead; i++) {
                            if (r0 + i * of_step >= rows) break;
                            uint32_t t, h;
                            locate(r0 + i * of_step, t, h);
                            float v[16];
                            raw[i].numbers(v);
                            typedef std::conditional_t<sizeof(T) == 4, double, float> F;
                            if (rotated.pair >= 0) turn<F, NEIGHBOURS>(v, cosines + t * half + (uint32_t)rotated.pair, sines + t * half + (uint32_t)rotated.pair);
                            T *const to = static_cast<T *>(a.q_out.data) + (at0 + t) * a.q_out.row_stride + (int64_t)h * a.q_out.head_stride;
                            store8<T>(to + rotated.a, v);
                            store8<T>(to + rotated.b, v + 8);
                        }
                    }
                }
            }
            if (store && pass == 0) {
#pragma unroll
                for (int m = 32; m; m >>= 1) largest = max(largest, (uint32_t)__shfl_xor((int)largest, m));
                // (append_kernel has the reasons)
                const int exponent = max((int)(largest >> 23) - 8 + ((largest & 0x7FFFFFu) > 0x600000u ? 1 : 0), 127 - 100);
                const float need = __uint_as_float((uint32_t)exponent << 23);
                s = fmaxf(need, had);
                exact = s == need;
                inv = __uint_as_float((uint32_t)(254 - exponent) << 23);
                if (slot0 && s != had) {        // what the block held already
                    const float f = had / s;
                    const uint32_t eights = a.c.dim / 8u;
                    for (uint32_t u = lane; u < slot0 * eights; u += 64u) {
                        u32x2 *at = reinterpret_cast<u32x2 *>(code_at(a.c, (int)kv, entry, u / eights, head) + (u % eights) * 8u);
                        u32x2 w = *at;
                        w[0] = scaled_codes(w[0], f);
                        w[1] = scaled_codes(w[1], f);
                        *at = w;
                    }
                }
            }
        }
        if (store && !lane) *scale_p = s;
    }
}

hipError_t launch_rotate(RotateArgs a, uint32_t dtype, hipStream_t s)
{
    const Reach reach = reach_of(a.c, a.b);
    a.counted = reach.counted;
    const uint32_t half = a.rotary / 2u;
    a.tokens = std::max(1u, std::min({a.c.bs, a.b.max_new, kTableBytes / (8u * half)}));
    // Few blocks: their items over more workgroups, each of which computes the block's cosines for itself.
    const uint32_t ahead = (dtype == DMI_DTYPE_FP32 ? kAheadOf<float> : kAheadOf<_Float16>) * (64u / (a.c.dim / 16u));
    a.q_each = std::max(1u, 2u * ahead / std::max(1u, a.q_heads));
    a.q_part = a.q_heads > 1u ? (uint32_t)(((1ull << 32) + a.q_heads - 1u) / a.q_heads) : 0u;
    const uint32_t items = 2u * a.c.heads + (a.q_heads ? (a.tokens + a.q_each - 1u) / a.q_each : 0u);
    const uint64_t blocks = reach.blocks * reach.reqs;
    a.each = (uint32_t)std::min<uint64_t>((items + 3u) & ~3u, std::max<uint64_t>(4u, (blocks * items / 2048u + 3u) & ~3ull));
    a.groups = (items + a.each - 1u) / a.each;
    const uint64_t groups = reach.blocks * a.groups;
    if (!launchable(groups, 256)) return hipErrorInvalidConfiguration;
    const dim3 grid((uint32_t)groups, reach.reqs);
    const uint32_t lds = a.tokens * half * 8u;
    auto launch = [&](auto type) {
        typedef decltype(type) T;
        if (a.neighbours) rotate_kernel<T, true><<<grid, 256, lds, s>>>(a);
        else rotate_kernel<T, false><<<grid, 256, lds, s>>>(a);
        return hipGetLastError();
    };
    return dtype == DMI_DTYPE_BF16 ? launch(Bf16Bits{}) : dtype == DMI_DTYPE_FP16 ? launch((_Float16)0) : launch(0.0f);
}

// ---------------------------------------------------------------- bounds
// Codes in an order of unsigned bytes: those of negative numbers reversed, below the others.  NaN is at either end: 0xFF (of positive
// sign), 0x00.
__device__ __forceinline__ uint32_t ordered(uint32_t w)
{
    const uint32_t sign = w >> 7 & 0x01010101u;
    return w ^ (sign * 0x7Fu | 0x80808080u);
}
__device__ __forceinline__ uint32_t unordered(uint32_t w)
{
    const uint32_t sign = ~w >> 7 & 0x01010101u;
    return w ^ (sign * 0x7Fu | 0x80808080u);
}
// The top bit of every byte that is 255
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) { return (w & 0x7F7F7F7Fu) + 0x01010101u & w & 0x80808080u; }

// The largest and the least of bytes, of each of a word's four: as the upper bytes of 16-bit numbers, whose order they decide, the second and
// fourth where they are, the first and third shifted there.
struct Extremes {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    u16x2 most[2] = {{0, 0}, {0, 0}}, least[2] = {{0xFFFF, 0xFFFF}, {0xFFFF, 0xFFFF}};
    __device__ __forceinline__ void take(uint32_t for_most, uint32_t for_least)
    {
#pragma unroll
        for (int i = 0; i < 2; i++) {
            most[i] = __builtin_elementwise_max(most[i], __builtin_bit_cast(u16x2, i ? for_most << 8 : for_most));
            least[i] = __builtin_elementwise_min(least[i], __builtin_bit_cast(u16x2, i ? for_least << 8 : for_least));
        }
    }
    static __device__ __forceinline__ uint32_t bytes(const u16x2 (&x)[2])
    {
        return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, x[0]), __builtin_bit_cast(uint32_t, x[1]), 0x07030501u);
    }
};

// A wavefront per block that new tokens reach and 64 places of its heads' rows, a lane 16 elements of every token (of every few, where the
// heads have fewer places): what the wavefront reads of a token lies in one piece where heads follow each other, and no extreme has to cross
// lanes.  Bound by memory where there is much: 32 prompts, 2200 blocks of 16 x 8 x 128, 40 MB in 10.5 us (3.8 TB/s; 21 us with a wavefront a
// head, whose lanes shared a token's elements: vector instructions); single tokens of 128 requests 4.2 us, loads that wait for each other.
__global__ __launch_bounds__(256) void bound_kernel(BoundArgs a)
{
    const uint32_t lane = threadIdx.x & 63u, item = blockIdx.x * 4u + (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t wide = a.c.dim / 16u, places = a.c.heads * wide, parts = (places + 63u) / 64u, nth = item / parts;
    if (!a.counted && nth >= a.touched) return;
    const Reached x = reached_by(a.b, a.c, a.counted ? -1 : (int)blockIdx.y, nth);
    if (x.lo >= x.hi) return;
    const int entry = entry_of(a.c, x.q.row, (uint32_t)x.block);
    if (entry < 0) return;
    const uint32_t tokens = (uint32_t)x.hi - (uint32_t)x.block * a.c.bs, each = min(places, 64u), teams = 64u / each, team = lane / each;
    const uint32_t place = (item - nth * parts) * 64u + lane - team * each, head = place / wide, d = 16u * (place - head * wide);
    const bool there = team < teams && place < places;
    Extremes e[4];
    if (there) {
        constexpr uint32_t kAhead = 8;
        const uint8_t *const from = code_at(a.c, 0, entry, 0, head) + d;
        for (uint32_t t = team; t < tokens; t += kAhead * teams) {
            u32x4 w[kAhead];
#pragma unroll
            for (uint32_t i = 0; i < kAhead; i++) w[i] = *reinterpret_cast<const u32x4 *>(from + (int64_t)min(t + i * teams, tokens - 1u) * a.c.slot_stride);
#pragma unroll
            for (uint32_t i = 0; i < kAhead; i++)
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    const uint32_t o = ordered(w[i][k]);
                    e[k].take(o, o);
                }
        }
    }
    // over the teams: those behind hand theirs to those in front (a last one that has no partner keeps its own)
    for (uint32_t n = teams; n > 1u;) {
        const uint32_t half = (n + 1u) / 2u;
#pragma unroll
        for (int k = 0; k < 4; k++) {
            const uint32_t most = (uint32_t)__shfl((int)Extremes::bytes(e[k].most), (int)(lane + half * each));
            const uint32_t least = (uint32_t)__shfl((int)Extremes::bytes(e[k].least), (int)(lane + half * each));
            if (team + half < n) e[k].take(most, least);
        }
        n = half;
    }
    if (team || !there) return;
    uint8_t *const to = a.bounds + (int64_t)entry * a.bounds_block_stride + (int64_t)head * a.bounds_head_stride + d;
    u32x4 low, high;
#pragma unroll
    for (int k = 0; k < 4; k++) {
        high[k] = Extremes::bytes(e[k].most), low[k] = Extremes::bytes(e[k].least);
        const uint32_t all = ((nan_bytes(high[k]) | nan_bytes(~low[k])) >> 7) * 0xFFu;
        high[k] = (unordered(high[k]) & ~all) | (0x7F7F7F7Fu & all);
        low[k] = (unordered(low[k]) & ~all) | (0x7F7F7F7Fu & all);
    }
    *reinterpret_cast<u32x4 *>(to) = low;
    *reinterpret_cast<u32x4 *>(to + a.c.dim) = high;
}

hipError_t launch_bound(BoundArgs a, hipStream_t s)
{
    const Reach reach = reach_of(a.c, a.b);
    a.counted = reach.counted;
    a.touched = (uint32_t)std::min<uint64_t>(reach.blocks, 0xffffffffu);
    const uint64_t groups = (reach.blocks * ((a.c.heads * (a.c.dim / 16u) + 63u) / 64u) + 3u) / 4u;
    if (!launchable(groups, 256)) return hipErrorInvalidConfiguration;
    bound_kernel<<<dim3((uint32_t)groups, reach.reqs), 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace kv8
}  // namespace dmi
