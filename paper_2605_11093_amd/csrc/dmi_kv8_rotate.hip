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

// How many of them a launch is made for, for every request or for all; the rule is launch_append's.
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

// Eight pairs turned, in F: fp64 for K, whose scale and codes then hang on no order of operations, and fp32 for queries of 16 bits.
template <typename F> __device__ __forceinline__ void turn(float (&x)[16], const float *cos, const float *sin, bool neighbours)
{
    float c[8], s[8];
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
        *reinterpret_cast<f32x4 *>(c + i) = *reinterpret_cast<const f32x4 *>(cos + i);
        *reinterpret_cast<f32x4 *>(s + i) = *reinterpret_cast<const f32x4 *>(sin + i);
    }
    float y[16];
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const F u = neighbours ? x[2 * i] : x[i], v = neighbours ? x[2 * i + 1] : x[8 + i];
        const float a = (float)(u * (F)c[i] - v * (F)s[i]), b = (float)(u * (F)s[i] + v * (F)c[i]);
        y[i] = a, y[8 + i] = b;
    }
#pragma unroll
    for (int i = 0; i < 8; i++) {
        x[neighbours ? 2 * i : i] = y[i];
        x[neighbours ? 2 * i + 1 : 8 + i] = y[8 + i];
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

constexpr uint32_t kQueryHeads = 4;             // query heads that a wavefront takes at a time
constexpr uint32_t kTableBytes = 32768;         // cosines and sines in LDS: as many tokens as they are room for

// A workgroup per block that new tokens reach and a.each of its items: K of a head, V of a head, four heads of queries.  Cosines and sines
// of the block's tokens are computed once into LDS, in 64 bits (angles of far positions have no others), and every item takes them from
// there; a wavefront has an item at a time.  As in append_kernel the scale of K and V wants the largest of all the block's new elements
// first; what a lane can hold of them it does.
template <typename T>
__global__ __launch_bounds__(256) void rotate_kernel(RotateArgs a)
{
    extern __shared__ __align__(16) float table[];
    constexpr int kHeld = 2;                    // sixteens a lane keeps
    const uint32_t lane = threadIdx.x & 63u, wave = (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Reached x = reached_by(a.b, a.c, a.counted ? -1 : (int)blockIdx.y, blockIdx.x / a.groups);
    if (x.lo >= x.hi) return;
    const uint32_t half = a.rotary / 2u, per_row = a.c.dim / 16u, stored = 2u * a.c.heads;
    const uint32_t items = stored + (a.q_heads + kQueryHeads - 1u) / kQueryHeads;
    const uint32_t first_item = blockIdx.x % a.groups * a.each, last_item = min(first_item + a.each, items);
    const int first = x.q.len - x.q.fresh;      // the first new token's place
    const int entry = entry_of(a.c, x.q.row, (uint32_t)x.block);
    const uint32_t slot0 = (uint32_t)x.lo - (uint32_t)x.block * a.c.bs;
    float *const cosines = table, *const sines = table + a.tokens * half;
    const bool neighbours = a.neighbours;

    auto fill = [&](int lo, int tokens) {
        for (uint32_t u = threadIdx.x; u < (uint32_t)tokens * half; u += 256u) {
            const uint32_t t = u / half, i = u - t * half;
            const int row = x.q.start + lo - first + (int)t, at = a.positions ? a.positions[row] : lo + (int)t;
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
    // a lane's sixteen of a row as numbers, rotated where it is
    auto numbers = [&](const T *row, const Place &p, float (&v)[16]) {
        Eight<T> e, f;
        e.load(row + p.a);
        f.load(row + p.b);
        e.numbers(*reinterpret_cast<float(*)[8]>(&v[0]));
        f.numbers(*reinterpret_cast<float(*)[8]>(&v[8]));
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
        float held[kHeld][16];
        uint32_t largest = 0;
        float s = 0.0f, inv = 0.0f;
        bool exact = false;
        // twice over the tokens for K and V, the second time with their scale
        for (int pass = 0; pass < (one && !store ? 1 : 2); pass++) {
            for (int lo = 0; lo < tokens; lo += chunk) {
                const int here = min(chunk, tokens - lo);
                if (!one) {
                    __syncthreads();            // (the cosines of the last chunk have been used)
                    fill(x.lo + lo, here);
                    __syncthreads();
                }
                const uint32_t units = (uint32_t)here * per_row;
                auto get = [&](uint32_t u, float (&v)[16]) {
                    const uint32_t t = u / per_row;
                    const Place p = place_of(u - t * per_row, kv ? 0u : a.rotary, neighbours);
                    numbers(src + (int64_t)(lo + (int)t) * a.x[kv].row_stride, p, v);
                    if (p.pair >= 0) {
                        const uint32_t at = t * half + (uint32_t)p.pair;
                        if (neighbours) turn<double>(v, cosines + at, sines + at, true);
                        else turn<double>(v, cosines + at, sines + at, false);
                    }
                };
                auto look = [&](const float (&v)[16]) {
#pragma unroll
                    for (int i = 0; i < 16; i++) {
                        const uint32_t m = __float_as_uint(v[i]) & 0x7FFFFFFFu;
                        largest = max(largest, m < 0x7F800000u ? m : 0u);
                    }
                };
                auto put = [&](uint32_t u, const float (&v)[16]) {
                    const uint32_t t = u / per_row;
                    const Place p = place_of(u - t * per_row, kv ? 0u : a.rotary, neighbours);
                    float y[16];
#pragma unroll
                    for (int i = 0; i < 16; i++) y[i] = exact ? v[i] * inv : v[i] / s;
                    uint8_t *const to = code_at(a.c, (int)kv, entry, slot0 + (uint32_t)lo + t, head);
                    *reinterpret_cast<u32x2 *>(to + p.a) = u32x2{to_codes(y[0], y[1], y[2], y[3]), to_codes(y[4], y[5], y[6], y[7])};
                    *reinterpret_cast<u32x2 *>(to + p.b) = u32x2{to_codes(y[8], y[9], y[10], y[11]), to_codes(y[12], y[13], y[14], y[15])};
                };
                if (store && pass == 0) {
                    if (one) {
#pragma unroll
                        for (int i = 0; i < kHeld; i++)
                            if (lane + 64u * i < units) get(lane + 64u * i, held[i]), look(held[i]);
                    }
                    for (uint32_t u = lane + (one ? 64u * kHeld : 0u); u < units; u += 64u) {
                        float v[16];
                        get(u, v);
                        look(v);
                    }
                } else if (store) {
                    if (one) {
#pragma unroll
                        for (int i = 0; i < kHeld; i++)
                            if (lane + 64u * i < units) put(lane + 64u * i, held[i]);
                    }
                    for (uint32_t u = lane + (one ? 64u * kHeld : 0u); u < units; u += 64u) {
                        float v[16];
                        get(u, v);
                        put(u, v);
                    }
                } else if (turns_q && pass == 0) {
                    const uint32_t head0 = (item - stored) * kQueryHeads, heads = min(kQueryHeads, a.q_heads - head0);
                    for (uint32_t u = lane; u < units * heads; u += 64u) {
                        const uint32_t t = u / (per_row * heads), w = u - t * per_row * heads, h = w / per_row;
                        const Place p = place_of(w - h * per_row, a.rotary, neighbours);
                        const int64_t row = x.q.start + x.lo - first + lo + (int)t;
                        float v[16];
                        numbers(static_cast<const T *>(a.q.data) + row * a.q.row_stride + (int64_t)(head0 + h) * a.q.head_stride, p, v);
                        if (p.pair >= 0) {
                            typedef std::conditional_t<sizeof(T) == 4, double, float> F;
                            const uint32_t at = t * half + (uint32_t)p.pair;
                            if (neighbours) turn<F>(v, cosines + at, sines + at, true);
                            else turn<F>(v, cosines + at, sines + at, false);
                        }
                        T *const to = static_cast<T *>(a.q_out.data) + row * a.q_out.row_stride + (int64_t)(head0 + h) * a.q_out.head_stride;
                        store8<T>(to + p.a, v);
                        store8<T>(to + p.b, v + 8);
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
                        u32x2 *p = reinterpret_cast<u32x2 *>(code_at(a.c, (int)kv, entry, u / eights, head) + (u % eights) * 8u);
                        u32x2 w = *p;
                        w[0] = scaled_codes(w[0], f);
                        w[1] = scaled_codes(w[1], f);
                        *p = w;
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
    const uint32_t items = 2u * a.c.heads + (a.q_heads + kQueryHeads - 1u) / kQueryHeads;
    const uint64_t blocks = reach.blocks * reach.reqs;
    a.each = (uint32_t)std::min<uint64_t>((items + 3u) & ~3u, std::max<uint64_t>(4u, (blocks * items / 2048u + 3u) & ~3ull));
    a.groups = (items + a.each - 1u) / a.each;
    const uint64_t groups = reach.blocks * a.groups;
    if (!launchable(groups, 256)) return hipErrorInvalidConfiguration;
    const dim3 grid((uint32_t)groups, reach.reqs);
    const uint32_t lds = a.tokens * half * 8u;
    switch (dtype) {
    case DMI_DTYPE_BF16: rotate_kernel<Bf16Bits><<<grid, 256, lds, s>>>(a); break;
    case DMI_DTYPE_FP16: rotate_kernel<_Float16><<<grid, 256, lds, s>>>(a); break;
    default: rotate_kernel<float><<<grid, 256, lds, s>>>(a); break;
    }
    return hipGetLastError();
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
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
// The larger of two words' bytes, each
__device__ __forceinline__ uint32_t larger(uint32_t x, uint32_t y)
{
    const u16x2 a = __builtin_bit_cast(u16x2, x & 0x00FF00FFu), b = __builtin_bit_cast(u16x2, y & 0x00FF00FFu);
    const u16x2 c = __builtin_bit_cast(u16x2, x & 0xFF00FF00u), d = __builtin_bit_cast(u16x2, y & 0xFF00FF00u);
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(a, b)) | __builtin_bit_cast(uint32_t, __builtin_elementwise_max(c, d));
}

// A wavefront per block that new tokens reach and head: a lane has 16 elements of every few tokens, as words whose bytes compare like the
// numbers (the least as the largest of what is left to 255).
__global__ __launch_bounds__(256) void bound_kernel(BoundArgs a)
{
    const uint32_t lane = threadIdx.x & 63u, item = blockIdx.x * 4u + (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t head = item % a.c.heads;
    if (!a.counted && item / a.c.heads >= a.touched) return;
    const Reached x = reached_by(a.b, a.c, a.counted ? -1 : (int)blockIdx.y, item / a.c.heads);
    if (x.lo >= x.hi) return;
    const int entry = entry_of(a.c, x.q.row, (uint32_t)x.block);
    if (entry < 0) return;
    const uint32_t tokens = (uint32_t)x.hi - (uint32_t)x.block * a.c.bs, wide = a.c.dim / 16u, teams = 64u / wide;
    const uint32_t team = lane / wide, d = 16u * (lane - team * wide);
    u32x4 low = {0u, 0u, 0u, 0u}, high = low;
    auto take = [&](const u32x4 &w) {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const uint32_t o = ordered(w[i]);
            high[i] = larger(high[i], o);
            low[i] = larger(low[i], ~o);
        }
    };
    if (team < teams) {
        constexpr uint32_t kAhead = 4;
        for (uint32_t t = team; t < tokens; t += kAhead * teams) {
            u32x4 w[kAhead];
#pragma unroll
            for (uint32_t i = 0; i < kAhead; i++) w[i] = *reinterpret_cast<const u32x4 *>(code_at(a.c, 0, entry, min(t + i * teams, tokens - 1u), head) + d);
#pragma unroll
            for (uint32_t i = 0; i < kAhead; i++) take(w[i]);
        }
    }
    // over the teams: those behind hand theirs to those in front (a last one that has no partner keeps its own)
    for (uint32_t n = teams; n > 1u;) {
        const uint32_t half = (n + 1u) / 2u;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const uint32_t h = (uint32_t)__shfl((int)high[i], (int)(lane + half * wide)), l = (uint32_t)__shfl((int)low[i], (int)(lane + half * wide));
            if (team + half < n) high[i] = larger(high[i], h), low[i] = larger(low[i], l);
        }
        n = half;
    }
    if (team) return;
    uint8_t *const to = a.bounds + (int64_t)entry * a.bounds_block_stride + (int64_t)head * a.bounds_head_stride + d;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const uint32_t nan = (nan_bytes(high[i]) | nan_bytes(low[i])) >> 7, all = nan * 0xFFu;
        high[i] = (unordered(high[i]) & ~all) | (0x7F7F7F7Fu & all);
        low[i] = (unordered(~low[i]) & ~all) | (0x7F7F7F7Fu & all);
    }
    *reinterpret_cast<u32x4 *>(to) = low;
    *reinterpret_cast<u32x4 *>(to + a.c.dim) = high;
}

hipError_t launch_bound(BoundArgs a, hipStream_t s)
{
    const Reach reach = reach_of(a.c, a.b);
    a.counted = reach.counted;
    a.touched = (uint32_t)std::min<uint64_t>(reach.blocks, 0xffffffffu);
    const uint64_t groups = (reach.blocks * a.c.heads + 3u) / 4u;
    if (!launchable(groups, 256)) return hipErrorInvalidConfiguration;
    bound_kernel<<<dim3((uint32_t)groups, reach.reqs), 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace kv8
}  // namespace dmi
