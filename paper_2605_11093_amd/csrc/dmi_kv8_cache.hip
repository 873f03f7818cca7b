// Kernels that write the 8-bit KV cache: tokens appended, tokens kept.
#include "dmi_internal.h"
#include "dmi_kv8_internal.h"

#include <hip/hip_fp16.h>

namespace dmi {
namespace kv8 {

// Largest of a word over the wavefront
__device__ __forceinline__ uint32_t wave_largest(uint32_t v)
{
#pragma unroll
    for (int m = 32; m; m >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, m));
    return v;
}

// ---------------------------------------------------------------- append
// Eight neighbours of a row as they lie in memory, and as numbers.
template <typename T> struct Eight {
    u32x4 w[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T *p)
    {
#pragma unroll
        for (unsigned i = 0; i < sizeof(T) / 2; i++) w[i] = reinterpret_cast<const u32x4 *>(p)[i];
    }
    __device__ __forceinline__ void numbers(float x[8]) const;
};
struct Bf16Bits { uint16_t u; };
template <> __device__ __forceinline__ void Eight<Bf16Bits>::numbers(float x[8]) const
{
#pragma unroll
    for (int i = 0; i < 4; i++) {
        x[2 * i] = __uint_as_float(w[0][i] << 16);
        x[2 * i + 1] = __uint_as_float(w[0][i] & 0xFFFF0000u);
    }
}
template <> __device__ __forceinline__ void Eight<_Float16>::numbers(float x[8]) const
{
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const uint32_t two = w[0][i];
        const f16x2 h = __builtin_bit_cast(f16x2, two);
        x[2 * i] = (float)h[0];
        x[2 * i + 1] = (float)h[1];
    }
}
template <> __device__ __forceinline__ void Eight<float>::numbers(float x[8]) const
{
#pragma unroll
    for (int i = 0; i < 8; i++) x[i] = __uint_as_float(w[i / 4][i % 4]);
}

// One wavefront per (request, block that it reaches, head, K or V): the largest magnitude of the new tokens' elements, the scale
// from its exponent, then the codes.  What a block of 16 tokens and 128 elements holds stays in registers between the two, so x is
// read once; a scale is one block's and head's alone, so wavefronts share nothing.  Bound by memory where there is much to write: 32
// prompts, 38600 tokens of 8 heads x 128 in bf16, 237 MB in 52 us (4.6 TB/s; a copy reaches 5.0 on this card); elsewhere by a chain of
// four loads that wait for each other (length, table, scale, rows): 128 single tokens 4.6 us.  Non-temporal loads and stores gained
// 4 us with the prompts and lost 3 to 4 where the caller has just written x (16 requests of some 30 tokens, fp32: 8.5 us).
template <typename T>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a)
{
    constexpr int kHeld = 4;                    // units of 8 elements a lane keeps
    const uint32_t lane = threadIdx.x & 63u;
    const uint32_t item = blockIdx.x * 4u + (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t kv = item & 1u, head = (item >> 1) % a.c.heads;
    uint32_t nth = (item >> 1) / a.c.heads;
    Request q{0, 0, 0, 0};
    if (a.counted) {
        // as many wavefronts as all requests' new tokens make: the blocks that they reach are counted here
        for (uint32_t n0 = 0;; n0 += 64u) {
            if (n0 >= a.b.n_reqs) return;
            Request own{0, 0, 0, 0};
            if (n0 + lane < a.b.n_reqs) own = request_of(a.b, a.c, (int)(n0 + lane));
            const int begin = max(own.len - own.fresh, 0);
            const int reached = own.len > begin ? (int)(block_of(a.c, (uint32_t)(own.len - 1) >> 4) - block_of(a.c, (uint32_t)begin >> 4)) + 1 : 0;
            const int upto = lanes_scan(reached);
            const uint64_t behind = __ballot(upto > (int)nth);
            if (!behind) {
                nth -= (uint32_t)__builtin_amdgcn_readlane(upto, 63);
                continue;
            }
            const int in = __ffsll((unsigned long long)behind) - 1;
            if (in) nth -= (uint32_t)__builtin_amdgcn_readlane(upto, in - 1);
            q = request_in(own, in);
            break;
        }
    } else {
        if (nth >= a.touched) return;
        q = request_of(a.b, a.c, (int)blockIdx.y);
    }
    const int first = q.len - q.fresh;          // the first new token's position; below 0: that token has none
    const int from = max(first, 0);
    const uint32_t block = block_of(a.c, (uint32_t)from >> 4) + nth;
    const int lo = max(from, (int)(block * a.c.bs)), hi = min(q.len, (int)((block + 1u) * a.c.bs));
    if (lo >= hi) return;
    const int b = entry_of(a.c, q.row, block);
    if (b < 0) return;

    const uint32_t per_row = a.c.dim >> 3, units = (uint32_t)(hi - lo) * per_row;
    const T *src = static_cast<const T *>(a.x[kv].data) + (int64_t)(q.start + lo - first) * a.x[kv].row_stride +
                   (int64_t)head * a.x[kv].head_stride;
    const uint32_t slot0 = (uint32_t)lo - block * a.c.bs;
    float *const scale_p = scale_at(a.c, (int)kv, b, head);
    const float had = slot0 ? *scale_p : 0.0f;

    Eight<T> held[kHeld];
    uint32_t largest = 0;
    auto look = [&](const Eight<T> &e) {
        float x[8];
        e.numbers(x);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const uint32_t m = __float_as_uint(x[i]) & 0x7FFFFFFFu;
            largest = max(largest, m < 0x7F800000u ? m : 0u);
        }
    };
    auto place = [&](uint32_t u) { return src + (int64_t)(u / per_row) * a.x[kv].row_stride + (u % per_row) * 8u; };
#pragma unroll
    for (int i = 0; i < kHeld; i++)
        if (lane + 64u * i < units) held[i].load(place(lane + 64u * i));
#pragma unroll
    for (int i = 0; i < kHeld; i++)
        if (lane + 64u * i < units) look(held[i]);
    for (uint32_t u = lane + 64u * kHeld; u < units; u += 64u) {
        Eight<T> e;
        e.load(place(u));
        look(e);
    }
    largest = wave_largest(largest);

    // 448 = 1.75 * 2^8: the exponent of the least power of two that is no less than largest / 448
    const int exponent = max((int)(largest >> 23) - 8 + ((largest & 0x7FFFFFu) > 0x600000u ? 1 : 0), 127 - 100);
    const float need = __uint_as_float((uint32_t)exponent << 23);
    const float s = fmaxf(need, had);
    if (slot0 && s != had) {                    // what the block held already
        const float f = had / s;
        for (uint32_t u = lane; u < slot0 * per_row; u += 64u) {
            u32x2 *p = reinterpret_cast<u32x2 *>(code_at(a.c, (int)kv, b, u / per_row, head) + (u % per_row) * 8u);
            u32x2 w = *p;
            w[0] = scaled_codes(w[0], f);
            w[1] = scaled_codes(w[1], f);
            *p = w;
        }
    }
    auto put = [&](uint32_t u, const Eight<T> &e) {
        float x[8];
        e.numbers(x);
        if (s == need) {
            const float inv = __uint_as_float((uint32_t)(254 - exponent) << 23);
#pragma unroll
            for (int i = 0; i < 8; i++) x[i] *= inv;
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++) x[i] /= s;
        }
        u32x2 w;
        w[0] = to_codes(x[0], x[1], x[2], x[3]);
        w[1] = to_codes(x[4], x[5], x[6], x[7]);
        *reinterpret_cast<u32x2 *>(code_at(a.c, (int)kv, b, slot0 + u / per_row, head) + (u % per_row) * 8u) = w;
    };
#pragma unroll
    for (int i = 0; i < kHeld; i++)
        if (lane + 64u * i < units) put(lane + 64u * i, held[i]);
    for (uint32_t u = lane + 64u * kHeld; u < units; u += 64u) {
        Eight<T> e;
        e.load(place(u));
        put(u, e);
    }
    if (!lane) *scale_p = s;
}

hipError_t launch_append(AppendArgs a, uint32_t dtype, hipStream_t s)
{
    // Blocks that all new tokens reach at most: as many as they fill, and a part of one at either end of a request.  Where the most that one
    // request may reach, for every request, is more than twice that, the kernel counts for itself (us, without / with): a prompt of
    // 8192 tokens among 63 single ones 74 / 15, one of 2048 among 255 70 / 10, 32 ragged prompts 52 either way.
    const uint64_t reached = (uint64_t)a.b.total_new / a.c.bs + 2u * (uint64_t)a.b.n_reqs;
    a.counted = (uint64_t)a.touched * a.b.n_reqs > 2u * reached;
    const uint64_t groups = ((a.counted ? reached : a.touched) * a.c.heads * 2u + 3u) / 4u;
    if (!launchable(groups, 256)) return hipErrorInvalidConfiguration;
    const dim3 grid((uint32_t)groups, a.counted ? 1u : a.b.n_reqs);
    switch (dtype) {
    case DMI_DTYPE_BF16: append_kernel<Bf16Bits><<<grid, 256, 0, s>>>(a); break;
    case DMI_DTYPE_FP16: append_kernel<_Float16><<<grid, 256, 0, s>>>(a); break;
    default: append_kernel<float><<<grid, 256, 0, s>>>(a); break;
    }
    return hipGetLastError();
}

// ---------------------------------------------------------------- evict
// Weights in an order of unsigned numbers: NaN as -inf, -0 as 0.
__device__ __forceinline__ uint32_t order_of(float w)
{
    if (w != w) return 0x007FFFFFu;
    const uint32_t u = w == 0.0f ? 0u : __float_as_uint(w);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr uint32_t kSelectThreads = 512, kHeldKeys = 16;     // keys a thread keeps: 8192 tokens of a workgroup
constexpr uint32_t kBins = 2048;                            // digits of 11, 11 and 10 bits

// One workgroup per (request, head): the want-th largest weight among the older tokens, digit by digit, then the positions of
// what is larger, and of as many that equal it as are still wanted, in order.  Weights are read once where a thread can keep its
// own (up to 8192 tokens), and again for every digit behind that.  Weights of attention share few exponents: 11 bits spread them over
// more counters than 8 do, and that lanes meet on one counter is what this kernel waits for (128 requests of 512-8192 tokens, 8 heads:
// 29 us for 18 MB, 38 us with digits of 8 bits that read the weights four times).
__global__ __launch_bounds__(kSelectThreads) void select_kernel(EvictArgs a)
{
    __shared__ uint32_t hist[kBins], wave_n[kSelectThreads / 64][2], found[2];
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6, head = blockIdx.x, r = blockIdx.y;
    const Request q = request_of(a.b, a.c, (int)r);
    const uint32_t len = (uint32_t)q.len, left = min(len, a.keep);
    if (!head && !tid) a.to_lens[r] = (int32_t)left;
    int32_t *pos = a.positions + ((int64_t)r * a.c.heads + head) * a.keep;
    const float *w = a.w.data + (int64_t)q.row * a.w.row_stride + (int64_t)head * a.w.head_stride;
    float *to_w = a.to_w.data + (int64_t)q.row * a.to_w.row_stride + (int64_t)head * a.to_w.head_stride;
    for (uint32_t i = left + tid; i < a.keep; i += kSelectThreads) pos[i] = -1;
    if (len <= a.keep) {
        for (uint32_t i = tid; i < len; i += kSelectThreads) {
            pos[i] = (int32_t)i;
            to_w[i] = w[i];
        }
        return;
    }
    const uint32_t old = len - a.recent, want = a.keep - a.recent;
    for (uint32_t i = tid; i < a.recent; i += kSelectThreads) {
        pos[want + i] = (int32_t)(old + i);
        to_w[want + i] = w[old + i];
    }
    if (!want) return;
    float held[kHeldKeys];
#pragma unroll
    for (uint32_t k = 0; k < kHeldKeys; k++) held[k] = k * kSelectThreads + tid < old ? w[k * kSelectThreads + tid] : 0.0f;
    // the want-th largest: of the keys that begin with `prefix`, the rank-th
    uint32_t prefix = 0, rank = want;
    for (int digit = 0; digit < 3; digit++) {
        const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0;
        const uint32_t bins = digit == 2 ? 1024u : kBins, above = digit == 0 ? 0u : digit == 1 ? ~0u << 21 : ~0u << 10;
        for (uint32_t i = tid; i < kBins; i += kSelectThreads) hist[i] = 0;
        __syncthreads();
        auto count = [&](float x) {
            const uint32_t k = order_of(x);
            if ((k & above) == prefix) atomicAdd(&hist[(k >> shift) & (bins - 1u)], 1u);
        };
#pragma unroll
        for (uint32_t k = 0; k < kHeldKeys; k++)
            if (k * kSelectThreads + tid < old) count(held[k]);
        for (uint32_t i = kHeldKeys * kSelectThreads + tid; i < old; i += kSelectThreads) count(w[i]);
        __syncthreads();
        // four bins a thread, from the largest down
        uint32_t n[4], sum = 0;
#pragma unroll
        for (int i = 0; i < 4; i++) sum += n[i] = hist[kBins - 1u - 4u * tid - i];
        uint32_t before = sum;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            const uint32_t up = (uint32_t)__shfl_up((int)before, m);
            if (lane >= (uint32_t)m) before += up;
        }
        if (lane == 63u) wave_n[wave][0] = before;
        __syncthreads();
        before -= sum;
#pragma unroll
        for (uint32_t v = 0; v < kSelectThreads / 64; v++)
            if (v < wave) before += wave_n[v][0];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            if (before < rank && rank <= before + n[i]) {
                found[0] = kBins - 1u - 4u * tid - i;
                found[1] = rank - before;
            }
            before += n[i];
        }
        __syncthreads();
        prefix |= found[0] << shift;
        rank = found[1];
    }
    // `rank` of the keys that equal `prefix` are taken, the lowest positions first
    uint32_t taken = 0, equal = 0;
    auto take = [&](uint32_t base, float x) {
        const uint32_t i = base + tid, k = order_of(x);
        const bool is_more = i < old && k > prefix, is_equal = i < old && k == prefix;
        const uint64_t more = __ballot(is_more), same = __ballot(is_equal);
        __syncthreads();
        if (!lane) {
            wave_n[wave][0] = (uint32_t)__popcll(more);
            wave_n[wave][1] = (uint32_t)__popcll(same);
        }
        __syncthreads();
        uint32_t m = 0, e = 0, all_m = 0, all_e = 0;
#pragma unroll
        for (uint32_t v = 0; v < kSelectThreads / 64; v++) {
            if (v < wave) m += wave_n[v][0], e += wave_n[v][1];
            all_m += wave_n[v][0];
            all_e += wave_n[v][1];
        }
        const uint64_t below = (1ull << lane) - 1ull;
        m += (uint32_t)__popcll(more & below);
        e += (uint32_t)__popcll(same & below);
        // of the equal ones in front of this one, those that are taken
        const uint32_t at = taken + m + min(equal + e, rank) - min(equal, rank);
        if (is_more || (is_equal && equal + e < rank)) {
            pos[at] = (int32_t)i;
            to_w[at] = x;
        }
        taken += all_m + min(equal + all_e, rank) - min(equal, rank);
        equal += all_e;
    };
#pragma unroll
    for (uint32_t k = 0; k < kHeldKeys; k++)
        if (k * kSelectThreads < old) take(k * kSelectThreads, held[k]);
    for (uint32_t base = kHeldKeys * kSelectThreads; base < old; base += kSelectThreads) take(base, base + tid < old ? w[base + tid] : 0.0f);
}

constexpr uint32_t kMoveWaves = 4096;           // four on each SIMD
constexpr int64_t kNowhere = INT64_MIN;         // an offset of codes that are not there (any other may lie on either side of 0)

// One wavefront per (request, head) and as many whole blocks of `to` as 64 tokens make, at least one (just one while that leaves
// wavefronts to spare: four requests of 8 heads that keep 256 tokens take 6.4 us so and 10.6 with 64 tokens each): where its tokens lie, a token a
// lane; the largest scales of K and V that meet in each block; then their codes, 16 bytes a lane, eight loads at a time.  The heads
// of a span of tokens follow each other on one XCD: they read the same pages, and write one block.  Bound by memory: 128 requests cut to
// 2048 tokens, 243000 tokens of 8 heads x 128 read and written, 996 MB in 203 us, 4.9 TB/s, the rate of a copy (212 us with loads and
// stores through the caches, 318 with one block, and K or V alone, a wavefront).
__global__ __launch_bounds__(256) void move_kernel(EvictArgs a, uint32_t blocks, uint32_t spans)
{
    const uint32_t lane = threadIdx.x & 63u, span = blocks * a.c.bs;
    const uint32_t unit = (blockIdx.x >> 3) * 4u + (threadIdx.x >> 6);
    const uint32_t item = unit / a.c.heads * 8u + (blockIdx.x & 7u), head = unit % a.c.heads, r = item / spans, nth = item - r * spans;
    if (r >= a.b.n_reqs) return;
    const Request q = request_of(a.b, a.c, (int)r);
    const uint32_t left = min((uint32_t)q.len, a.keep), first = nth * span;
    if (first >= left) return;
    const uint32_t m = min(span, left - first), per_row = a.c.dim >> 4;
    const int32_t *pos = a.positions + ((int64_t)r * a.c.heads + head) * a.keep + first;
    // a token's codes and scales
    auto source = [&](uint32_t t, int64_t &at, float &sk, float &sv) {
        const uint32_t p = (uint32_t)pos[t], lb = block_of(a.c, p >> 4);
        const int b = p < (uint32_t)q.len ? entry_of(a.c, q.row, lb) : -1;     // (a length that is another than select_kernel saw)
        at = b < 0 ? kNowhere : (int64_t)b * a.c.block_stride + (int64_t)(p - lb * a.c.bs) * a.c.slot_stride + (int64_t)head * a.c.head_stride;
        sk = b < 0 ? 0.0f : *scale_at(a.c, 0, b, head);
        sv = b < 0 ? 0.0f : *scale_at(a.c, 1, b, head);
    };
    int64_t at = kNowhere;
    float sk = 0.0f, sv = 0.0f, most_k = 0.0f, most_v = 0.0f;       // the largest: of the block that the lane's token joins
    for (uint32_t t0 = 0; t0 < m; t0 += 64u) {      // (more than one round only for blocks of more than 64 tokens)
        at = kNowhere, sk = sv = 0.0f;
        if (t0 + lane < m) source(t0 + lane, at, sk, sv);
        most_k = fmaxf(most_k, sk);
        most_v = fmaxf(most_v, sv);
    }
    const int joined = blocks == 1u ? 64 : (int)a.c.bs;             // lanes
    for (int x = 1; x < joined; x <<= 1) most_k = fmaxf(most_k, __shfl_xor(most_k, x)), most_v = fmaxf(most_v, __shfl_xor(most_v, x));
    // nothing but entries outside the cache
    if (!(most_k > 0.0f)) most_k = __uint_as_float((127u - 100u) << 23);
    if (!(most_v > 0.0f)) most_v = __uint_as_float((127u - 100u) << 23);
    const int to = lane < blocks ? entry_of(a.to, q.row, nth * blocks + lane) : -1;
    for (uint32_t t0 = 0; t0 < m; t0 += 64u) {
        if (m > 64u) {
            at = kNowhere, sk = sv = 0.0f;
            if (t0 + lane < m) source(t0 + lane, at, sk, sv);
        }
        const float fk = sk / most_k, fv = sv / most_v;
        const uint32_t units = min(64u, m - t0) * per_row;
        for (uint32_t u0 = 0; u0 < units; u0 += 256u) {
            u32x4 wk[4], wv[4];
            float gk[4], gv[4];
            int64_t dst[4];
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const uint32_t u = u0 + 64u * j + lane, t = u / per_row, part = (u - t * per_row) * 16u;
                const int from = (int)(t & 63u);
                const int64_t src = (int64_t)(uint32_t)__shfl((int)(uint32_t)at, from) | (int64_t)__shfl((int)(at >> 32), from) << 32;
                gk[j] = __shfl(fk, from);
                gv[j] = __shfl(fv, from);
                const uint32_t slot = t0 + t, block = blocks == 1u ? 0u : slot / a.c.bs;
                const int e = __shfl(to, (int)(block & 63u));
                dst[j] = u < units && e >= 0 ? (int64_t)e * a.to.block_stride + (int64_t)(slot - block * a.c.bs) * a.to.slot_stride +
                                                   (int64_t)head * a.to.head_stride + part : kNowhere;
                wk[j] = wv[j] = u32x4{0u, 0u, 0u, 0u};
                if (dst[j] != kNowhere && src != kNowhere) {
                    wk[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(a.c.code[0] + src + part));
                    wv[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(a.c.code[1] + src + part));
                }
            }
#pragma unroll
            for (int j = 0; j < 4; j++) {
                if (dst[j] == kNowhere) continue;
                if (gk[j] != 1.0f) {
#pragma unroll
                    for (int i = 0; i < 4; i++) wk[j][i] = scaled_codes(wk[j][i], gk[j]);
                }
                if (gv[j] != 1.0f) {
#pragma unroll
                    for (int i = 0; i < 4; i++) wv[j][i] = scaled_codes(wv[j][i], gv[j]);
                }
                __builtin_nontemporal_store(wk[j], reinterpret_cast<u32x4 *>(a.to.code[0] + dst[j]));
                __builtin_nontemporal_store(wv[j], reinterpret_cast<u32x4 *>(a.to.code[1] + dst[j]));
            }
        }
    }
    most_k = __shfl(most_k, (int)(lane * a.c.bs & 63u));
    most_v = __shfl(most_v, (int)(lane * a.c.bs & 63u));
    if (lane < blocks && lane * a.c.bs < m && to >= 0) {
        *scale_at(a.to, 0, to, head) = most_k;
        *scale_at(a.to, 1, to, head) = most_v;
    }
}

hipError_t launch_evict(const EvictArgs &a, hipStream_t s)
{
    const uint32_t left = min(a.keep, max(a.b.max_len, 1u));
    uint32_t blocks = max(1u, 64u / a.c.bs);
    if ((uint64_t)left * a.b.n_reqs * a.c.heads < 64u * kMoveWaves) blocks = 1;
    const uint32_t span = blocks * a.c.bs, spans = (left + span - 1u) / span;
    const uint64_t units = ((uint64_t)spans * a.b.n_reqs + 7u) / 8u * a.c.heads, groups = (units + 3u) / 4u * 8u;    // units: on each XCD
    if (!launchable(groups, 256)) return hipErrorInvalidConfiguration;
    select_kernel<<<dim3(a.c.heads, a.b.n_reqs), kSelectThreads, 0, s>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    move_kernel<<<(uint32_t)groups, 256, 0, s>>>(a, blocks, spans);
    return hipGetLastError();
}

}  // namespace kv8
}  // namespace dmi
