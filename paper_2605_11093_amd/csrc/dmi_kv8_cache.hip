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
struct Bf16 { uint16_t u; };
template <> __device__ __forceinline__ void Eight<Bf16>::numbers(float x[8]) const
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
// from its exponent, then the codes.  What a block of 16 tokens and 128 elements holds stays in registers between the two.
template <typename T>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a)
{
    constexpr int kHeld = 4;                    // units of 8 elements a lane keeps
    const uint32_t lane = threadIdx.x & 63u;
    const uint32_t item = blockIdx.x * 4u + (threadIdx.x >> 6);
    const uint32_t kv = item & 1u, head = (item >> 1) % a.c.heads, nth = (item >> 1) / a.c.heads;
    if (nth >= a.touched) return;
    const Request q = request_of(a.b, a.c, (int)blockIdx.y);
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

hipError_t launch_append(const AppendArgs &a, uint32_t dtype, hipStream_t s)
{
    const dim3 grid((a.touched * a.c.heads * 2u + 3u) / 4u, a.b.n_reqs);
    switch (dtype) {
    case DMI_DTYPE_BF16: append_kernel<Bf16><<<grid, 256, 0, s>>>(a); break;
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

constexpr uint32_t kSelectThreads = 512;

// One workgroup per (request, head): the want-th largest weight among the older tokens, digit by digit, then the positions of
// what is larger, and of as many that equal it as are still wanted, in order.
__global__ __launch_bounds__(kSelectThreads) void select_kernel(EvictArgs a)
{
    __shared__ uint32_t hist[256], wave_n[kSelectThreads / 64][2], found[2];
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
    // the want-th largest: of the keys that begin with `prefix`, the rank-th
    uint32_t prefix = 0, rank = want;
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (tid < 256u) hist[tid] = 0;
        __syncthreads();
        for (uint32_t i = tid; i < old; i += kSelectThreads) {
            const uint32_t k = order_of(w[i]);
            if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255u], 1u);
        }
        __syncthreads();
        if (wave == 0) {                        // four bins a lane, from the largest down
            uint32_t n[4], sum = 0;
#pragma unroll
            for (int i = 0; i < 4; i++) sum += n[i] = hist[255u - 4u * lane - i];
            uint32_t before = sum;
#pragma unroll
            for (int m = 1; m < 64; m <<= 1) {
                const uint32_t up = (uint32_t)__shfl_up((int)before, m);
                if (lane >= (uint32_t)m) before += up;
            }
            before -= sum;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                if (before < rank && rank <= before + n[i]) {
                    found[0] = 255u - 4u * lane - i;
                    found[1] = rank - before;
                }
                before += n[i];
            }
        }
        __syncthreads();
        prefix |= found[0] << shift;
        rank = found[1];
        __syncthreads();
    }
    // `rank` of the keys that equal `prefix` are taken, the lowest positions first
    uint32_t taken = 0, equal = 0;
    for (uint32_t base = 0; base < old; base += kSelectThreads) {
        const uint32_t i = base + tid;
        const float x = i < old ? w[i] : 0.0f;
        const uint32_t k = order_of(x);
        const bool is_more = i < old && k > prefix, is_equal = i < old && k == prefix;
        const uint64_t more = __ballot(is_more), same = __ballot(is_equal);
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
        __syncthreads();
    }
}

// One wavefront per (request, block of `to`, head, K or V): the largest scale among the tokens that meet in the block, then
// their codes, 16 bytes a lane.
__global__ __launch_bounds__(256) void move_kernel(EvictArgs a)
{
    const uint32_t lane = threadIdx.x & 63u;
    const uint32_t item = blockIdx.x * 4u + (threadIdx.x >> 6);
    const uint32_t kv = item & 1u, head = (item >> 1) % a.c.heads, nth = (item >> 1) / a.c.heads, r = blockIdx.y;
    const Request q = request_of(a.b, a.c, (int)r);
    const uint32_t left = min((uint32_t)q.len, a.keep), first = nth * a.c.bs;
    if (first >= left) return;
    const int to = entry_of(a.to, q.row, nth);
    if (to < 0) return;
    const uint32_t m = min(a.c.bs, left - first), per_row = a.c.dim >> 4;
    const int32_t *pos = a.positions + ((int64_t)r * a.c.heads + head) * a.keep + first;
    // a token's block, or -1, its slot and its scale
    auto source = [&](uint32_t t, int &b, uint32_t &slot, float &s) {
        const uint32_t p = (uint32_t)pos[t], lb = block_of(a.c, p >> 4);
        b = entry_of(a.c, q.row, lb);
        slot = p - lb * a.c.bs;
        s = b < 0 ? 0.0f : *scale_at(a.c, (int)kv, b, head);
    };
    float largest = 0.0f, s = 0.0f;
    int b = -1;
    uint32_t slot = 0;
    for (uint32_t t = lane; t < m; t += 64u) {
        source(t, b, slot, s);
        largest = fmaxf(largest, s);
    }
    largest = __uint_as_float(wave_largest(__float_as_uint(largest)));
    if (!(largest > 0.0f)) largest = __uint_as_float((127u - 100u) << 23);      // nothing but entries outside the cache
    for (uint32_t t0 = 0; t0 < m; t0 += 64u) {
        if (m > 64u) {
            b = -1;
            if (t0 + lane < m) source(t0 + lane, b, slot, s);
        }
        const float f = s / largest;
        const uint32_t units = min(64u, m - t0) * per_row;
        for (uint32_t u0 = 0; u0 < units; u0 += 64u) {
            const uint32_t u = u0 + lane, t = u / per_row, part = u % per_row * 16u;
            const int b_t = __shfl(b, (int)(t & 63u));
            const uint32_t slot_t = (uint32_t)__shfl((int)slot, (int)(t & 63u));
            const float f_t = __shfl(f, (int)(t & 63u));
            if (u >= units) continue;
            u32x4 w = {0u, 0u, 0u, 0u};
            if (b_t >= 0) {
                w = *reinterpret_cast<const u32x4 *>(code_at(a.c, (int)kv, b_t, slot_t, head) + part);
                if (f_t != 1.0f) {
#pragma unroll
                    for (int i = 0; i < 4; i++) w[i] = scaled_codes(w[i], f_t);
                }
            }
            *reinterpret_cast<u32x4 *>(code_at(a.to, (int)kv, to, t0 + t, head) + part) = w;
        }
    }
    if (!lane) *scale_at(a.to, (int)kv, to, head) = largest;
}

hipError_t launch_evict(const EvictArgs &a, hipStream_t s)
{
    select_kernel<<<dim3(a.c.heads, a.b.n_reqs), kSelectThreads, 0, s>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const uint32_t blocks = (min(a.keep, max(a.b.max_len, 1u)) + a.c.bs - 1u) / a.c.bs;
    move_kernel<<<dim3((blocks * a.c.heads * 2u + 3u) / 4u, a.b.n_reqs), 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace kv8
}  // namespace dmi
