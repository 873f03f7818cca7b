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
constexpr uint32_t kRowsAtOnce = 4;             // query rows whose scores a lane sums at a time

// A workgroup per new token, head and 256 blocks, a lane per block: the larger of q x least and q x largest is one product with the
// one or the other, by q's sign, so that a score is the sum of two products' and every term but rounding in 64 bits is exact.  The
// order in which it is summed moves a score by some 2^-50 of its terms, and which blocks are taken hangs on no order.
template <typename T, int DP>
__global__ __launch_bounds__(256) void score_kernel(SelectArgs a)
{
    __shared__ __align__(16) double lq[DP][kRowsAtOnce][2];
    const uint32_t per = (a.stride + 255u) / 256u, item = blockIdx.x / per, chunk = blockIdx.x - item * per;
    const uint32_t token = item / a.c.heads, head = item - token * a.c.heads;
    const Request q = token_of(a.b, a.c, (int)token);
    const Choice x = choice_of(a, q);
    const uint32_t block = x.lo + 256u * chunk + threadIdx.x;
    if (q.fresh <= 0 || x.lo + 256u * chunk >= x.hi) return;

    const int entry = block < x.hi ? entry_of(a.c, q.row, block) : -1;
    u32x4 low[DP / 16], high[DP / 16];
    const uint8_t *const at = a.bounds + (int64_t)max(entry, 0) * a.bounds_block_stride + (int64_t)head * a.bounds_head_stride;
#pragma unroll
    for (int i = 0; i < DP / 16; i++) low[i] = *reinterpret_cast<const u32x4 *>(at + (16u * i < a.c.dim ? 16u * i : 0u));
#pragma unroll
    for (int i = 0; i < DP / 16; i++) high[i] = *reinterpret_cast<const u32x4 *>(at + a.c.dim + (16u * i < a.c.dim ? 16u * i : 0u));
    const double scale = entry >= 0 ? (double)*scale_at(a.c, 0, entry, head) : 0.0;

    double best = -INFINITY;
    bool bad = false;
    for (uint32_t row0 = 0; row0 < a.group; row0 += kRowsAtOnce) {
        const uint32_t rows = min(kRowsAtOnce, a.group - row0);
        if (row0) __syncthreads();
        for (uint32_t u = threadIdx.x; u < DP * kRowsAtOnce; u += 256u) {
            const uint32_t r = u / DP, d = u - r * DP;
            double v = 0.0;
            if (r < rows && d < a.c.dim)
                v = T::number(static_cast<const uint16_t *>(a.q.data)[(int64_t)token * a.q.row_stride + (int64_t)(head * a.group + row0 + r) * a.q.head_stride + d]);
            lq[d][r][0] = v > 0.0 ? 0.0 : v;
            lq[d][r][1] = v > 0.0 ? v : 0.0;
        }
        __syncthreads();
        double sum[kRowsAtOnce] = {};
#pragma unroll
        for (int i = 0; i < DP / 16; i++) {
            if (16u * i >= a.c.dim) break;
#pragma unroll
            for (int w = 0; w < 4; w++) {
                const f32x2 l[2] = {__builtin_amdgcn_cvt_pk_f32_fp8((int)low[i][w], false), __builtin_amdgcn_cvt_pk_f32_fp8((int)low[i][w], true)};
                const f32x2 h[2] = {__builtin_amdgcn_cvt_pk_f32_fp8((int)high[i][w], false), __builtin_amdgcn_cvt_pk_f32_fp8((int)high[i][w], true)};
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const double least = l[e >> 1][e & 1], largest = h[e >> 1][e & 1];
#pragma unroll
                    for (uint32_t r = 0; r < kRowsAtOnce; r++) {
                        sum[r] = __builtin_fma(lq[16 * i + 4 * w + e][r][0], least, sum[r]);
                        sum[r] = __builtin_fma(lq[16 * i + 4 * w + e][r][1], largest, sum[r]);
                    }
                }
            }
        }
#pragma unroll
        for (uint32_t r = 0; r < kRowsAtOnce; r++)
            if (r < rows) {
                bad |= sum[r] != sum[r];
                best = sum[r] > best ? sum[r] : best;
            }
    }
    if (block < x.hi) a.keys[(int64_t)item * a.stride + block] = order_of(entry < 0 || bad ? -INFINITY : best * scale);
}

constexpr uint32_t kChooseThreads = 256, kChooseHeld = 16;      // keys a thread keeps: 4096 blocks
constexpr uint32_t kChooseBins = 2048;

// A workgroup per new token and head: the want-th largest score digit by digit, from the top and only as far as it takes to tell
// it from the others, then the blocks in order.
__global__ __launch_bounds__(kChooseThreads) void choose_kernel(SelectArgs a)
{
    constexpr uint32_t kWaves = kChooseThreads / 64;
    __shared__ uint32_t hist[kChooseBins], wave_n[kWaves][2], found[3];
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6, item = blockIdx.x, token = item / a.c.heads;
    const Request q = token_of(a.b, a.c, (int)token);
    if (q.fresh <= 0) return;                   // no request's
    const Choice x = choice_of(a, q);
    int32_t *const to = a.blocks + (int64_t)item * a.n_select;
    if (x.seen <= a.n_select) {
        for (uint32_t i = tid; i < a.n_select; i += kChooseThreads) to[i] = i < x.seen ? (int32_t)i : -1;
        return;
    }
    const uint32_t want = a.n_select - a.n_first - a.n_recent, count = x.hi - x.lo;
    for (uint32_t i = tid; i < a.n_first; i += kChooseThreads) to[i] = (int32_t)i;
    for (uint32_t i = tid; i < a.n_recent; i += kChooseThreads) to[a.n_first + want + i] = (int32_t)(x.hi + i);
    if (!want) return;
    const uint64_t *const keys = a.keys + (int64_t)item * a.stride + x.lo;
    uint64_t held[kChooseHeld];
#pragma unroll
    for (uint32_t k = 0; k < kChooseHeld; k++) held[k] = k * kChooseThreads + tid < count ? keys[k * kChooseThreads + tid] : 0ull;
    // of the keys that begin with `prefix` the rank-th is looked for; all of those that begin with a larger one are taken
    uint64_t prefix = 0;
    uint32_t rank = want;
    int shift = 64;
    while (shift > 0) {
        const int bits = min(11, shift);
        const uint32_t bins = 1u << bits;
        const int above = shift;
        shift -= bits;
        for (uint32_t i = tid; i < kChooseBins; i += kChooseThreads) hist[i] = 0;
        __syncthreads();
        auto add = [&](uint64_t k) {
            if (above == 64 || k >> above == prefix) atomicAdd(&hist[(uint32_t)(k >> shift) & (bins - 1u)], 1u);
        };
#pragma unroll
        for (uint32_t k = 0; k < kChooseHeld; k++)
            if (k * kChooseThreads + tid < count) add(held[k]);
        for (uint32_t i = kChooseHeld * kChooseThreads + tid; i < count; i += kChooseThreads) add(keys[i]);
        __syncthreads();
        // eight bins a thread, from the largest down
        uint32_t n[8], sum = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) sum += n[i] = hist[kChooseBins - 1u - 8u * tid - i];
        uint32_t before = (uint32_t)lanes_scan((int)sum);
        if (lane == 63u) wave_n[wave][0] = before;
        __syncthreads();
        before -= sum;
#pragma unroll
        for (uint32_t v = 0; v < kWaves; v++)
            if (v < wave) before += wave_n[v][0];
#pragma unroll
        for (int i = 0; i < 8; i++) {
            if (before < rank && rank <= before + n[i]) {
                found[0] = kChooseBins - 1u - 8u * tid - i;
                found[1] = rank - before;
                found[2] = n[i];
            }
            before += n[i];
        }
        __syncthreads();
        prefix = prefix << bits | found[0];
        rank = found[1];
        if (found[2] == rank) break;            // all of these are taken
    }
    // `rank` of the keys that begin with `prefix` are taken, the lowest blocks first
    uint32_t taken = 0, equal = 0;
    for (uint32_t base = 0; base < count; base += kChooseThreads) {
        const uint32_t i = base + tid;
        const uint64_t k = i < count ? keys[i] >> shift : 0ull;
        const bool is_more = i < count && k > prefix, is_equal = i < count && k == prefix;
        const uint64_t more = __ballot(is_more), same = __ballot(is_equal);
        __syncthreads();
        if (!lane) {
            wave_n[wave][0] = (uint32_t)__popcll(more);
            wave_n[wave][1] = (uint32_t)__popcll(same);
        }
        __syncthreads();
        uint32_t m = 0, e = 0, all_m = 0, all_e = 0;
#pragma unroll
        for (uint32_t v = 0; v < kWaves; v++) {
            if (v < wave) m += wave_n[v][0], e += wave_n[v][1];
            all_m += wave_n[v][0];
            all_e += wave_n[v][1];
        }
        const uint64_t below = (1ull << lane) - 1ull;
        m += (uint32_t)__popcll(more & below);
        e += (uint32_t)__popcll(same & below);
        const uint32_t at = taken + m + min(equal + e, rank) - min(equal, rank);
        if (is_more || (is_equal && equal + e < rank)) to[a.n_first + at] = (int32_t)(x.lo + i);
        taken += all_m + min(equal + all_e, rank) - min(equal, rank);
        equal += all_e;
    }
}

template <typename T> static void scores(const SelectArgs &a, uint32_t groups, hipStream_t s)
{
    if (a.c.dim <= 64) score_kernel<T, 64><<<groups, 256, 0, s>>>(a);
    else if (a.c.dim <= 128) score_kernel<T, 128><<<groups, 256, 0, s>>>(a);
    else score_kernel<T, 256><<<groups, 256, 0, s>>>(a);
}

hipError_t launch_select(const SelectArgs &a, uint32_t dtype, hipStream_t s)
{
    const uint64_t items = (uint64_t)a.b.total_new * a.c.heads, groups = items * ((a.stride + 255u) / 256u);
    if (!launchable(items, kChooseThreads) || !launchable(groups, 256)) return hipErrorInvalidConfiguration;
    if (a.stride > a.n_select) {
        if (dtype == DMI_DTYPE_BF16) scores<Bf16>(a, (uint32_t)groups, s);
        else scores<Fp16>(a, (uint32_t)groups, s);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    choose_kernel<<<(uint32_t)items, kChooseThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace kv8
}  // namespace dmi
