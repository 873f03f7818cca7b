// Kernels of attention over the 8-bit KV cache.
#include "dmi_internal.h"
#include "dmi_kv8_internal.h"

#include <hip/hip_fp16.h>

namespace dmi {
namespace kv8 {

struct PlainBf16 { uint16_t u; };
__device__ __forceinline__ float number(PlainBf16 x) { return __uint_as_float((uint32_t)x.u << 16); }
__device__ __forceinline__ float number(_Float16 x) { return (float)x; }
__device__ __forceinline__ void put(PlainBf16 *p, float x)
{
    const uint32_t u = __float_as_uint(x);
    p->u = x != x ? 0x7FC0u : (uint16_t)((u + 0x7FFFu + (u >> 16 & 1u)) >> 16);
}
__device__ __forceinline__ void put(_Float16 *p, float x) { *p = (_Float16)x; }

__device__ __forceinline__ float code_number(uint8_t c) { return __builtin_amdgcn_cvt_f32_fp8((int)c, 0); }

// Score of token t, as a power of two
template <typename T>
__device__ __forceinline__ float score(const AttendArgs &a, const Request &r, const T *q, uint32_t head, int t)
{
    const uint32_t block = block_of(a.c, (uint32_t)t >> 4);
    const int b = entry_of(a.c, r.row, block);
    if (b < 0) return -INFINITY;
    const uint8_t *k = code_at(a.c, 0, b, (uint32_t)t - block * a.c.bs, head);
    float z = 0.0f;
    for (uint32_t d = 0; d < a.c.dim; d++) z += number(q[d]) * code_number(k[d]);
    return z * *scale_at(a.c, 0, b, head) * a.scale_log2;
}

// One workgroup per (new token, query head): a token a thread for the scores, an element a thread for the output.
template <typename T>
__global__ __launch_bounds__(256) void plain_attend_kernel(AttendArgs a, float *lse2)
{
    __shared__ float p[256], red[256];
    const uint32_t tid = threadIdx.x, qh = blockIdx.x, head = qh / a.group, n = blockIdx.y;
    const Request r = request_of(a.b, a.c, (int)n);
    for (int i = (int)blockIdx.z; i < r.fresh; i += (int)gridDim.z) {
        const int64_t row = r.start + i;
        const T *q = static_cast<const T *>(a.q.data) + row * a.q.row_stride + (int64_t)qh * a.q.head_stride;
        const int seen = max(r.len - r.fresh + i + 1, 0);
        float m = -INFINITY, l = 0.0f, o = 0.0f;
        for (int t0 = 0; t0 < seen; t0 += 256) {
            const int t = t0 + (int)tid;
            const float z = t < seen ? score(a, r, q, head, t) : -INFINITY;
            red[tid] = z;
            __syncthreads();
            float top = m;
            bool nan = false;
            for (int j = 0; j < 256; j++) nan |= red[j] != red[j], top = fmaxf(top, red[j]);
            if (nan) top = NAN;
            const float base = top == -INFINITY ? 0.0f : top;
            p[tid] = exp2f(z - base);
            const float f = exp2f(m - base);
            m = top;
            __syncthreads();
            l *= f;
            o *= f;
            for (int j = 0; j < min(256, seen - t0); j++) {
                l += p[j];
                const uint32_t block = block_of(a.c, (uint32_t)(t0 + j) >> 4);
                const int b = entry_of(a.c, r.row, block);
                if (b >= 0 && tid < a.c.dim)
                    o += p[j] * (code_number(code_at(a.c, 1, b, (uint32_t)(t0 + j) - block * a.c.bs, head)[tid]) * *scale_at(a.c, 1, b, head));
            }
            __syncthreads();
        }
        const bool empty = m == -INFINITY;
        if (tid < a.c.dim)
            put(static_cast<T *>(a.out.data) + row * a.out.row_stride + (int64_t)qh * a.out.head_stride + tid, empty ? 0.0f : o / l);
        if (!tid) {
            const float total = empty ? -INFINITY : m + log2f(l);
            if (a.lse) a.lse[row * a.q_heads + qh] = total * 0.693147180559945309417f;
            if (lse2) lse2[row * a.q_heads + qh] = total;
        }
    }
}

template <typename T>
__global__ __launch_bounds__(256) void plain_weight_kernel(AttendArgs a, const float *lse2)
{
    const uint32_t head = blockIdx.y, n = blockIdx.z;
    const int t = (int)(blockIdx.x * 256u + threadIdx.x);
    const Request r = request_of(a.b, a.c, (int)n);
    if (t >= r.len) return;
    const int64_t at = (int64_t)r.row * a.w.row_stride + (int64_t)head * a.w.head_stride + t;
    float w = 0.0f;
    if (a.prior.data && t < r.len - r.fresh)
        w = a.decay * a.prior.data[(int64_t)r.row * a.prior.row_stride + (int64_t)head * a.prior.head_stride + t];
    float sum = 0.0f;
    for (int i = max(t - (r.len - r.fresh), 0); i < r.fresh; i++)
        for (uint32_t g = 0; g < a.group; g++) {
            const int64_t row = r.start + i;
            const uint32_t qh = head * a.group + g;
            const float total = lse2[row * a.q_heads + qh];
            if (total == -INFINITY) continue;
            sum += exp2f(score(a, r, static_cast<const T *>(a.q.data) + row * a.q.row_stride + (int64_t)qh * a.q.head_stride, head, t) - total);
        }
    a.w.data[at] = w + sum;
}

template <typename T> hipError_t attend(const AttendArgs &a, float *lse2, hipStream_t s)
{
    plain_attend_kernel<T><<<dim3(a.q_heads, a.b.n_reqs, min(a.b.max_new, 1024u)), 256, 0, s>>>(a, lse2);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.w.data || !a.b.max_len) return e;
    plain_weight_kernel<T><<<dim3((a.b.max_len + 255u) / 256u, a.c.heads, a.b.n_reqs), 256, 0, s>>>(a, lse2);
    return hipGetLastError();
}

hipError_t launch_attend(const AttendArgs &a, uint32_t dtype, float *lse2, hipStream_t s)
{
    return dtype == DMI_DTYPE_BF16 ? attend<PlainBf16>(a, lse2, s) : attend<_Float16>(a, lse2, s);
}

}  // namespace kv8
}  // namespace dmi
