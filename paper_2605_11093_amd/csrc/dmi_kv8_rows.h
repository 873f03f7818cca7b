// Rows as they come from a model, in bf16, fp16 or fp32, for the kernels that write the 8-bit KV cache.
#pragma once
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

}  // namespace kv8
}  // namespace dmi
