// What the attention kernels of the 8-bit KV cache share: the types that matrix instructions take, conversions into them.
#pragma once
#include "dmi_kv8_internal.h"

#include <hip/hip_fp16.h>

namespace dmi {
namespace kv8 {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// Matrix instructions take bf16 or f16 as q comes; an e4m3 number is one of either exactly.
struct Bf16 {
    static constexpr bool kNarrow = false;      // as wide a range of exponents as fp32
    static constexpr uint32_t kOne = 0x3F80u, kExponent = 0x7F80u;
    static __device__ __forceinline__ float number(uint16_t w) { return __uint_as_float((uint32_t)w << 16); }
    // two neighbouring codes of a word, times a power of two
    static __device__ __forceinline__ uint32_t two_codes(uint32_t w, bool hi, float power = 1.0f)
    {
        return __builtin_bit_cast(uint32_t, hi ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, power, true)
                                               : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, power, false));
    }
    static __device__ __forceinline__ uint32_t pack(float a, float b)
    {
        const f32x2 v = {a, b};
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
    }
    static __device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};

struct Fp16 {
    static constexpr bool kNarrow = true;
    static constexpr uint32_t kOne = 0x3C00u, kExponent = 0x7C00u;
    static __device__ __forceinline__ float number(uint16_t w) { return (float)__builtin_bit_cast(_Float16, w); }
    static __device__ __forceinline__ uint32_t two_codes(uint32_t w, bool hi, float power = 1.0f)
    {
        return __builtin_bit_cast(uint32_t, hi ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, power, true)
                                               : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, power, false));
    }
    static __device__ __forceinline__ uint32_t pack(float a, float b)
    {
        const f32x2 v = {a, b};
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
    }
    static __device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
};

// Loads at 32-bit offsets from an address that is the same in every lane.  kOnce in the last argument: the line is not read
// again soon.
typedef __amdgpu_buffer_rsrc_t Buffer;
constexpr int kOnce = 2;
__device__ __forceinline__ Buffer buffer_at(const uint8_t *p)
{
    // (said to be the same in every lane: a load from what may differ becomes a loop over the lanes' addresses)
    const uint64_t at = (uint64_t)p;
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)at), hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(at >> 32));
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>((uint64_t)hi << 32 | lo), 0, 0x7FFFFFFF, 0x00027000);
}
template <int AUX> __device__ __forceinline__ u32x4 load_b128(Buffer b, uint32_t at)
{
    return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(b, (int)at, 0, AUX));
}
template <int AUX> __device__ __forceinline__ u32x2 load_b64(Buffer b, uint32_t at)
{
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(b, (int)at, 0, AUX));
}
template <int AUX> __device__ __forceinline__ uint32_t load_b32(Buffer b, uint32_t at)
{
    return __builtin_amdgcn_raw_buffer_load_b32(b, (int)at, 0, AUX);
}

// A barrier for what passes through LDS: __syncthreads() waits for loads from memory as well, also for those that a loop has
// just started for its next round.
__device__ __forceinline__ void lds_barrier()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// The same among the lanes of one wavefront, whose accesses to LDS are carried out in order: only the compiler has to keep it.
__device__ __forceinline__ void lds_handover()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_of(float x) { return __builtin_amdgcn_logf(x); }
constexpr float kLn2 = 0.693147180559945309417f;

template <int N> struct Int {
    static constexpr int value = N;
};

// Sums over lanes that differ in one bit of their number: of the 2 N values each lane goes on with the sums of N, the upper half of
// them where its bit is set.
template <int BIT, int N> __device__ __forceinline__ void halve(float *x, int lane)
{
#pragma unroll
    for (int e = 0; e < N; e++) {
        const float low = x[e], high = x[e + N], other = __shfl_xor(lane & BIT ? low : high, BIT);
        x[e] = (lane & BIT ? high : low) + other;
    }
}

// Scores may rise this far (as powers of two) above the maximum that p is taken against before everything is taken against
// a new one: p stays below 2^8, which costs no precision, and the rescaling becomes rare.
constexpr float kSlack = 8.0f;

// V's scale is m 2^e, 1 <= m < 2 (more where e would pass 119).  m goes into p, in fp32 and before p's one rounding; 2^e goes into the codes as they are converted,
// without one: bf16 holds every code times 2^-117 to 2^119.  fp16 holds them times 2^-15 to 2^7.  There outputs are summed in units of
// 2^unit and codes converted times 2^(e - unit); a tile some of whose scales lie outside of that takes another unit, to which the sums are
// brought first (in fp32, by a power of two: nothing is rounded).  Where a tile's own scales are further apart than 2^22 the largest
// ones are held exactly and the others to 2^-32 of them: less than half of fp16's smallest number, as long as V's own numbers
// are none that fp16 cannot hold.  So is what a scale below 2^-40 stands for, which therefore moves no unit.
__device__ __forceinline__ int exponent_of(uint32_t bits) { return min(max((int)(bits >> 23), 1) - 127, 119); }
__device__ __forceinline__ float mantissa_of(uint32_t bits) { return __uint_as_float(bits - ((uint32_t)exponent_of(bits) << 23)); }
__device__ __forceinline__ float power_of(int e) { return __uint_as_float((uint32_t)(max(e, -126) + 127) << 23); }
constexpr int kLeast = -15, kMost = 7, kFaint = -40;
__device__ __forceinline__ bool outside(int e, int unit) { return e >= kFaint && (e < unit + kLeast || e > unit + kMost); }
template <int N> __device__ __forceinline__ int unit_for(int unit, const int (&e)[N])
{
    int hi = kFaint, lo = 127;                  // of the scales that count
#pragma unroll
    for (int x = 0; x < N; x++) hi = max(hi, e[x]), lo = min(lo, e[x] < kFaint ? 127 : e[x]);
    if (lo == 127 || (hi <= unit + kMost && lo >= unit + kLeast)) return unit;
    return max(hi - kMost, min(hi, lo - kLeast));
}

// The top bit of every byte of w that is a NaN.
__device__ __forceinline__ uint32_t nan_codes(uint32_t w) { return ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u; }

// A query row among those that share a head of the cache: row = token * group + query head within the group.
struct QueryRow {
    int token;
    uint32_t head;
};
__device__ __forceinline__ QueryRow query_row(const AttendArgs &a, uint32_t head, uint32_t row)
{
    const uint32_t i = row / a.group;
    return {(int)i, head * a.group + (row - i * a.group)};
}

}  // namespace kv8
}  // namespace dmi
