// Types and small pieces of the attention kernels that take tiles of 32 rows and 32 keys to the bf16 matrix cores.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ss {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint32_t pack_bf16(float x, float y)
{
    const float2v v = {x, y};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}
// four consecutive elements of bf16 or e4m3, from a multiple of four
template <bool FP8>
__device__ __forceinline__ float4v load4(const void *base, int64_t i)
{
    if constexpr (FP8) {
        const uint32_t w = *reinterpret_cast<const uint32_t *>(static_cast<const uint8_t *>(base) + i);
        const float2v x = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), y = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
        return float4v{x.x, x.y, y.x, y.y};
    } else {
        const uint2 w = *reinterpret_cast<const uint2 *>(static_cast<const uint16_t *>(base) + i);
        return float4v{__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u)};
    }
}
// x and the two of a pair of bf16, added
__device__ __forceinline__ float pair_sum(uint32_t pair, float x)
{
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), __builtin_bit_cast(bf16x2, 0x3f803f80u), x, false);
}
// What the lane of the row's other keys has, joined.
__device__ __forceinline__ float max_of_halves(float x)
{
    const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __builtin_elementwise_maximum(__uint_as_float(h[0]), __uint_as_float(h[1]));
}
__device__ __forceinline__ float sum_of_halves(float x)
{
    const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(h[0]) + __uint_as_float(h[1]);
}
// The place of a row's pieces of 16 bytes in LDS: piece c of row t stands at c ^ turn(t).
template <int D>
__device__ __forceinline__ int turn(int t)
{
    return D == 128 ? (t & 3) << 2 | (t >> 2 & 3) : (t >> 1 & 1) << 2 | (t >> 2 & 3);
}
// Waits until at most N of this wavefront's loads from memory (the youngest) are on their way, and keeps the compiler from moving accesses across.
template <int N>
__device__ __forceinline__ void wait_loads()
{
    static_assert(N < 16, "the low bits of the count");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0f70 | N);
    asm volatile("" ::: "memory");
}
// Waits for this wavefront's LDS accesses, and keeps the compiler from moving any across.
__device__ __forceinline__ void wave_lds_fence()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0)
    asm volatile("" ::: "memory");
}

}  // namespace
}  // namespace ss
