// Channel-wise minima and maxima of bf16 keys, two channels per register, for
// the kernels that build cuboid metadata.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace ss {

typedef short i16x2_t __attribute__((ext_vector_type(2)));

// two bf16 values -> two 16-bit keys whose signed order is IEEE totalOrder
// (-0 < +0): negative values flip their magnitude bits.  Its own inverse.
__device__ __forceinline__ uint32_t key2(uint32_t w)
{
    const i16x2_t sign = __builtin_bit_cast(i16x2_t, w) >> 15;
    return w ^ (__builtin_bit_cast(uint32_t, sign) & 0x7FFF7FFFu);
}

__device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b)
{
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(i16x2_t, a),
                                                                  __builtin_bit_cast(i16x2_t, b)));
}

// lanes 0..31: the minimum of a over its two halves, lanes 32..63: that of b
__device__ __forceinline__ uint32_t min_halves(uint32_t a, uint32_t b)
{
    const auto x = __builtin_amdgcn_permlane32_swap(a, b, false, false);
    return min2(x[0], x[1]);
}

// per 32 lanes: the first 16 hold the minimum of a over its two 16-lane rows, the others that of b
__device__ __forceinline__ uint32_t min_rows(uint32_t a, uint32_t b)
{
    const auto x = __builtin_amdgcn_permlane16_swap(a, b, false, false);
    return min2(x[0], x[1]);
}

}  // namespace ss
