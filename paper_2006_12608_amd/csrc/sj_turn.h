// sj_turn.h -- the arithmetic of rotary positions, shared by the kernels that turn rows
// (sj_rotary.hip, sj_append8.hip).
#pragma once

#include "sj_cache.h"

namespace sjc {

__device__ __forceinline__ float to_float(int dt, uint32_t x)
{
    return dt == sjk::DT_F16 ? (float)__builtin_bit_cast(_Float16, (uint16_t)x)
                             : __uint_as_float(x << 16);
}

__device__ __forceinline__ uint32_t to_bits(int dt, float x)
{
    return dt == sjk::DT_F16 ? (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)x)
                             : (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x);
}

// The turned pair.  Which product is fused with the sum is said, not left to the compiler, so that
// all variants, and the two items of a chunk that is moved back, round alike.
__device__ __forceinline__ float turn_a(float a, float b, float c, float s)
{
    return __builtin_fmaf(a, c, -(b * s));
}

__device__ __forceinline__ float turn_b(float a, float b, float c, float s)
{
    return __builtin_fmaf(b, c, a * s);
}

// Cosine and sine of pair p at a position, times the factor.
__device__ __forceinline__ float2 sine_of(const Turn &t, uint64_t pos, uint32_t p)
{
    const uint64_t phase = pos * (uint64_t)t.turns[p];
    // signed fraction of a turn; 2^-31 half turns a unit
    const float half = (float)(int32_t)(phase >> 32) * 4.656612873077393e-10f;
    float s, c;
    sincospif(half, &s, &c);
    return float2{c * t.factor, (t.inverse ? -s : s) * t.factor};
}

}  // namespace sjc
