// The quantizer of Sec. 3.2 over short runs of fp16 channels (a group of a weight row, a head of a cached row): the step
// is kept in fp16, the code of x is floor(x / step + 1/2).
#pragma once

#include "sq_common.h"

namespace sq {

// max(a, b) of two pairs of fp16 magnitudes (sign bits clear: the order of the bits is the order of the values)
__device__ __forceinline__ uint32_t max_magnitudes(uint32_t a, uint32_t b)
{
    typedef unsigned short v2us __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(v2us, a), __builtin_bit_cast(v2us, b)));
}

// Largest magnitude (fp16 bits) of the eight channels of every one of LANES neighbouring lanes, in all of them.
template <int LANES>
__device__ __forceinline__ uint32_t run_max(const uint4 x)
{
    static_assert(LANES == 4 || LANES == 8 || LANES == 16 || LANES == 32, "runs of 32 to 256 channels");
    constexpr uint32_t kMag = 0x7FFF7FFFu;
    uint32_t m = max_magnitudes(max_magnitudes(x.x & kMag, x.y & kMag), max_magnitudes(x.z & kMag, x.w & kMag));
#define SQ_DPP_MAX(ctrl) m = max_magnitudes(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, ctrl, 0xF, 0xF, false))
    SQ_DPP_MAX(0xB1);                          // quad_perm [1,0,3,2]
    SQ_DPP_MAX(0x4E);                          // quad_perm [2,3,0,1]
    if constexpr (LANES >= 8) SQ_DPP_MAX(0x141);       // row_half_mirror
    if constexpr (LANES >= 16) SQ_DPP_MAX(0x140);      // row_mirror
#undef SQ_DPP_MAX
    if constexpr (LANES >= 32) m = max_magnitudes(m, (uint32_t)__shfl_xor((int)m, 16, kWave));
    return max_magnitudes(m, m >> 16) & 0xFFFFu;
}

// step = fp16(max / 7), 1 where that is zero (an all-zero run, or one below 7 * 2^-25, whose codes are then all 0)
__device__ __forceinline__ __half run_step(uint32_t max_bits)
{
    const float top = __half2float(__ushort_as_half((unsigned short)max_bits));
    const __half s = __float2half_rn(top / 7.0f);
    return __half_as_ushort(s) == 0 ? __ushort_as_half(0x3C00) : s;
}

// Eight codes plus 8, one nibble each, the even channel low.  inv is 1 / step to within an ulp of fp32.
//
// floor(x inv + 1/2 + 2^-16) is floor(x / step + 1/2) exactly, halves going up: for x, step of fp16 a quotient that is
// no half-integer misses the next one by more than 2^-13 (both sides are integers below 2^11 over powers of two), the
// product and the sum are off by less than 2^-18 for quotients up to 16, and the added 2^-16 lies between the two.
// The nibbles are put together as digits of base 16 in fp32, four at a time (below 2^24: exact).
__device__ __forceinline__ uint32_t run_codes_plus8(const uint4 x, float inv)
{
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    float half4[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float u[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const v2h pair = __builtin_bit_cast(v2h, w[2 * h + e / 2]);
            const float t = __builtin_fmaf((float)pair[e & 1], inv, 0.5f + 0x1p-16f);
            u[e] = fminf(fmaxf(__builtin_floorf(t), -8.f), 7.f);
        }
        // (u + 8) in base 16: the eights of the four digits are 0x8888
        half4[h] = __builtin_fmaf(__builtin_fmaf(__builtin_fmaf(u[3], 16.f, u[2]), 16.f, u[1]), 16.f, u[0]) + 34952.f;
    }
    return (uint32_t)half4[0] | ((uint32_t)half4[1] << 16);
}

}  // namespace sq
