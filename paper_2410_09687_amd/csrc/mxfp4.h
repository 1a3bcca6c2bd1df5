// MXFP4: blocks of 32 values of E2M1 (0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives, four bits each) that share a power of
// two 2^(E - 127), E one byte.  What a code stands for is exact in bf16, so products with bf16 operands are exact and the
// matrix cores' fp32 sums are the only rounding.
#pragma once
#include "gemm_core.h"

namespace moin {

// Scale byte of a block whose largest magnitude has these fp32 bits: the smallest power of two in whose units it rounds to 6
// or less (7 units and more round to 8), so no value is clamped: rms error 0.112 of a Gaussian's deviation, 0.115 with
// the floor of the logarithm alone.  At least 2: every value that a code stands for is then a normal number.  127 for a block of
// zeros; 255, which stands for NaN, where a value is infinite or NaN.  At most 252: 6 units are the largest value then that bf16 holds
// (what is beyond 7 of them, 2.98e38, becomes 6).
__device__ __forceinline__ uint32_t mx4_scale_byte(uint32_t amax)
{
    const int e = (int)((amax + 0x200000u) >> 23) - 2;
    return amax == 0 ? 127u : amax >= 0x7F800000u ? 255u : (uint32_t)min(max(e, 2), 252);
}
// The scale's operand of the conversions, which go by the exponent field alone: sign and mantissa may hold anything, so that
// byte `i` of a word is one shift away from it.
__device__ __forceinline__ float mx4_scale(uint32_t word, int i)
{
    return bits_f32(i < 3 ? word << (23 - 8 * i) : word >> 1);
}
// Eight bf16 (a word of two each) to a word of codes, the first value in the lowest bits; nearest, ties to even.
__device__ __forceinline__ uint32_t mx4_encode(const uint4 &v, float scale)
{
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, v.x), scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, v.y), scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, v.z), scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, v.w), scale, 3);
}
template <int BYTE>
__device__ __forceinline__ uint32_t mx4_pair(uint32_t codes, float scale)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, BYTE));
}
__device__ __forceinline__ uint4 mx4_decode(uint32_t codes, float scale)
{
    return make_uint4(mx4_pair<0>(codes, scale), mx4_pair<1>(codes, scale), mx4_pair<2>(codes, scale), mx4_pair<3>(codes, scale));
}
// Largest magnitude of eight bf16, as fp32 bits.
__device__ __forceinline__ uint32_t bf16x8_amax(const uint4 &v)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = max(m, max((w[i] << 16) & 0x7FFF0000u, w[i] & 0x7FFF0000u));
    return m;
}

}  // namespace moin
