// Rows of a cache held in 4 bits.
//
// A group of 32 values of a row shares a power-of-two scale X, kept as the byte
// of its biased exponent; a value is the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6
// times X with its sign (a 4-bit float, 1 sign, 2 exponent and 1 mantissa bits),
// ties to the even code, and 6 X for what lies above.  X is the smallest power of
// two with max|x| < 7 X: no value is then off by more than X, half of the widest
// step.  X lies in 2^-100 .. 2^125, so that no product is subnormal or passes the
// largest bf16; a smaller group reads as zeros.  A group with an infinity or a NaN
// has scale byte 255 and reads as NaN.  The values are exact in bf16, so what is
// computed from them is as exact as from bf16 rows.
//
// A row of one KV head is D / 2 bytes of codes (value 2 i in the low half of byte i),
// so that 16 bytes are one group; the D / 32 scale bytes stand in an array of their
// own, row by row.  Behind the codes, in rows of 68 bytes (D = 128), they spare a dense
// launch a second stream, which no longer showed once that stream went past the caches
// (8 x 32k tokens, 8 KV heads: 66.3 us behind the codes, 64.6 in their own array), and the
// rows of a list with gaps straddle lines: 47.6 us against 38.4 where 35 % attend.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace asrkf {

constexpr int kScaleGroup = 32;

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short ushortx2 __attribute__((ext_vector_type(2)));
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));

// the larger magnitudes of two pairs of bf16, as bits
__device__ __forceinline__ uint32_t max_magnitude(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(ushortx2, a & 0x7FFF7FFFu),
                                                                  __builtin_bit_cast(ushortx2, b & 0x7FFF7FFFu)));
}

// scale byte of a group, from the bits of its largest magnitude
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax) {
    if (amax >= 0x7F80u) return 255u;
    const int e = (int)((amax + 0x20u) >> 7) - 2;     // 7 X for the power of two below passes at 1.75
    return (uint32_t)(e < 27 ? 27 : e > 252 ? 252 : e);
}

__device__ __forceinline__ float scale_value(uint32_t byte) { return __uint_as_float(byte << 23); }

// eight bf16 (four pairs) as eight codes
__device__ __forceinline__ uint32_t encode8(uint32_t a, uint32_t b, uint32_t c, uint32_t d, float scale) {
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, a), scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, b), scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, c), scale, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, d), scale, 3);
    return r;
}

// codes 2 SEL and 2 SEL + 1 of a word as two bf16
template <int SEL>
__device__ __forceinline__ uint32_t decode2(uint32_t codes, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, SEL));
}

// Eight values of a row, whose group's others the lane's three neighbours hold, as
// codes, and (lanes at the start of a row's 16, or of rows of 64 values at the start of
// its 8) the scale bytes of those lanes' groups.
__device__ __forceinline__ uint32_t round8(uintx4 x, bool rows_of_64, uint32_t& scales) {
    uint32_t top = max_magnitude(max_magnitude(x[0], x[1]), max_magnitude(x[2], x[3]));
    top = max(top & 0xFFFFu, top >> 16);
    top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xF, 0xF, false));   // quad_perm [1,0,3,2]
    top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xF, 0xF, false));   // quad_perm [2,3,0,1]
    const uint32_t byte = scale_byte(top);
    scales = byte << (threadIdx.x / 4 & (rows_of_64 ? 1 : 3)) * 8;
    if (rows_of_64) {
        scales |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)scales, 0x141, 0xF, 0xF, false);     // row_half_mirror
    } else {
        scales |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)scales, 0x124, 0xF, 0xF, false);     // row_ror 4
        scales |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)scales, 0x128, 0xF, 0xF, false);     // row_ror 8
    }
    return encode8(x[0], x[1], x[2], x[3], scale_value(byte));
}

}  // namespace asrkf
