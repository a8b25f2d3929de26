// Values in 4 bits: E2M1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign) with one power of two for every 32 of them (E8M0: 2^(byte - 127)).
//
// The power of two of a block is that of its largest magnitude, rounded to the two bits of significand that an element has, so that the
// largest element falls on 4 or 6 and nothing is off by more than half a step: bits of a float + 0x1FFFFF carry into the exponent above 7/4.
// It is kept within 2^-125 .. 2^125, where every product of element and power is a normal bf16 (and fp32) number: reading a cache rounds
// nothing.  (The conversions read the exponent bits of a scale alone: bytes 0 and 1, which other encoders write, come out right, with their subnormal
// values.)  Elements are rounded to nearest, ties to the even code, and end at 6; a block that holds an infinity or a NaN gets the byte 255,
// for which the conversion instructions give NaN.  Both directions are single instructions for two values.
#pragma once

#include "common.h"

namespace sepattn {

constexpr int kFp4Block = 32;  // values that share a scale
constexpr uint32_t kFp4Nan = 255;

typedef __bf16 fp4_bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 fp4_bf16x8 __attribute__((ext_vector_type(8)));
typedef float fp4_f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned short fp4_u16x2 __attribute__((ext_vector_type(2)));

// the scale byte of a block whose largest magnitude has these bits
__device__ inline uint32_t fp4_scale_byte(uint32_t largest) {
    const int s = (int)((largest + 0x1FFFFFu) >> 23) - 2;
    return largest >= 0x7F800000u ? kFp4Nan : (uint32_t)min(max(s, 2), 252);
}
// byte `i` of the packed scale bytes of a row, as the float that the conversions take
__device__ inline float fp4_scale(uint32_t bytes, int i) { return __uint_as_float(((bytes >> (8 * i)) & 0xFFu) << 23); }

// bits of the largest magnitude of eight values (a NaN counts as larger than everything)
__device__ inline uint32_t fp4_largest(const uint4 &x) {  // bf16
    auto mag = [](uint32_t u) { return __builtin_bit_cast(fp4_u16x2, u & 0x7FFF7FFFu); };
    const fp4_u16x2 m = __builtin_elementwise_max(__builtin_elementwise_max(mag(x.x), mag(x.y)), __builtin_elementwise_max(mag(x.z), mag(x.w)));
    return (uint32_t)max(m.x, m.y) << 16;
}
__device__ inline uint32_t fp4_largest(const uint4 &x, const uint4 &y) {  // fp32
    constexpr uint32_t k = 0x7FFFFFFFu;
    return max(max(max(x.x & k, x.y & k), max(x.z & k, x.w & k)), max(max(y.x & k, y.y & k), max(y.z & k, y.w & k)));
}

// eight values as codes (value i in bits 4i .. 4i+3)
__device__ inline uint32_t fp4_codes(const uint4 &x, float scale) {  // bf16
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(fp4_bf16x2, x.x), scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(fp4_bf16x2, x.y), scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(fp4_bf16x2, x.z), scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(fp4_bf16x2, x.w), scale, 3);
}
__device__ inline uint32_t fp4_codes(const uint4 &x, const uint4 &y, float scale) {  // fp32
    auto f = [](uint32_t u) { return __uint_as_float(u); };
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f(x.x), f(x.y), scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f(x.z), f(x.w), scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f(y.x), f(y.y), scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f(y.z), f(y.w), scale, 3);
}

// the values of eight codes
__device__ inline fp4_bf16x8 fp4_to_bf16(uint32_t codes, float scale) {
    const fp4_bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1),
                     c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
    return fp4_bf16x8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}
__device__ inline void fp4_to_f32(uint32_t codes, float scale, float (&v)[8]) {
    const fp4_f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1),
                    c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 3);
    v[0] = a.x, v[1] = a.y, v[2] = b.x, v[3] = b.y, v[4] = c.x, v[5] = c.y, v[6] = d.x, v[7] = d.y;
}

// largest value over the four neighbouring lanes that hold one block
__device__ inline uint32_t fp4_block_max(uint32_t x) {
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, true));   // quad_perm [1, 0, 3, 2]
    return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, true));  // quad_perm [2, 3, 0, 1]
}

// Eight consecutive values of a row per lane (D / 8 neighbouring lanes a row) -> their codes, and the row's scale bytes in every lane
struct Fp4Piece {
    uint32_t codes, scales;
};
template <int D>
__device__ inline uint32_t fp4_row_scales(uint32_t byte, int piece) {  // piece: which of the row's D / 8
    uint32_t s = byte << (8 * (piece >> 2));
    s |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)s, 0x141, 0xF, 0xF, true);  // row_half_mirror: the other four of eight lanes
    if constexpr (D == 128) s |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)s, 0x140, 0xF, 0xF, true);  // row_mirror
    return s;
}
template <int D>
__device__ inline Fp4Piece fp4_round(const uint4 &x, int piece) {  // bf16
    const uint32_t byte = fp4_scale_byte(fp4_block_max(fp4_largest(x)));
    return {byte == kFp4Nan ? 0u : fp4_codes(x, fp4_scale(byte, 0)), fp4_row_scales<D>(byte, piece)};
}
template <int D>
__device__ inline Fp4Piece fp4_round(const uint4 &x, const uint4 &y, int piece) {  // fp32
    const uint32_t byte = fp4_scale_byte(fp4_block_max(fp4_largest(x, y)));
    return {byte == kFp4Nan ? 0u : fp4_codes(x, y, fp4_scale(byte, 0)), fp4_row_scales<D>(byte, piece)};
}

// a row's scale bytes: one word (d = 128) or half of one
template <int D>
using Fp4Scales = std::conditional_t<D == 128, uint32_t, uint16_t>;

}  // namespace sepattn
