// MXFP4 (microscaled 4-bit floating point): device arithmetic shared by the
// quantizer and the linear layer.
//
// A block is 32 consecutive elements along K.  With a = max|x| of the block
// and e = floor(log2 a), its scale is 2^E, E = max(e - 2, -127) (2 is the
// exponent of e2m1's largest value, 6), stored as the byte E + 127, and the
// elements are x 2^-E rounded to e2m1 {0, .5, 1, 1.5, 2, 3, 4, 6}, ties to the
// even code, saturating at 6.  Everything is exact but that one rounding: E
// comes from the exponent bits of the bf16 maximum (subnormal maxima have
// e < -126 and take E = -127), and the conversion instruction rounds x / 2^E
// once (checked for every bf16 value at the lowest, ordinary and highest
// scales).  A block that holds an infinity or a NaN gets the byte 255, which
// the matrix instructions and the decoder read as NaN.
//
// Layout, for rows r of an [R][K] tensor (activations: R = M, weights: R = N):
//   codes   u8 [K/32][R][16]        element 2i of a block in the low half of byte i
//   scales  u8 [ceil(K/128)][R][4]  byte j of a word: block 4 w + j
// A 32-element block of a row is the 16 bytes that one lane gives a matrix
// instruction, and consecutive rows are consecutive: a fragment of 16 (32)
// rows is a run of 256 (512) bytes, and one word of scales serves four blocks.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace quartz {

constexpr int kMxBlock = 32;

inline int64_t mx_code_bytes(int64_t rows, int64_t K) { return rows * (K / 2); }
inline int64_t mx_scale_bytes(int64_t rows, int64_t K) { return (K + 127) / 128 * rows * 4; }

typedef unsigned short mx_us2 __attribute__((ext_vector_type(2)));
typedef __bf16 mx_bf2 __attribute__((ext_vector_type(2)));

// largest magnitude bits (15 bits each) of the bf16 pairs, per half
__device__ __forceinline__ uint32_t mx_max2(uint32_t a, uint32_t b)
{
    return __builtin_bit_cast(uint32_t,
                              __builtin_elementwise_max(__builtin_bit_cast(mx_us2, a & 0x7FFF7FFFu),
                                                        __builtin_bit_cast(mx_us2, b & 0x7FFF7FFFu)));
}
__device__ __forceinline__ uint32_t mx_max8(uint4 v)
{
    return mx_max2(mx_max2(v.x, v.y), mx_max2(v.z, v.w));
}

// magnitude bits of the block's maximum -> its scale byte
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t top)
{
    const uint32_t e = top >> 7;
    return e == 255u ? 255u : (uint32_t)max((int)e - 2, 0);
}

// eight bf16 values (four pairs) -> eight e2m1 codes of x / 2^E
__device__ __forceinline__ uint32_t mx_codes8(uint4 v, uint32_t byte)
{
    const float scale = __uint_as_float(byte << 23);
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(mx_bf2, v.x), scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(mx_bf2, v.y), scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(mx_bf2, v.z), scale, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(mx_bf2, v.w), scale, 3);
    return r;
}

}  // namespace quartz
