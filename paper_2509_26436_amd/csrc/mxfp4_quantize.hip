// MXFP4 quantizer and decoder (mxfp4.h has the format): one pass over memory.
//
// A wave takes 16 rows x 128 elements: lane 4 r + q holds elements 8 q .. 8 q + 7
// of each of the four blocks of row r, so that a load instruction reads 64
// bytes of 16 rows, the four of them whole 256-byte stretches of each row, a
// block's maximum is a reduction over 4 lanes, a store of codes writes 256
// contiguous bytes (16 rows of one block), and the row's four scales are one
// word.
#include "mxfp4.h"
#include "quartz_internal.h"

namespace quartz {
namespace {

constexpr int kWaves = 4;

template <int CTRL>
__device__ __forceinline__ uint32_t quad(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, false);
}

__global__ __launch_bounds__(64 * kWaves) void mxfp4_quantize_kernel(
    const uint16_t* __restrict__ x, int64_t M, int32_t K, int64_t ldx, uint32_t words,
    uint8_t* __restrict__ codes, uint8_t* __restrict__ scales)
{
    const int lane = threadIdx.x & 63, q = lane & 3;
    const uint32_t item = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t tile = item / words, word = item - tile * words;
    const int64_t row = (int64_t)tile * 16 + (lane >> 2);
    if (row >= M)
        return;
    const int blocks = min(4, (K >> 5) - 4 * (int)word);
    const uint16_t* src = x + row * ldx + (int64_t)word * 128 + 8 * q;
    uint4 v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
        v[j] = j < blocks ? *reinterpret_cast<const uint4*>(src + 32 * j) : uint4{0, 0, 0, 0};
    uint32_t packed = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t top = mx_max8(v[j]);
        top = max(top & 0xFFFFu, top >> 16);
        top = max(top, quad<0xB1>(top));       // quad_perm [1,0,3,2]
        top = max(top, quad<0x4E>(top));       // quad_perm [2,3,0,1]
        const uint32_t byte = mx_scale_byte(top);
        packed |= byte << (8 * j);
        if (j < blocks)
            *reinterpret_cast<uint32_t*>(codes + (((int64_t)word * 4 + j) * M + row) * 16 + 4 * q) =
                mx_codes8(v[j], byte);
    }
    if (q == 0)
        *reinterpret_cast<uint32_t*>(scales + ((int64_t)word * M + row) * 4) = packed;
}

__global__ __launch_bounds__(64 * kWaves) void mxfp4_dequantize_kernel(
    const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t M, int32_t K,
    uint32_t words, uint16_t* __restrict__ y, int64_t ldy)
{
    const int lane = threadIdx.x & 63, q = lane & 3;
    const uint32_t item = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t tile = item / words, word = item - tile * words;
    const int64_t row = (int64_t)tile * 16 + (lane >> 2);
    if (row >= M)
        return;
    const int blocks = min(4, (K >> 5) - 4 * (int)word);
    uint32_t c[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
        c[j] = j < blocks ? *reinterpret_cast<const uint32_t*>(
                                codes + (((int64_t)word * 4 + j) * M + row) * 16 + 4 * q)
                          : 0u;
    const uint32_t packed = *reinterpret_cast<const uint32_t*>(scales + ((int64_t)word * M + row) * 4);
    uint16_t* dst = y + row * ldy + (int64_t)word * 128 + 8 * q;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t byte = (packed >> (8 * j)) & 255u;
        const float scale = __uint_as_float(byte << 23);
        uint4 v;
        v.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[j], scale, 0));
        v.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[j], scale, 1));
        v.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[j], scale, 2));
        v.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[j], scale, 3));
        if (byte == 255u)
            v = uint4{0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u};
        if (j < blocks)
            *reinterpret_cast<uint4*>(dst + 32 * j) = v;
    }
}

// blocks of one launch; M K / 64 <= 2^28 keeps the items below 2^25
uint32_t grid_of(int64_t M, uint32_t words)
{
    return (uint32_t)(((M + 15) / 16 * words + kWaves - 1) / kWaves);
}

}  // namespace

hipError_t launch_mxfp4_quantize(const uint16_t* x, int64_t M, int64_t K, int64_t ldx, uint8_t* codes,
                                 uint8_t* scales, hipStream_t stream)
{
    const uint32_t words = (uint32_t)((K + 127) / 128);
    mxfp4_quantize_kernel<<<grid_of(M, words), 64 * kWaves, 0, stream>>>(x, M, (int32_t)K, ldx, words, codes, scales);
    return hipGetLastError();
}

hipError_t launch_mxfp4_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t M, int64_t K,
                                   uint16_t* y, int64_t ldy, hipStream_t stream)
{
    const uint32_t words = (uint32_t)((K + 127) / 128);
    mxfp4_dequantize_kernel<<<grid_of(M, words), 64 * kWaves, 0, stream>>>(codes, scales, M, (int32_t)K, words, y, ldy);
    return hipGetLastError();
}

}  // namespace quartz
