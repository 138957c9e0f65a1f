// MXFP4 quantizer and decoder (mxfp4.h has the format): one pass over memory,
// which bounds both (18432 x 4608: 35.7 us, 6.0 TB/s, and 32.6).
//
// A wave takes 16 rows x 128 elements.  On the bf16 side an access of the wave is
// the 128-byte halves (two blocks) of eight rows: lane 8 r + 4 c + i has eight
// elements of block c of row r, those from 8 i (c = 0) or 8 (3 - i) (c = 1) on.
// On the side of the codes it is one block of all 16 rows, 256 contiguous bytes:
// lanes of c = 0 have rows 0 to 7, those of c = 1 rows 8 to 15.  Between the two
// each lane exchanges half of its words with lane 7 - i of its eight, which is
// why c = 1 counts backwards.  With 64-byte pieces of 16 rows on the bf16 side,
// which need no exchange, loads around the caches fetch lines twice: 42.3 and
// 45.0 us.
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

// the word of lane 7 - i of the same eight lanes
__device__ __forceinline__ uint32_t mirrored(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, false);
}

typedef uint32_t v4u __attribute__((ext_vector_type(4)));

// the work of a wave and the place of a lane in it
struct Lane {
    uint32_t tile, word;
    int64_t row0;                                  // bf16 side: rows row0 and row0 + 8
    int64_t row;                                   // codes
    int blocks;                                    // of this word: 2 or 4
    bool odd;
    int q;                                         // of the four words of a block's codes
};
__device__ __forceinline__ Lane lane_of(uint32_t words, int32_t K)
{
    Lane l;
    const int lane = threadIdx.x & 63;
    const uint32_t item = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    l.tile = item / words;
    l.word = item - l.tile * words;
    l.row0 = (int64_t)l.tile * 16 + (lane >> 3);
    l.odd = lane & 4;
    l.row = l.row0 + (l.odd ? 8 : 0);
    l.blocks = min(4, (K >> 5) - 4 * (int)l.word);
    l.q = l.odd ? 3 - (lane & 3) : lane & 3;
    return l;
}

// PAST: x is read around the caches
template <bool PAST>
__global__ __launch_bounds__(64 * kWaves) void mxfp4_quantize_kernel(
    const uint16_t* __restrict__ x, int64_t M, int32_t K, int64_t ldx, uint32_t words,
    uint8_t* __restrict__ codes, uint8_t* __restrict__ scales)
{
    const Lane l = lane_of(words, K);
    if ((int64_t)l.tile * 16 >= M)                 // whole waves: the others' lanes all exchange
        return;
    uint4 v[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint16_t* src =
            x + min(l.row0 + 8 * i, M - 1) * ldx + (int64_t)l.word * 128 + (l.odd ? 32 : 0) + 8 * l.q;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            v4u w = {0, 0, 0, 0};
            if (2 * j < l.blocks) {
                const v4u* p = reinterpret_cast<const v4u*>(src + 64 * j);
                w = PAST ? __builtin_nontemporal_load(p) : *p;
            }
            v[i][j] = uint4{w[0], w[1], w[2], w[3]};
        }
    }
    uint32_t code[2][2], packed[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        packed[i] = 0;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            uint32_t top = mx_max8(v[i][j]);
            top = max(top & 0xFFFFu, top >> 16);
            top = max(top, quad<0xB1>(top));       // quad_perm [1,0,3,2]
            top = max(top, quad<0x4E>(top));       // quad_perm [2,3,0,1]
            const uint32_t byte = mx_scale_byte(top);
            packed[i] |= byte << (16 * j);
            code[i][j] = mx_codes8(v[i][j], byte);
        }
        packed[i] <<= l.odd ? 8 : 0;
        packed[i] |= mirrored(packed[i]);
    }
    uint32_t first[2], second[2];                  // codes of blocks 2 j and 2 j + 1
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const uint32_t got = mirrored(l.odd ? code[0][j] : code[1][j]);
        first[j] = l.odd ? got : code[0][j];
        second[j] = l.odd ? code[1][j] : got;
    }
    if (l.row >= M)
        return;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        if (2 * j >= l.blocks)
            break;
        uint8_t* dst = codes + (((int64_t)l.word * 4 + 2 * j) * M + l.row) * 16 + 4 * l.q;
        *reinterpret_cast<uint32_t*>(dst) = first[j];
        *reinterpret_cast<uint32_t*>(dst + M * 16) = second[j];
    }
    if (l.q == 0)
        *reinterpret_cast<uint32_t*>(scales + ((int64_t)l.word * M + l.row) * 4) = l.odd ? packed[1] : packed[0];
}

// Writes around the caches, whole lines at a time: 32.6 us where ordinary
// stores take 43.6.
__global__ __launch_bounds__(64 * kWaves) void mxfp4_dequantize_kernel(
    const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t M, int32_t K,
    uint32_t words, uint16_t* __restrict__ y, int64_t ldy)
{
    const Lane l = lane_of(words, K);
    if ((int64_t)l.tile * 16 >= M)
        return;
    const int64_t row = min(l.row, M - 1);
    uint32_t first[2] = {}, second[2] = {};
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        if (2 * j >= l.blocks)
            break;
        const uint8_t* src = codes + (((int64_t)l.word * 4 + 2 * j) * M + row) * 16 + 4 * l.q;
        first[j] = *reinterpret_cast<const uint32_t*>(src);
        second[j] = *reinterpret_cast<const uint32_t*>(src + M * 16);
    }
    const uint32_t mine = *reinterpret_cast<const uint32_t*>(scales + ((int64_t)l.word * M + row) * 4);
    const uint32_t theirs = mirrored(mine);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (l.row0 + 8 * i >= M)                   // all eight lanes of a row
            break;
        const uint32_t packed = ((i == 1) == l.odd ? mine : theirs) >> (l.odd ? 8 : 0);
        uint16_t* dst = y + (l.row0 + 8 * i) * ldy + (int64_t)l.word * 128 + (l.odd ? 32 : 0) + 8 * l.q;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint32_t got = mirrored(l.odd ? first[j] : second[j]);
            const uint32_t c = i == 0 ? (l.odd ? got : first[j]) : (l.odd ? second[j] : got);
            const uint32_t byte = (packed >> (16 * j)) & 255u;
            const float scale = __uint_as_float(byte << 23);
            v4u v;
            v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 0));
            v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 1));
            v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 2));
            v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 3));
            if (byte == 255u)
                v = v4u{0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u};
            if (2 * j < l.blocks)
                __builtin_nontemporal_store(v, reinterpret_cast<v4u*>(dst + 64 * j));
        }
    }
}

// Inputs past 80 MiB are hardly in the last-level cache any more, with what else was
// written since, and are read around it.  Around it and through it (us, three inputs
// in turn): 4608 x 8192 (72 MiB) 18.1, 16.6; 6144 x 8192 (96) 23.1, 24.2; 8192 x 8192
// 30.1, 31.2; 18432 x 4608 37.8, 39.7; 30000 x 8192 98, 112.
constexpr int64_t kPastElements = (int64_t)5 << 23;

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
    const auto kernel = M * K > kPastElements ? mxfp4_quantize_kernel<true> : mxfp4_quantize_kernel<false>;
    kernel<<<grid_of(M, words), 64 * kWaves, 0, stream>>>(x, M, (int32_t)K, ldx, words, codes, scales);
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
