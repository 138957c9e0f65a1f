// MXFP4 linear layer: y[m][n] = bf16(act(sum_k a[m,k] w[n,k] + bias[n])), both
// operands in MXFP4 (mxfp4.h), on the scaled fp4 matrix instructions, which
// multiply the 32-element blocks of a row and a column, scale each product by
// 2^(E_a + E_w) and add in fp32.  The weights are the instructions' rows and
// the tokens their columns, so that a lane holds outputs of one token, and the
// weight rows are given to the instructions in an order that makes a lane's
// outputs neighbours in n.
#include "mxfp4.h"
#include "quartz_internal.h"

namespace quartz {
namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));

// the matrix instructions' fp4 operand is the low half of their register range
__device__ __forceinline__ v8i wide(v4i a)
{
    return __builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1);
}

__device__ __forceinline__ float gelu_tanh(float v)
{
    // 0.5 v (1 + tanh(u)) = v / (1 + exp(-2 u)), u = sqrt(2/pi) (v + 0.044715 v^3)
    constexpr float c0 = -2.0f * 1.4426950408889634f * 0.7978845608028654f;
    constexpr float c1 = c0 * 0.044715f;
    const float w = __builtin_fmaf(c1, v * v, c0);
    return v * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(w * v));
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    typedef float f2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{a, b}, mx_bf2));
}

__device__ __forceinline__ float bf16_value(uint16_t b)
{
    return __uint_as_float((uint32_t)b << 16);
}

// ------------------------------------------------------------ few tokens, small layers
//
// A block owns 16 TN columns x 16 TM tokens of the output.  Its eight waves
// take the 128-element steps of K in turn, each accumulating the whole tile
// from fragments read straight from memory (a fragment is read once in the
// block, so shared memory would only add a copy), and their sums meet in
// shared memory.  FUSED: the activations arrive in bf16 and each wave
// quantizes the fragment it needs, a block being the 32 consecutive elements
// that a lane holds anyway.
constexpr int kDirectWaves = 8;

template <int TM, int TN, bool FUSED>
__global__ __launch_bounds__(64 * kDirectWaves) void mxfp4_direct_kernel(const MxLinear a)
{
    __shared__ v4f part[kDirectWaves][TM * TN][64];
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t n0 = (int64_t)blockIdx.x * (16 * TN), m0 = (int64_t)blockIdx.y * (16 * TM);
    const int blocks = (int)(a.K >> 5), steps = (int)((a.K + 127) >> 7);

    v4f acc[TN][TM] = {};
    int64_t wrow[TN], xrow[TM];
#pragma unroll
    for (int t = 0; t < TN; ++t)
        wrow[t] = min(n0 + 4 * TN * (r >> 2) + 4 * t + (r & 3), a.N - 1);
#pragma unroll
    for (int t = 0; t < TM; ++t)
        xrow[t] = min(m0 + 16 * t + r, a.M - 1);

    for (int c = wave; c < steps; c += kDirectWaves) {
        const int block = 4 * c + g;
        const bool have = block < blocks;         // the last step may hold two blocks
        v4i wf[TN], xf[TM];
        uint32_t ws[TN], xs[TM];
#pragma unroll
        for (int t = 0; t < TN; ++t) {
            wf[t] = have ? *reinterpret_cast<const v4i*>(a.w_codes + ((int64_t)block * a.N + wrow[t]) * 16)
                         : v4i{0, 0, 0, 0};
            ws[t] = *reinterpret_cast<const uint32_t*>(a.w_scales + ((int64_t)c * a.N + wrow[t]) * 4) >> (8 * g);
            ws[t] = have ? ws[t] : 0u;
        }
#pragma unroll
        for (int t = 0; t < TM; ++t) {
            if constexpr (FUSED) {
                uint4 v[4] = {};
                if (have) {
                    const uint4* src = reinterpret_cast<const uint4*>(a.x + xrow[t] * a.ldx + block * 32);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        v[j] = src[j];
                }
                uint32_t top = mx_max2(mx_max2(mx_max8(v[0]), mx_max8(v[1])),
                                       mx_max2(mx_max8(v[2]), mx_max8(v[3])));
                xs[t] = mx_scale_byte(max(top & 0xFFFFu, top >> 16));
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    xf[t][j] = (int)mx_codes8(v[j], xs[t]);
            } else {
                xf[t] = have ? *reinterpret_cast<const v4i*>(a.x_codes + ((int64_t)block * a.M + xrow[t]) * 16)
                             : v4i{0, 0, 0, 0};
                xs[t] = *reinterpret_cast<const uint32_t*>(a.x_scales + ((int64_t)c * a.M + xrow[t]) * 4) >> (8 * g);
                xs[t] = have ? xs[t] : 0u;
            }
        }
#pragma unroll
        for (int t = 0; t < TN; ++t)
#pragma unroll
            for (int u = 0; u < TM; ++u)
                acc[t][u] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                    wide(wf[t]), wide(xf[u]), acc[t][u], 4, 4, 0, (int)ws[t], 0, (int)xs[u]);
    }

#pragma unroll
    for (int t = 0; t < TN; ++t)
#pragma unroll
        for (int u = 0; u < TM; ++u)
            part[wave][t * TM + u][lane] = acc[t][u];
    __syncthreads();
    for (int tile = wave; tile < TN * TM; tile += kDirectWaves) {
        v4f s = part[0][tile][lane];
#pragma unroll
        for (int w = 1; w < kDirectWaves; ++w)
            s += part[w][tile][lane];
        const int t = tile / TM, u = tile % TM;
        const int64_t n = n0 + 4 * TN * g + 4 * t, m = m0 + 16 * u + r;
        if (m >= a.M || n >= a.N)
            continue;
        uint16_t* dst = a.y + m * a.ldy + n;
        const int count = (int)min((int64_t)4, a.N - n);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (a.bias && i < count)
                s[i] += bf16_value(a.bias[n + i]);
            if (a.gelu)
                s[i] = gelu_tanh(s[i]);
        }
        const uint2 out = {pack_bf16(s[0], s[1]), pack_bf16(s[2], s[3])};
        if (count == 4 && (a.ldy & 3) == 0) {
            *reinterpret_cast<uint2*>(dst) = out;
        } else {
            for (int i = 0; i < count; ++i)
                dst[i] = (uint16_t)((i & 2 ? out.y : out.x) >> (16 * (i & 1)));
        }
    }
}

template <int TM, int TN, bool FUSED>
hipError_t launch_direct(const MxLinear& a, hipStream_t stream)
{
    const dim3 grid((uint32_t)((a.N + 16 * TN - 1) / (16 * TN)), (uint32_t)((a.M + 16 * TM - 1) / (16 * TM)));
    mxfp4_direct_kernel<TM, TN, FUSED><<<grid, 64 * kDirectWaves, 0, stream>>>(a);
    return hipGetLastError();
}

// ------------------------------------------------------------ large layers
//
// A block owns 256 tokens x 256 columns; eight waves, 4 (tokens) x 2 (columns),
// of 64 x 128 each: eight tiles of 32 x 32, 128 accumulator registers.  K goes
// by in steps of 256: while the waves work on one step in shared memory the
// next one's codes and scales are on their way there without passing
// registers, one barrier a step.
constexpr int kTile = 256;
constexpr int kStepBlocks = 8;                              // 256 elements of K
constexpr int kStageCodes = kStepBlocks * kTile * 16;       // bytes of one operand
constexpr int kStageScales = kStepBlocks / 4 * kTile * 4;
constexpr int kStage = 2 * (kStageCodes + kStageScales);

__device__ __forceinline__ void to_lds(const void* src, void* lds, std::integral_constant<int, 16>)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                     (__attribute__((address_space(3))) void*)lds, 16, 0, 0);
}
__device__ __forceinline__ void to_lds(const void* src, void* lds, std::integral_constant<int, 4>)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                     (__attribute__((address_space(3))) void*)lds, 4, 0, 0);
}

__global__ __launch_bounds__(512) void mxfp4_tiled_kernel(const MxLinear a, uint32_t tiles_m, uint32_t tiles_n)
{
    __shared__ __attribute__((aligned(16))) uint8_t lds[2 * kStage];
    const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t tile_n = blockIdx.x / tiles_m, tile_m = blockIdx.x - tile_n * tiles_m;
    const int64_t n0 = (int64_t)tile_n * kTile, m0 = (int64_t)tile_m * kTile;
    const int blocks = (int)(a.K >> 5), stages = (blocks + kStepBlocks - 1) / kStepBlocks;

    // shared memory holds a tile's rows in the order of the instructions' rows:
    // row 8 q + 4 h + i of 32 weight rows is n = 16 h + 4 q + i, so that a lane's
    // 16 outputs are n = 16 h .. 16 h + 15.  Wave w carries rows 64 (w % 4) .. + 63
    // of the weights (w < 4) or of the tokens.
    const bool weights = wave < 4;
    const int slot = (wave & 3) * 64 + lane;
    const int order = weights ? (slot & ~31) + 16 * ((slot >> 2) & 1) + 4 * ((slot >> 3) & 3) + (slot & 3) : slot;
    const int64_t rows = weights ? a.N : a.M;
    const int64_t row = min((weights ? n0 : m0) + order, rows - 1);
    const uint8_t* codes = (weights ? a.w_codes : a.x_codes) + row * 16;
    const uint8_t* scales = (weights ? a.w_scales : a.x_scales) + row * 4;
    const int at_codes = weights ? 0 : kStageCodes;
    const int at_scales = 2 * kStageCodes + (weights ? 0 : kStageScales);

    auto load = [&](int stage) {
        uint8_t* base = lds + (stage & 1) * kStage;
#pragma unroll
        for (int j = 0; j < kStepBlocks; ++j) {
            const int block = stage * kStepBlocks + j;
            if (block < blocks)
                to_lds(codes + (int64_t)block * rows * 16,
                       base + at_codes + (j * kTile + (wave & 3) * 64) * 16, std::integral_constant<int, 16>());
        }
#pragma unroll
        for (int j = 0; j < kStepBlocks / 4; ++j) {
            const int word = stage * (kStepBlocks / 4) + j;
            if (4 * word < blocks)
                to_lds(scales + (int64_t)word * rows * 4,
                       base + at_scales + (j * kTile + (wave & 3) * 64) * 4, std::integral_constant<int, 4>());
        }
    };

    const int wn = (wave & 1) * 128, wm = (wave >> 1) * 64;
    v16f acc[4][2] = {};
    load(0);
    for (int stage = 0; stage < stages; ++stage) {
        // this stage has arrived, and nobody reads the other one any more
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (stage + 1 < stages)
            load(stage + 1);
        const uint8_t* base = lds + (stage & 1) * kStage;
        const int pairs = min(kStepBlocks, blocks - stage * kStepBlocks) / 2;
        uint32_t ws[4], xs[2];
        auto product = [&](int s, auto odd) {
            constexpr int kOdd = decltype(odd)::value;
            v4i wf[4], xf[2];
            const uint8_t* c = base + (2 * s + h) * (kTile * 16) + r * 16;
#pragma unroll
            for (int t = 0; t < 4; ++t)
                wf[t] = *reinterpret_cast<const v4i*>(c + (wn + 32 * t) * 16);
#pragma unroll
            for (int u = 0; u < 2; ++u)
                xf[u] = *reinterpret_cast<const v4i*>(c + kStageCodes + (wm + 32 * u) * 16);
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    acc[t][u] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
                        wide(wf[t]), wide(xf[u]), acc[t][u], 4, 4, 2 * kOdd, (int)ws[t], 2 * kOdd, (int)xs[u]);
        };
#pragma unroll
        for (int word = 0; word < kStepBlocks / 4; ++word) {
            if (2 * word >= pairs)
                break;
            const uint8_t* sc = base + 2 * kStageCodes + (word * kTile + r) * 4;
            // blocks 2 s + h of a word: a lane of the upper half takes the odd bytes
#pragma unroll
            for (int t = 0; t < 4; ++t)
                ws[t] = *reinterpret_cast<const uint32_t*>(sc + (wn + 32 * t) * 4) >> (8 * h);
#pragma unroll
            for (int u = 0; u < 2; ++u)
                xs[u] = *reinterpret_cast<const uint32_t*>(sc + kStageScales + (wm + 32 * u) * 4) >> (8 * h);
            product(2 * word, std::integral_constant<int, 0>());
            if (2 * word + 1 < pairs)
                product(2 * word + 1, std::integral_constant<int, 1>());
        }
    }

#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const int64_t n = n0 + wn + 32 * t + 16 * h;
        const int count = (int)max((int64_t)0, min((int64_t)16, a.N - n));
        float bias[16];
#pragma unroll
        for (int i = 0; i < 16; ++i)
            bias[i] = a.bias && i < count ? bf16_value(a.bias[n + i]) : 0.0f;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int64_t m = m0 + wm + 32 * u + r;
            if (m >= a.M || count == 0)
                continue;
            uint32_t out[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float lo = acc[t][u][2 * i] + bias[2 * i], hi = acc[t][u][2 * i + 1] + bias[2 * i + 1];
                if (a.gelu) {
                    lo = gelu_tanh(lo);
                    hi = gelu_tanh(hi);
                }
                out[i] = pack_bf16(lo, hi);
            }
            uint16_t* dst = a.y + m * a.ldy + n;
            if (count == 16 && (a.ldy & 7) == 0) {
                reinterpret_cast<uint4*>(dst)[0] = uint4{out[0], out[1], out[2], out[3]};
                reinterpret_cast<uint4*>(dst)[1] = uint4{out[4], out[5], out[6], out[7]};
            } else {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (i < count)
                        dst[i] = (uint16_t)(out[i / 2] >> (16 * (i & 1)));
            }
        }
    }
}

hipError_t launch_tiled(const MxLinear& a, hipStream_t stream)
{
    const uint32_t tm = (uint32_t)((a.M + kTile - 1) / kTile), tn = (uint32_t)((a.N + kTile - 1) / kTile);
    mxfp4_tiled_kernel<<<tm * tn, 512, 0, stream>>>(a, tm, tn);
    return hipGetLastError();
}

}  // namespace

bool mxfp4_fuses(int64_t M) { return M <= 16; }

hipError_t launch_mxfp4_linear(const MxLinear& a, hipStream_t stream)
{
    if (a.x)
        return launch_direct<1, 1, true>(a, stream);
    const int64_t tiles = ((a.M + kTile - 1) / kTile) * ((a.N + kTile - 1) / kTile);
    if (tiles < 64)
        return a.M <= 16 ? launch_direct<1, 1, false>(a, stream) : launch_direct<4, 4, false>(a, stream);
    return launch_tiled(a, stream);
}

}  // namespace quartz
