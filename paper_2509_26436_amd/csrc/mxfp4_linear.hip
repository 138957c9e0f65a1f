// MXFP4 linear layer: y[m][n] = bf16(act(sum_k a[m,k] w[n,k] + bias[n])), both
// operands in MXFP4 (mxfp4.h), on the scaled fp4 matrix instructions, which
// multiply the 32-element blocks of a row and a column, scale each product by
// 2^(E_a + E_w) and add in fp32.  The weights are the instructions' rows and
// the tokens their columns, so that a lane holds outputs of one token, and the
// weight rows are given to the instructions in an order that makes a lane's
// outputs neighbours in n.
#include <algorithm>
#include <cmath>

#include "mxfp4.h"
#include "quartz_internal.h"

namespace quartz {
namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));

// Rows of outputs begin at any element (ldy is any number): wide stores all the
// same, which the memory takes at any address (3093 tokens, K = 768, 4775 columns,
// from bf16: 71.9 us with single elements, 27.6 so).
typedef uint32_t some_u2 __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t some_u4 __attribute__((ext_vector_type(4), aligned(2)));

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
// shared memory.  FUSED: the activations, at most kFusedElements of them,
// arrive in bf16; each block quantizes them all into shared memory while its
// first weights are on their way.
constexpr int kDirectWaves = 8, kDirectThreads = 64 * kDirectWaves;
constexpr int kFusedElements = 32768, kFusedRows = 8;

template <int CTRL>
__device__ __forceinline__ uint32_t quad(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, false);
}

// x [M][ldx] -> codes [K/32][M][16], scales [ceil(K/128)][M][4]; lane quads take a block each
__device__ __forceinline__ void quantize_to_lds(const MxLinear& a, uint8_t* codes, uint8_t* scales)
{
    constexpr int kBatch = 4;
    const uint32_t columns = (uint32_t)a.K / 8, count = (uint32_t)a.M * columns;
    for (uint32_t first = threadIdx.x; first < count; first += kBatch * kDirectThreads) {
        uint4 v[kBatch];
        uint32_t row[kBatch], column[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const uint32_t at = first + kDirectThreads * i;
            row[i] = at / columns;
            column[i] = at - row[i] * columns;
            if (at < count)
                v[i] = *reinterpret_cast<const uint4*>(a.x + row[i] * a.ldx + 8 * column[i]);
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            if (first + kDirectThreads * i >= count)       // whole quads: count is a multiple of 4
                break;
            uint32_t top = mx_max8(v[i]);
            top = max(top & 0xFFFFu, top >> 16);
            top = max(top, quad<0xB1>(top));               // quad_perm [1,0,3,2]
            top = max(top, quad<0x4E>(top));               // quad_perm [2,3,0,1]
            const uint32_t byte = mx_scale_byte(top), block = column[i] >> 2;
            *reinterpret_cast<uint32_t*>(codes + (block * (uint32_t)a.M + row[i]) * 16 + 4 * (column[i] & 3)) =
                mx_codes8(v[i], byte);
            if ((column[i] & 3) == 0)
                scales[((block >> 2) * (uint32_t)a.M + row[i]) * 4 + (block & 3)] = (uint8_t)byte;
        }
    }
}

template <int TM, int TN, bool FUSED>
__global__ __launch_bounds__(kDirectThreads) void mxfp4_direct_kernel(const MxLinear a)
{
    static_assert(!FUSED || TM == 1, "a fused block holds all tokens");
    __shared__ v4f part[kDirectWaves][TM * TN][64];
    __shared__ __attribute__((aligned(16))) uint8_t x_lds[FUSED ? kFusedElements / 2 : 16];
    // one more word: K % 128 == 64 leaves half of a row's last word unused
    __shared__ __attribute__((aligned(16))) uint8_t x_lds_scales[FUSED ? kFusedElements / 32 + 4 * kFusedRows : 16];
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t n0 = (int64_t)blockIdx.x * (16 * TN), m0 = (int64_t)blockIdx.y * (16 * TM);
    const int blocks = (int)(a.K >> 5), steps = (int)((a.K + 127) >> 7);
    // steps of a wave whose loads are issued together
        constexpr int kAhead = TM * TN >= 4 ? 2 : 4;

    v4f acc[TN][TM] = {};
    int64_t wrow[TN], xrow[TM];
#pragma unroll
    for (int t = 0; t < TN; ++t)
        wrow[t] = min(n0 + 4 * TN * (r >> 2) + 4 * t + (r & 3), a.N - 1);
#pragma unroll
    for (int t = 0; t < TM; ++t)
        xrow[t] = min(m0 + 16 * t + r, a.M - 1);

    v4i wf[kAhead][TN], xf[kAhead][TM];
    uint32_t ws[kAhead][TN], xs[kAhead][TM];
    auto load = [&](int first) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int c = first + kDirectWaves * i, block = min(4 * c + g, blocks - 1);
            if (c >= steps)
                break;
#pragma unroll
            for (int t = 0; t < TN; ++t) {
                wf[i][t] = *reinterpret_cast<const v4i*>(a.w_codes + ((int64_t)block * a.N + wrow[t]) * 16);
                ws[i][t] = *reinterpret_cast<const uint32_t*>(a.w_scales + ((int64_t)c * a.N + wrow[t]) * 4);
            }
            if constexpr (!FUSED) {
#pragma unroll
                for (int t = 0; t < TM; ++t) {
                    xf[i][t] = *reinterpret_cast<const v4i*>(a.x_codes + ((int64_t)block * a.M + xrow[t]) * 16);
                    xs[i][t] = *reinterpret_cast<const uint32_t*>(a.x_scales + ((int64_t)c * a.M + xrow[t]) * 4);
                }
            }
        }
    };
    load(wave);
    if constexpr (FUSED) {
        quantize_to_lds(a, x_lds, x_lds_scales);
        __syncthreads();
    }
    for (int first = wave; first < steps; first += kDirectWaves * kAhead) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int c = first + kDirectWaves * i;
            if (c >= steps)
                break;
            const bool have = 4 * c + g < blocks;          // the last step may hold two blocks
            if constexpr (FUSED) {
                const uint32_t row = (uint32_t)xrow[0];
                xf[i][0] = *reinterpret_cast<const v4i*>(x_lds + (min(4 * c + g, blocks - 1) * (uint32_t)a.M + row) * 16);
                xs[i][0] = *reinterpret_cast<const uint32_t*>(x_lds_scales + (c * (uint32_t)a.M + row) * 4);
            }
#pragma unroll
            for (int t = 0; t < TN; ++t)
                ws[i][t] = have ? ws[i][t] >> (8 * g) : 0u;
#pragma unroll
            for (int t = 0; t < TM; ++t) {
                xs[i][t] = have ? xs[i][t] >> (8 * g) : 0u;
                xf[i][t] = have ? xf[i][t] : v4i{0, 0, 0, 0};
            }
#pragma unroll
            for (int t = 0; t < TN; ++t)
#pragma unroll
                for (int u = 0; u < TM; ++u)
                    acc[t][u] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                        wide(wf[i][t]), wide(xf[i][u]), acc[t][u], 4, 4, 0, (int)ws[i][t], 0, (int)xs[i][u]);
        }
        if (first + kDirectWaves * kAhead < steps)
            load(first + kDirectWaves * kAhead);
    }

    // wave w finishes tiles w, w + 8, ...: their bias is on its way while the sums meet
    constexpr int kMine = (TN * TM + kDirectWaves - 1) / kDirectWaves;
    v4f bias[kMine] = {};
    if (a.bias) {
#pragma unroll
        for (int j = 0; j < kMine; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                bias[j][i] = bf16_value(
                    a.bias[min(n0 + 4 * TN * g + 4 * ((wave + kDirectWaves * j) / TM) + i, a.N - 1)]);
    }
#pragma unroll
    for (int t = 0; t < TN; ++t)
#pragma unroll
        for (int u = 0; u < TM; ++u)
            part[wave][t * TM + u][lane] = acc[t][u];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kMine; ++j) {
        const int tile = wave + kDirectWaves * j;
        if (tile >= TN * TM)
            break;
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
            s[i] += bias[j][i];
            if (a.gelu)
                s[i] = gelu_tanh(s[i]);
        }
        const uint2 out = {pack_bf16(s[0], s[1]), pack_bf16(s[2], s[3])};
        if (count == 4) {
            *reinterpret_cast<some_u2*>(dst) = some_u2{out.x, out.y};
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
// A block owns 64 TM tokens x 64 TN columns; four waves, 2 x 2, one on each
// SIMD, of 32 TM x 32 TN each: TM TN accumulators of 32 x 32.  K goes by in
// stages of 128, two steps of one matrix instruction each, through a ring of
// four stages in shared memory, which loads reach without passing registers.
// While a step's TM TN products run, the next step's fragments come from shared
// memory into the other half of the fragment registers.  Before the second
// step of a stage, whose fragments are in registers already, one barrier says
// that the next stage has arrived and that this one may be overwritten: its
// place is loaded again at once, three stages ahead of its use.
constexpr int kStageBlocks = 4;
constexpr int kRing = 4;

// a pointer that is the same in all lanes, kept in scalar registers
__device__ __forceinline__ const uint8_t* uniform(const uint8_t* p)
{
    const uint64_t v = reinterpret_cast<uint64_t>(p);
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
    return reinterpret_cast<const uint8_t*>((uint64_t)hi << 32 | lo);
}

// 16 (4) bytes a lane from base + offset to shared memory, lane after lane
template <int BYTES>
__device__ __forceinline__ void to_lds(const uint8_t* base, uint32_t offset, uint8_t* lds)
{
    // keeps the 32-bit offset in the loop (hoisted, it would be widened and every load take a 64-bit add)
    asm volatile("" : "+v"(offset));
    const auto* from = (const __attribute__((address_space(1))) void*)(base + offset);
    auto* to = (__attribute__((address_space(3))) void*)lds;
    if constexpr (BYTES == 16)
        __builtin_amdgcn_global_load_lds(from, to, 16, 0, 0);
    else
        __builtin_amdgcn_global_load_lds(from, to, 4, 0, 0);
}

template <int TM, int TN>
__global__ __launch_bounds__(256) void mxfp4_tiled_kernel(const MxLinear a, uint32_t tiles_m, uint32_t tiles_n)
{
    constexpr int kM = 64 * TM, kN = 64 * TN, kRows = kM + kN;
    constexpr int kCodes = kStageBlocks * kRows * 16;
    // a stage: codes [4][weights, tokens][16], scales [weights, tokens][4]
    __shared__ __attribute__((aligned(16))) uint8_t lds[kRing][kCodes + kRows * 4];
    const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

    // Consecutive blocks go to the eight XCDs in turn: each XCD takes a
    // consecutive run of tiles, and a run walks bands of 4 token tiles, so that
    // the 32 tiles at work on an XCD share 4 + 8 operand tiles in its L2.
    const uint32_t tiles = tiles_m * tiles_n, xcd = blockIdx.x & 7, each = tiles >> 3, more = tiles & 7;
    const uint32_t at = xcd * each + min(xcd, more) + (blockIdx.x >> 3);
    const uint32_t band = at / (4 * tiles_n), in_band = at - band * 4 * tiles_n;
    const uint32_t high = min(4u, tiles_m - 4 * band);
    const uint32_t tile_n = in_band / high, tile_m = 4 * band + (in_band - tile_n * high);
    const int64_t n0 = (int64_t)tile_n * kN, m0 = (int64_t)tile_m * kM;
    const int blocks = (int)(a.K >> 5), stages = (blocks + kStageBlocks - 1) / kStageBlocks;

    // Shared memory holds weight rows in the order of the instruction's rows:
    // row 8 q + 4 h + i of 32 is n = 16 h + 4 q + i, so that a lane's 16 outputs
    // are n = 16 h .. 16 h + 15.  Rows past the end are read from the last one,
    // blocks past K from the last one too (no step multiplies them).
    const int order = (lane & 32) + 16 * ((lane >> 2) & 1) + 4 * ((lane >> 3) & 3) + (lane & 3);
    const int last_w = (int)min((int64_t)kN, a.N - n0) - 1, last_x = (int)min((int64_t)kM, a.M - m0) - 1;
    uint32_t wrow[TN], xrow[TM];
#pragma unroll
    for (int t = 0; t < TN; ++t)
        wrow[t] = (uint32_t)min(64 * t + order, last_w);
#pragma unroll
    for (int u = 0; u < TM; ++u)
        xrow[u] = (uint32_t)min(64 * u + lane, last_x);

    // Wave w loads block w of a stage, and every fourth run of 64 rows of its scales, from run w on.
    constexpr int kRuns = (TN + TM + 3) / 4, kLoads = TN + TM + kRuns;
    const uint8_t* run_from[kRuns];
    int64_t run_step[kRuns];
    uint32_t run_row[kRuns], run_to[kRuns];
#pragma unroll
    for (int i = 0; i < kRuns; ++i) {
        const int run = min(4 * i + wave, TN + TM - 1);
        const bool weights = run < TN;
        run_from[i] = weights ? a.w_scales + n0 * 4 : a.x_scales + m0 * 4;
        run_step[i] = (weights ? a.N : a.M) * 4;
        run_row[i] = (uint32_t)min(64 * (weights ? run : run - TN) + (weights ? order : lane), weights ? last_w : last_x);
        run_to[i] = (uint32_t)(64 * run) * 4;
    }
    // load i of a stage: the weight runs of the wave's block, the token runs, the runs of scales
    auto load_item = [&](int stage, int i) {
        uint8_t* base = lds[stage & (kRing - 1)];
        const int block = min(stage * kStageBlocks + wave, blocks - 1);
        if (i < TN)
            to_lds<16>(uniform(a.w_codes + ((int64_t)block * a.N + n0) * 16), wrow[i] * 16,
                       base + (wave * kRows + 64 * i) * 16);
        else if (i < TN + TM)
            to_lds<16>(uniform(a.x_codes + ((int64_t)block * a.M + m0) * 16), xrow[i - TN] * 16,
                       base + (wave * kRows + 64 * i) * 16);
        else
            to_lds<4>(uniform(run_from[i - TN - TM] + stage * run_step[i - TN - TM]), run_row[i - TN - TM] * 4,
                      base + kCodes + run_to[i - TN - TM]);
    };
    auto load = [&](int stage) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            load_item(stage, i);
    };
    using Zero = std::integral_constant<int, 0>;
    using One = std::integral_constant<int, 1>;
    // All but the `flying` newest loads of this wave have landed and its reads
    // are done, and so for the others.
    auto meet = [](auto flying) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(decltype(flying)::value) : "memory");
    };

    const int wn = (wave & 1) * 32 * TN, wm = kN + (wave >> 1) * 32 * TM;
    v16f acc[TN][TM] = {};
    v4i wf[2][TN], xf[2][TM];
    uint32_t ws[TN], xs[TM], ws_next[TN], xs_next[TM];
    // read i of a step's fragments, the instructions' rows before their columns; i past them: a stage's scale words
    constexpr int kReads = TN + TM;
    auto read_item = [&](int stage, auto step, int i) {
        constexpr int k = decltype(step)::value;
        const uint8_t* c = lds[stage & (kRing - 1)] + ((2 * k + h) * kRows + r) * 16;
        const uint8_t* sc = lds[stage & (kRing - 1)] + kCodes + r * 4;
        if (i < TN)
            wf[k][i] = *reinterpret_cast<const v4i*>(c + (wn + 32 * i) * 16);
        else if (i < kReads)
            xf[k][i - TN] = *reinterpret_cast<const v4i*>(c + (wm + 32 * (i - TN)) * 16);
        else if (i < kReads + TN)
            ws_next[i - kReads] = *reinterpret_cast<const uint32_t*>(sc + (wn + 32 * (i - kReads)) * 4);
        else if (i < 2 * kReads)
            xs_next[i - kReads - TN] = *reinterpret_cast<const uint32_t*>(sc + (wm + 32 * (i - kReads - TN)) * 4);
    };
    // step k multiplies blocks 2 k + h of the stage: bytes 0 and 2 of a word that
    // a lane of the upper half has shifted by one
    auto take_scales = [&] {
#pragma unroll
        for (int t = 0; t < TN; ++t)
            ws[t] = ws_next[t] >> (8 * h);
#pragma unroll
        for (int u = 0; u < TM; ++u)
            xs[u] = xs_next[u] >> (8 * h);
    };
    auto multiply = [&](auto step, int t, int u) {
        constexpr int k = decltype(step)::value;
        acc[t][u] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
            wide(wf[k][t]), wide(xf[k][u]), acc[t][u], 4, 4, 2 * k, (int)ws[t], 2 * k, (int)xs[u]);
    };
    // A stage that is not the last; at its barrier the next stage has to have
    // arrived, with the loads of the two after it on their way, or (near the
    // end, where no more are issued) all of them.  The order of products, reads
    // and loads is the one written: left to itself the compiler puts the loads
    // in one place, and the matrix unit waits there.
    auto whole = [&](int stage, auto flying) {
#pragma unroll
        for (int i = 0; i < TN * TM; ++i) {
            multiply(Zero(), i / TM, i % TM);
            read_item(stage, One(), 2 * i < kReads ? 2 * i : 2 * kReads);
            read_item(stage, One(), 2 * i + 1 < kReads ? 2 * i + 1 : 2 * kReads);
            __builtin_amdgcn_sched_barrier(0);
        }
        meet(flying);
#pragma unroll
        for (int i = 0; i < TN * TM; ++i) {
            multiply(One(), i / TM, i % TM);
            read_item(stage + 1, Zero(), 2 * i);
            read_item(stage + 1, Zero(), 2 * i + 1);
            if constexpr (decltype(flying)::value > 0) {
#pragma unroll
                for (int j = i * kLoads / (TN * TM); j < (i + 1) * kLoads / (TN * TM); ++j)
                    load_item(stage + kRing, j);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        take_scales();
    };
    auto last_step = [&](auto step) {
#pragma unroll
        for (int i = 0; i < TN * TM; ++i)
            multiply(step, i / TM, i % TM);
    };

    for (int stage = 0; stage < min(stages, kRing); ++stage)
        load(stage);
    if (stages >= kRing)
        meet(std::integral_constant<int, (kRing - 1) * kLoads>());
    else
        meet(Zero());
#pragma unroll
    for (int i = 0; i < 2 * kReads; ++i)
        read_item(0, Zero(), i);
    take_scales();
    int stage = 0;
    for (; stage < stages - kRing; ++stage)
        whole(stage, std::integral_constant<int, (kRing - 2) * kLoads>());
    for (; stage < stages - 1; ++stage)
        whole(stage, Zero());
    last_step(Zero());
    if (2 * stage + 1 < blocks / 2) {              // the last stage may be one step
#pragma unroll
        for (int i = 0; i < kReads; ++i)
            read_item(stage, One(), i);
        last_step(One());
    }

    // the bias of this lane's columns, all of it on its way at once
    v4i bias[TN][2];
#pragma unroll
    for (int t = 0; t < TN; ++t)
        bias[t][0] = bias[t][1] = v4i{0, 0, 0, 0};
    if (a.bias && a.N - n0 >= kN) {
#pragma unroll
        for (int t = 0; t < TN; ++t)
#pragma unroll
            for (int i = 0; i < 2; ++i)
                bias[t][i] = *reinterpret_cast<const v4i*>(a.bias + n0 + wn + 32 * t + 16 * h + 8 * i);
    } else if (a.bias) {
#pragma unroll
        for (int t = 0; t < TN; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int64_t n = min(n0 + wn + 32 * t + 16 * h + i, a.N - 1);
                bias[t][i / 8][i % 8 / 2] |= (int)((uint32_t)a.bias[n] << (16 * (i & 1)));
            }
    }
#pragma unroll
    for (int t = 0; t < TN; ++t) {
        const int64_t n = n0 + wn + 32 * t + 16 * h;
        const int count = (int)max((int64_t)0, min((int64_t)16, a.N - n));
#pragma unroll
        for (int u = 0; u < TM; ++u) {
            const int64_t m = m0 + wm - kN + 32 * u + r;
            float v[16];
#pragma unroll
            for (int i = 0; i < 16; ++i)
                v[i] = acc[t][u][i] + bf16_value((uint16_t)((uint32_t)bias[t][i / 8][i % 8 / 2] >> (16 * (i & 1))));
            if (a.gelu) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    v[i] = gelu_tanh(v[i]);
            }
            if (m >= a.M || count == 0)
                continue;
            uint32_t out[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                out[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
            uint16_t* dst = a.y + m * a.ldy + n;
            if (count == 16) {
                reinterpret_cast<some_u4*>(dst)[0] = some_u4{out[0], out[1], out[2], out[3]};
                reinterpret_cast<some_u4*>(dst)[1] = some_u4{out[4], out[5], out[6], out[7]};
            } else {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (i < count)
                        dst[i] = (uint16_t)(out[i / 2] >> (16 * (i & 1)));
            }
        }
    }
}

template <int TM, int TN>
hipError_t launch_tiled(const MxLinear& a, hipStream_t stream)
{
    const uint32_t tm = (uint32_t)((a.M + 64 * TM - 1) / (64 * TM)), tn = (uint32_t)((a.N + 64 * TN - 1) / (64 * TN));
    mxfp4_tiled_kernel<TM, TN><<<tm * tn, 256, 0, stream>>>(a, tm, tn);
    return hipGetLastError();
}

}  // namespace

bool mxfp4_fuses(int64_t M, int64_t K) { return M <= kFusedRows && M * K <= kFusedElements; }

// The kernel with the least expected time, from fits (microseconds, 256 compute
// units, kk = K / 1024) of measured ones.  A direct block's cost is its reads
// and the meeting of its waves' sums; a tiled one's is a fixed part (filling
// the ring, storing the tile) and its products, in rounds of one block a
// compute unit (tiles of 128 x 128: two, which halves the steps' latency but
// not their work).  Measured at 4096 columns and K = 4096: 64 tokens 4.0 us in
// direct blocks of 32 x 32, 6.8 in those of 64 x 64 and 12.2 tiled; 256 tokens
// 8.7, 7.3 and 12.5; 1024 tokens 27.9, 25.3 and 14.9 (tiles of 128 x 128, 28.1
// with 256 x 256); 4096 tokens 43 with 128 x 128 and 37 with 256 x 256.  Tiles
// of 192 serve what they fill whole rounds of: 4608 x 8192 x 8192 takes 151 us
// with 192 x 256 (three rounds) and 168 with 256 x 256 (two and a quarter).
// Where K is short, two blocks a compute unit hide each other's stores: 18432 x
// 4608 at K = 1152 takes 89 us in tiles of 128 x 128 (97 with bias and GELU) and
// 90 (107) in those of 192 x 256, at K = 4608 239 and 220.
MxShape mxfp4_shape(int64_t M, int64_t N, int64_t K)
{
    if (M <= 16)
        return {false, 1, 1};
    const double kk = (double)K / 1024;
    auto blocks = [&](int64_t rows, int64_t columns) {
        return (double)((M + rows - 1) / rows) * (double)((N + columns - 1) / columns);
    };
    const double small = std::max(blocks(32, 32), 256.0), medium = std::max(blocks(64, 64), 256.0);
    // (a direct grid has at most 65535 blocks of tokens)
    const bool direct = M <= 65535 * 32;
    MxShape best{!direct, 2, 2};
    double least = direct ? 2.5 + 0.1 * kk + small * (1.4 + 1.25 * kk) / 1000 : INFINITY;
    auto consider = [&](const MxShape& s, double time) {
        if (time < least) {
            best = s;
            least = time;
        }
    };
    if (direct)
        consider({false, 4, 4}, 2.5 + 0.15 * kk + medium * (8.6 + 3.15 * kk) / 1000);
    const double each = blocks(128, 128), x = each <= 512 ? each / 256 : 2 * std::ceil(each / 512);
    consider({true, 2, 2}, 3.5 + 1.4 * x + kk * std::max(2.1, 2.05 * x));
    for (const MxShape& s : {MxShape{true, 3, 4}, MxShape{true, 4, 3}, MxShape{true, 4, 4}})
        consider(s, 2 + std::ceil(blocks(64 * s.tm, 64 * s.tn) / 256) *
                            (0.5 * s.tm * s.tn + kk * (s.tm * s.tn == 16 ? 6.6 : 5.7)));
    return best;
}

hipError_t launch_mxfp4_linear(const MxLinear& a, hipStream_t stream)
{
    if (a.x)
        return launch_direct<1, 1, true>(a, stream);
    const MxShape s = mxfp4_shape(a.M, a.N, a.K);
    if (!s.tiled)
        return s.tm == 1   ? launch_direct<1, 1, false>(a, stream)
               : s.tm == 2 ? launch_direct<2, 2, false>(a, stream)
                           : launch_direct<4, 4, false>(a, stream);
    if (s.tm == 2)
        return launch_tiled<2, 2>(a, stream);
    if (s.tm == 3)
        return launch_tiled<3, 4>(a, stream);
    return s.tn == 3 ? launch_tiled<4, 3>(a, stream) : launch_tiled<4, 4>(a, stream);
}

}  // namespace quartz
