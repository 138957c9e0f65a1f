// Attention of one new token a sequence over the pages of its cache:
//   o[b][h] = sum_j p_j v_j,  p = softmax_j(scale q[b][h] . k_j),
// j over the sequence's keys (the last `window` of them if that is set); a
// sequence without keys gives zeros.  Bound by the memory that holds the keys
// and values: each is read once and used by the `group` query heads that share
// it, up to 16 of them as the columns of one matrix tile.
//
// No key or value passes through shared memory, because the matrix
// instructions' rows may be any keys and channels:
//   S^T = K Q^T: row 4 a + i of tile t is key 8 a + 4 t + i, so that the scores
//     a lane gets (one query, rows 4 g .. 4 g + 3 of two tiles) are keys 8 g ..
//     8 g + 7: exactly the 8 keys of its share of P^T in the next product;
//   O^T = V^T P^T: lane (m, g) reads a run of channels of keys 8 g .. 8 g + 7,
//     whole rows of V over the 16 lanes m, and turns the block of 8 keys x run in
//     registers; row m of tile t is channel t of lane m's run, so that at the end
//     a lane holds neighbouring channels of its query.
// The softmax runs over the pass with a running maximum and sum in fp32 (base-2
// exponentials).  P goes into the product as two bf16 parts, its rounding and the
// rest of it (a relative error of up to 2^-16 a weight, where one part would leave
// 2^-8), and the sum is that of the same parts (a row of ones beside V), so that
// weights add up to one.  The memory still bounds the call: 512 heads of 129 to
// 4096 e4m3 keys take 51.6 us with both parts and 51.1 with one.
// e4m3 keys and values are expanded to bf16, exactly, after the load; their
// scales go into the softmax scale and the output.
//
// The work of a call is a list of units, 128 keys of one (sequence, cache head,
// 16 queries) each, sequence after sequence, that the blocks share in equal
// runs: a block passes over its units with four waves of 32 keys, the next 32
// on their way while it computes, and whenever it leaves a sequence's head its
// waves' sums meet in shared memory.  A head that lies within one block's run is
// finished there; of the others each block leaves (maximum, sum, O) in the
// workspace, at most two such parts a block, and a second kernel joins them.
// Where the table is narrow a block takes a head, with as many waves as have keys
// to read, and there is no second kernel.
#include <algorithm>
#include <cfloat>

#include "quartz_internal.h"

namespace quartz {
namespace {

typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

constexpr int kKeys = 32;                        // keys of a matrix tile
// Tiles of a wave's step.  In a block that takes a head as many as make its loads
// 16 KB (8 KB for e4m3 of 64 channels); where blocks share the keys one, which
// lets more of them fit a compute unit and wastes less at a head's end (512 heads of
// 129 to 4096 e4m3 keys: 54.3 us, with two tiles 59.0).
constexpr int step_tiles(int d, bool fp8, bool shared) { return !shared && (d == 64 || (d == 128 && fp8)) ? 2 : 1; }
// keys of a unit of work: a step of four waves
constexpr int unit_keys(int d, bool fp8, bool shared) { return 4 * kKeys * step_tiles(d, fp8, shared); }
// A maximum no score is below.  Finite, so that parts without keys join without
// inf - inf; only keys of score -inf have no weight against it.
constexpr float kNoScore = -FLT_MAX;

// N words that are read once (16-byte loads around the caches' replacement
// reach 7.1 TB/s where ordinary ones reach 6.2)
template <int N>
__device__ __forceinline__ auto once(const uint8_t* p)
{
    typedef uint32_t words __attribute__((ext_vector_type(N)));
    return __builtin_nontemporal_load(reinterpret_cast<const words*>(p));
}

// 16 bytes of a key's row, whose 64-byte stretch an instruction reads.  Through the
// caches but where blocks share heads of 128 channels.  Once, plain, caches in turn
// (us): a block a head, 128 heads of 100 to 500 bf16 keys, 64 channels 8.2, 7.3, 128
// channels 12.0, 10.2, 256 channels 21.0, 18.3; shared, 8 heads of 262143 bf16 keys,
// 64 channels 95.1, 90.9; 128 channels, 512 heads of 129 to 4096 bf16 keys 99.6, 100.7,
// e4m3 57.1, 59.1, 8 heads of 32768 e4m3 keys 20.3, 20.1; 256 channels, 128 heads of
// 1000 to 16000 bf16 keys 188, 181.
template <bool ONCE>
__device__ __forceinline__ v4u load(const uint8_t* p)
{
    if constexpr (ONCE)
        return once<4>(p);
    else
        return *reinterpret_cast<const v4u*>(p);
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{a, b}, bf2));
}

__device__ __forceinline__ uint32_t e4m3_pair(uint32_t w, bool high)
{
    return __builtin_bit_cast(uint32_t, high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true)
                                             : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false));
}

// max over the lanes that hold the same query (lanes l, l ^ 16, l ^ 32, l ^ 48)
__device__ __forceinline__ float column_max(float v)
{
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

__device__ __forceinline__ v4f mfma(v4u a, v4u b, v4f c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, a), __builtin_bit_cast(bf8, b), c, 0,
                                                   0, 0);
}

// the keys of a sequence that count, [first, n), and their units from `from` on
struct KeyRange {
    int n, first, from, units;
};
__device__ __forceinline__ KeyRange key_range(const PagedAttention& a, int64_t b, int unit)
{
    KeyRange r;
    r.n = min(max(a.lengths[b], 0), a.cache.table_pages << a.cache.page_shift);
    r.first = a.window > 0 ? max(0, r.n - a.window) : 0;
    r.from = r.first & ~(kKeys - 1);
    r.units = (r.n - r.from + unit - 1) / unit;
    return r;
}

// units [first, first + count) of `total` that block i of `blocks` takes
struct Share {
    int64_t first, count;
};
__device__ __forceinline__ Share share_of(int64_t total, int64_t blocks, int64_t i)
{
    const int64_t each = total / blocks, more = total - each * blocks;
    return {i * each + min(i, more), each + (i < more ? 1 : 0)};
}
// the block that takes unit u
__device__ __forceinline__ int64_t block_of(int64_t total, int64_t blocks, int64_t u)
{
    const int64_t each = total / blocks, more = total - each * blocks, border = more * (each + 1);
    return u < border ? u / (each + 1) : more + (u - border) / each;
}

// What the blocks of a shared call leave: two parts each of 16 queries (sums of
// their first and their last head), a maximum and a sum a query, and, of a block
// in which a head begins that others go on with, where the join finds it.
struct Part {
    int64_t b;
    int head0, queries, slot, blocks;            // blocks that have a part, this one first; 0: nothing to join
};
__device__ __forceinline__ float* parts_o(const PagedAttention& a) { return a.workspace; }
__device__ __forceinline__ f2* parts_ml(const PagedAttention& a, int d)
{
    return reinterpret_cast<f2*>(a.workspace + (int64_t)a.shared * 32 * d);
}
__device__ __forceinline__ Part* parts_of(const PagedAttention& a, int d)
{
    return reinterpret_cast<Part*>(a.workspace + (int64_t)a.shared * 32 * (d + 2));
}

// the waves' shared-memory accesses are done; loads stay on their way
__device__ __forceinline__ void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// the head that a block works on: sequence b, cache head and queries `part`,
// units [unit, unit + count) of it
struct Head {
    int64_t b;
    int part, unit, count;
    KeyRange range;
};

// shared blocks, of four waves, that fit a compute unit
constexpr int fits(int d, bool fp8) { return d <= 128 ? 3 : fp8 ? 2 : 1; }

// SHARED: a block takes a run of units; otherwise a head.
template <int D, bool FP8, int WAVES, bool SHARED>
__global__ __launch_bounds__(64 * WAVES, SHARED ? fits(D, FP8) : 1) void paged_attention_kernel(
    const PagedAttention a, int tiles)
{
    constexpr int kWaves = WAVES, kThreads = 64 * kWaves;
    constexpr int kR = step_tiles(D, FP8, SHARED), kStep = kKeys * kR, kPass = kStep * kWaves;
    constexpr int kUnit = unit_keys(D, FP8, SHARED);
    constexpr int kSteps = D / 32;               // matrix steps over the channels
    constexpr int kTiles = D / 16;               // row tiles of O^T
    constexpr int kRun = FP8 || D < 256 ? kTiles : 8;        // channels of a lane's load of V: at most 16 bytes
    constexpr int kRow = D + 4;
    constexpr int kBytes = FP8 ? 1 : 2;
    __shared__ float part_o[kWaves][16][kRow];
    __shared__ float part_m[kWaves][16], part_l[kWaves][16];
    __shared__ uint32_t sums[kWaves];
    __shared__ int64_t found[2];

    const PagedCacheView& c = a.cache;
    const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int parts = c.heads * tiles, group = a.heads / c.heads;

    // ---- this block's run of units
    Head at;
    Share share{0, 0};
    int64_t total = 0;
    if constexpr (!SHARED) {
        at.b = blockIdx.x / (uint32_t)parts;
        at.part = (int)(blockIdx.x % (uint32_t)parts);
        at.unit = 0;
    } else {
        // sequences without keys are in no run
        for (int64_t b = blockIdx.x; b < c.sequences; b += gridDim.x)
            if (key_range(a, b, kUnit).units == 0)
                for (int i = 4 * threadIdx.x; i < a.heads * D; i += 4 * kThreads)
                    *reinterpret_cast<uint2*>(a.o + b * a.o_token + i / D * a.o_head + i % D) = uint2{0, 0};
        // prefix sums of the sequences' units, kThreads sequences at a time: the
        // total first, then where the run begins
        uint32_t mine = 0, before = 0, sum = 0;      // 2^23 units a sequence at most
        auto scan = [&](int64_t b0) {
            const int64_t b = b0 + threadIdx.x;
            mine = b < c.sequences ? (uint32_t)key_range(a, b, kUnit).units : 0u;
            uint32_t up = mine;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const uint32_t other = __shfl_up(up, d);
                up += lane >= d ? other : 0u;
            }
            __syncthreads();
            if (lane == 63)
                sums[wave] = up;
            __syncthreads();
            before = up - mine;
            sum = 0;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                before += w < wave ? sums[w] : 0u;
                sum += sums[w];
            }
        };
        for (int64_t b0 = 0; b0 < c.sequences; b0 += kThreads) {
            scan(b0);
            total += sum;
        }
        total *= parts;
        share = share_of(total, gridDim.x, blockIdx.x);
        if (share.count == 0) {
            if (threadIdx.x == 0)
                parts_of(a, D)[blockIdx.x] = Part{0, 0, 0, 0, 0};
            return;
        }
        int64_t behind = 0;
        for (int64_t b0 = 0;; b0 += kThreads) {
            if (c.sequences > kThreads)
                scan(b0);
            const int64_t begin = (behind + before) * parts;
            if (share.first >= begin && share.first < begin + (int64_t)mine * parts) {
                found[0] = b0 + threadIdx.x;
                found[1] = begin;
            }
            behind += sum;
            if (share.first < behind * parts)
                break;
        }
        __syncthreads();
        at.b = found[0];
        at.range = key_range(a, at.b, kUnit);
        const int64_t inside = share.first - found[1];
        at.part = (int)(inside / at.range.units);
        at.unit = (int)(inside - (int64_t)at.part * at.range.units);
        at.count = (int)min(share.count, (int64_t)(at.range.units - at.unit));
    }

    // the head in work: its pointers, Q^T, sums, and the first step's keys and values
    const int mask = (1 << c.page_shift) - 1, last_page = c.table_pages - 1;
    const uint8_t *keys, *values;
    const int32_t* table;
    int key0, end;
    v4u qf[kSteps];
    v4f acc[kTiles], sum;
    float top;

    // the pages of a step's keys: of key rows m and m + 16, and of value rows 8
    // g .. of each tile.  Past the sequence's end the table may hold anything.
    struct Pages {
        int32_t k[kR], v[kR];
    };
    auto find = [&](int key0) {
        Pages p;
#pragma unroll
        for (int r = 0; r < kR; ++r) {
            const int kb = key0 + kKeys * r + 8 * (m >> 2), vb = key0 + kKeys * r + 8 * g;
            p.k[r] = table[min(kb >> c.page_shift, last_page)];
            p.v[r] = table[min(vb >> c.page_shift, last_page)];
        }
        return p;
    };
    auto is_page = [&](int32_t id) { return id >= 0 && id < c.pages; };
    v4u kr[kR][2][FP8 ? kSteps / 2 : kSteps];
    uint32_t vr[kR][8][D * kBytes / 64];
    auto fetch_keys = [&](int key0, const Pages& pages) {
#pragma unroll
        for (int r = 0; r < kR; ++r) {
            const int kb = key0 + kKeys * r + 8 * (m >> 2);
            const int64_t page = is_page(pages.k[r]) ? pages.k[r] : 0;
            const uint8_t* p = keys + 16 * g + (page * c.page_stride + (int64_t)((kb & mask) + (m & 3)) * D) * kBytes;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int s = 0; s < (FP8 ? kSteps / 2 : kSteps); ++s)
                    kr[r][t][s] = load<SHARED && D == 128>(p + 4 * t * D * kBytes + 64 * s);
        }
    };
    auto fetch_values = [&](int key0, const Pages& pages) {
        constexpr int kWords = kRun * kBytes / 4;
#pragma unroll
        for (int r = 0; r < kR; ++r) {
            const int vb = key0 + kKeys * r + 8 * g;
            const int64_t page = is_page(pages.v[r]) ? pages.v[r] : 0;
            const uint8_t* p = values + (page * c.page_stride + (int64_t)(vb & mask) * D + kRun * m) * kBytes;
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int i = 0; i < kTiles / kRun; ++i) {
                    const auto w = once<kWords>(p + (j * D + 16 * kRun * i) * kBytes);
#pragma unroll
                    for (int n = 0; n < kWords; ++n)
                        vr[r][j][kWords * i + n] = w[n];
                }
        }
    };
    // S^T of a step, times the scale in units of log2
    auto score = [&](float (&p)[kR][8]) {
#pragma unroll
        for (int r = 0; r < kR; ++r) {
            v4f s0 = {}, s1 = {};
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                v4u k0, k1;
                if constexpr (FP8) {
                    const v4u w0 = kr[r][0][s / 2], w1 = kr[r][1][s / 2];
                    const int n = 2 * (s & 1);
                    k0 = v4u{e4m3_pair(w0[n], false), e4m3_pair(w0[n], true), e4m3_pair(w0[n + 1], false), e4m3_pair(w0[n + 1], true)};
                    k1 = v4u{e4m3_pair(w1[n], false), e4m3_pair(w1[n], true), e4m3_pair(w1[n + 1], false), e4m3_pair(w1[n + 1], true)};
                } else {
                    k0 = kr[r][0][s];
                    k1 = kr[r][1][s];
                }
                s0 = mfma(k0, qf[s], s0);
                s1 = mfma(k1, qf[s], s1);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                p[r][i] = s0[i] * a.scale;
                p[r][4 + i] = s1[i] * a.scale;
            }
        }
    };
    auto accumulate = [&](int key0, float (&p)[kR][8], const Pages& pages) {
        // keys outside the range and pages out of range: no weight, whatever
        // their places hold (a NaN there must not reach either product)
        bool all = key0 >= at.range.first && key0 + kStep <= end;
#pragma unroll
        for (int r = 0; r < kR; ++r)
            all = all && __all(is_page(pages.v[r]));
        if (!all) {
#pragma unroll
            for (int r = 0; r < kR; ++r)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int key = key0 + kKeys * r + 8 * g + j;
                    const bool counts = is_page(pages.v[r]) && key >= at.range.first && key < end;
                    p[r][j] = counts ? p[r][j] : -__builtin_inff();
#pragma unroll
                    for (int i = 0; i < D * kBytes / 64; ++i)
                        vr[r][j][i] = counts ? vr[r][j][i] : 0u;
                }
        }
        float most = p[0][0];
#pragma unroll
        for (int r = 0; r < kR; ++r)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                most = fmaxf(most, p[r][j]);
        most = column_max(most);
        if (__any(most > top)) {
            const float next = fmaxf(most, top);
            const float by = __builtin_amdgcn_exp2f(top - next);
            top = next;
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
                acc[t] *= by;
            sum *= by;
        }
#pragma unroll
        for (int r = 0; r < kR; ++r) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                p[r][j] = __builtin_amdgcn_exp2f(p[r][j] - top);
            v4u pf, rest;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float a = p[r][2 * j], b = p[r][2 * j + 1];
                pf[j] = pack_bf16(a, b);
                rest[j] = pack_bf16(a - __uint_as_float(pf[j] << 16), b - __uint_as_float(pf[j] & 0xFFFF0000u));
            }
            const uint32_t one = 0x3F803F80u;
            const v4u ones = {one, one, one, one};
            sum = mfma(ones, rest, mfma(ones, pf, sum));
            // a channel's 8 keys from a word (two channels, e4m3: four) of each key's row
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                const uint32_t pick = t & 1 ? 0x07060302u : 0x05040100u;
                v4u vf;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t lo, hi;
                    if constexpr (FP8) {
                        lo = e4m3_pair(vr[r][2 * j][t / 4], t / 2 & 1);
                        hi = e4m3_pair(vr[r][2 * j + 1][t / 4], t / 2 & 1);
                    } else {
                        lo = vr[r][2 * j][t / 2];
                        hi = vr[r][2 * j + 1][t / 2];
                    }
                    vf[j] = __builtin_amdgcn_perm(hi, lo, pick);
                }
                acc[t] = mfma(vf, rest, mfma(vf, pf, acc[t]));
            }
        }
    };

    // Everything of a head up to its first loads.  Q^T: lane (m, g) holds query m;
    // step s holds the channels that the key loads put there.
    Pages now, next;
    auto begin = [&](const Head& x) {
        const int kv = x.part / tiles, tile = x.part - kv * tiles;
        const int queries = min(16, group - 16 * tile), head0 = kv * group + 16 * tile;
        const int64_t head_at = ((int64_t)kv << c.page_shift) * D;
        keys = static_cast<const uint8_t*>(c.k) + head_at * kBytes;
        values = static_cast<const uint8_t*>(c.v) + head_at * kBytes;
        table = c.table + x.b * c.table_stride;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int channel = FP8 ? 64 * (s / 2) + 16 * g + 8 * (s & 1) : 32 * s + 8 * g;
            qf[s] = m < queries
                        ? *reinterpret_cast<const v4u*>(a.q + x.b * a.q_token + (head0 + m) * a.q_head + channel)
                        : v4u{0, 0, 0, 0};
        }
        now = find(key0);
        next = find(key0 + kPass);
        fetch_keys(key0, now);
        fetch_values(key0, now);
    };

    if constexpr (SHARED) {
        key0 = at.range.from + at.unit * kUnit + kStep * wave;
        begin(at);
    } else {
        at.range = key_range(a, at.b, kUnit);
        at.count = at.range.units;
        key0 = at.range.from + kStep * wave;
        if (key0 < at.range.n)
            begin(at);
    }

    for (int64_t left = share.count;;) {
        end = min(at.range.n, at.range.from + (at.unit + at.count) * kUnit);
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
            acc[t] = v4f{};
        sum = v4f{};
        top = kNoScore;
        // the next step's keys are asked for as soon as this one's scores have
        // used the registers, its values when the product has
        if (key0 < end) {
            float p[kR][8];
            for (; key0 + kPass < end; key0 += kPass) {
                score(p);
                const Pages after = find(key0 + 2 * kPass);
                fetch_keys(key0 + kPass, next);
                accumulate(key0, p, now);
                fetch_values(key0 + kPass, next);
                now = next;
                next = after;
            }
            score(p);
            accumulate(key0, p, now);
        }

        // the next head of this block's run: its first loads are on their way
        // while the waves' sums of this one meet
        const Head done = at;
        const bool first_head = left == share.count;
        left -= at.count;
        if (SHARED && left > 0) {
            if (++at.part == parts) {
                at.part = 0;
                do
                    at.range = key_range(a, ++at.b, kUnit);
                while (at.range.units == 0);
            }
            at.unit = 0;
            at.count = (int)min(left, (int64_t)at.range.units);
            key0 = at.range.from + kStep * wave;
            begin(at);
        }

        const int kv = done.part / tiles, tile = done.part - kv * tiles;
        const int queries = min(16, group - 16 * tile), head0 = kv * group + 16 * tile;
        // a short sequence may leave waves without keys
        const int used = SHARED ? kWaves : max(1, min(kWaves, (at.range.n - at.range.from + kStep - 1) / kStep));
        if (m < queries && wave < used) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int t = 0; t < kTiles; ++t)
                    part_o[wave][m][16 * kRun * (t / kRun) + kRun * (4 * g + i) + t % kRun] = acc[t][i];
            if (g == 0) {
                part_m[wave][m] = top;
                part_l[wave][m] = sum[0];
            }
        }
        meet();
        const bool whole = !SHARED || done.count == done.range.units;
        const int64_t row0 = (2 * (int64_t)blockIdx.x + (first_head ? 0 : 1)) * 16;
        for (int i = threadIdx.x * 4; i < queries * D; i += kThreads * 4) {
            const int query = i / D, channel = i % D;
            float high = part_m[0][query];
#pragma unroll
            for (int w = 1; w < kWaves; ++w)
                high = w < used ? fmaxf(high, part_m[w][query]) : high;
            v4f o = {};
            float l = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                if (w >= used)
                    break;
                const float by = __builtin_amdgcn_exp2f(part_m[w][query] - high);
                o += *reinterpret_cast<const v4f*>(&part_o[w][query][channel]) * by;
                l += part_l[w][query] * by;
            }
            if (whole) {
                const float by = l == 0.0f ? 0.0f : c.v_scale / l;     // normal: v_scale is at least 2^-96
                *reinterpret_cast<uint2*>(a.o + done.b * a.o_token + (head0 + query) * a.o_head + channel) =
                    uint2{pack_bf16(o[0] * by, o[1] * by), pack_bf16(o[2] * by, o[3] * by)};
            } else {
                *reinterpret_cast<v4f*>(parts_o(a) + (row0 + query) * D + channel) = o;
                if (channel == 0)
                    parts_ml(a, D)[row0 + query] = f2{high, l};
            }
        }
        if (SHARED && left <= 0 && threadIdx.x == 0) {
            // this block is the first of those that share its last head: what the join has to know
            const int rest = done.range.units - done.unit - done.count;
            Part r{done.b, head0, queries, first_head ? 0 : 1, 0};
            if (rest > 0 && done.unit == 0)
                r.blocks = (int)(block_of(total, gridDim.x, share.first + share.count + rest - 1) - blockIdx.x + 1);
            parts_of(a, D)[blockIdx.x] = r;
        }
        if (!SHARED || left <= 0)
            return;
        meet();                                  // the sums have been read
    }
}

// Joins the parts of the heads that several blocks worked on: block (i, query)
// those of a query of the head that began in block i and did not end there.  A
// thread takes four channels of every kTeams-th part.
template <int D>
__global__ __launch_bounds__(256) void paged_join_kernel(const PagedAttention a)
{
    constexpr int kLanes = D / 4, kTeams = 256 / kLanes;
    __shared__ v4f part[kTeams][kLanes];
    __shared__ float part_m[kTeams], part_l[kTeams];
    const Part r = parts_of(a, D)[blockIdx.x];
    const int query = blockIdx.y;
    if (r.blocks == 0 || query >= r.queries)
        return;
    const int at = threadIdx.x % kLanes, team = threadIdx.x / kLanes;
    v4f s = {};
    float high = kNoScore, l = 0.0f;
#pragma unroll 4
    for (int i = team; i < r.blocks; i += kTeams) {
        const int64_t row = (2 * ((int64_t)blockIdx.x + i) + (i == 0 ? r.slot : 0)) * 16 + query;
        const f2 w = parts_ml(a, D)[row];
        const v4f o = *reinterpret_cast<const v4f*>(parts_o(a) + row * D + 4 * at);
        const float next = fmaxf(high, w[0]);
        const float keep = __builtin_amdgcn_exp2f(high - next), by = __builtin_amdgcn_exp2f(w[0] - next);
        s = s * keep + o * by;
        l = l * keep + w[1] * by;
        high = next;
    }
    part[team][at] = s;
    if (at == 0) {
        part_m[team] = high;
        part_l[team] = l;
    }
    __syncthreads();
    if (team != 0)
        return;
    float most = high;
#pragma unroll
    for (int i = 1; i < kTeams; ++i)
        most = fmaxf(most, part_m[i]);
    s = v4f{};
    l = 0.0f;
#pragma unroll
    for (int i = 0; i < kTeams; ++i) {
        const float by = __builtin_amdgcn_exp2f(part_m[i] - most);
        s += part[i][at] * by;
        l += part_l[i] * by;
    }
    const float by = l == 0.0f ? 0.0f : a.cache.v_scale / l;
    *reinterpret_cast<uint2*>(a.o + r.b * a.o_token + (r.head0 + query) * a.o_head + 4 * at) =
        uint2{pack_bf16(s[0] * by, s[1] * by), pack_bf16(s[2] * by, s[3] * by)};
}

int tiles_of(int64_t heads, int64_t kv_heads) { return (int)((heads / kv_heads + 15) / 16); }

template <int D>
hipError_t launch(const PagedAttention& a, hipStream_t stream)
{
    const int tiles = tiles_of(a.heads, a.cache.heads);
    if (a.shared == 0) {
        const auto go = [&](auto waves) {
            constexpr int W = decltype(waves)::value;
            const uint32_t grid = (uint32_t)(a.cache.sequences * a.cache.heads * tiles);
            if (a.cache.fp8)
                paged_attention_kernel<D, true, W, false><<<grid, 64 * W, 0, stream>>>(a, tiles);
            else
                paged_attention_kernel<D, false, W, false><<<grid, 64 * W, 0, stream>>>(a, tiles);
        };
        if (a.waves == 1)
            go(std::integral_constant<int, 1>());
        else if (a.waves == 2)
            go(std::integral_constant<int, 2>());
        else
            go(std::integral_constant<int, 4>());
        return hipGetLastError();
    }
    if (a.cache.fp8)
        paged_attention_kernel<D, true, 4, true><<<(uint32_t)a.shared, 256, 0, stream>>>(a, tiles);
    else
        paged_attention_kernel<D, false, 4, true><<<(uint32_t)a.shared, 256, 0, stream>>>(a, tiles);
    paged_join_kernel<D><<<dim3((uint32_t)a.shared, (uint32_t)std::min(16, a.heads / a.cache.heads)), 256, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

int paged_blocks(int64_t sequences, int64_t heads, int64_t kv_heads, int64_t d, bool fp8, int64_t longest)
{
    const int64_t parts = sequences * kv_heads * tiles_of(heads, kv_heads);
    // Few heads: a block a compute unit, whose long runs one after the other the
    // memory serves best.  Many: as many as fit, so that one's change of heads is
    // another's work.  With one and three (us): 8 heads of 262144 bf16 keys 160, 169;
    // 64 of 32768 168, 174, of 256 to 7782 30.5, 29.5; 128 of 16384 168, 174, of 1024
    // to 31129 171, 172, as e4m3 95.8, 91.9; 512 of 256 to 7782 186, 174, as e4m3 118, 93
    // (equal lengths of 4096 as e4m3: 89, 94).
    const int64_t compute_units = device_compute_units();
    const int64_t resident = compute_units * (4 * parts <= compute_units ? 1 : fits((int)d, fp8));
    // a window's first key may lie inside a tile
    const int64_t unit = unit_keys((int)d, fp8, true), units = (longest + kKeys - 1 + unit - 1) / unit;
    // A block a head (one launch) where that is at most 4 passes of its waves, or 8
    // with a head for every compute unit.  So, and shared (us, caches in turn): 32
    // heads of 512 e4m3 keys (2 passes) 7.7, 9.5; of 1000 (4) 11.1, 10.0; of 1000 bf16
    // keys (8) 14.7, 11.1; 256 heads of 1000 to 1024 bf16 keys (8) 26.7, 32.7; 512 heads
    // of 1900 to 2000 e4m3 keys (8) 48.1, 56.8, of 100 to 2000 33.6, 36.1, of as many
    // bf16 keys (16, where one long head may hold up a call) 55.8, 57.4.
    const int64_t pass = unit_keys((int)d, fp8, false), passes = (longest + pass - 1) / pass;
    if (passes <= 4 || (passes <= 8 && parts >= compute_units))
        return 0;
    return (int)std::min(resident, parts * units);
}

// Four, or where there are few keys two, and one where more than two blocks a
// compute unit hide each other's latency.  With one and two (us), heads of up to 128
// keys: 32 of bf16 7.0, 5.9 (four: 5.8); 512 of 64 channels 6.4, 5.9, of 128 9.0, 8.3,
// of 256 12.9, 12.5; 640 7.1, 6.9; 9.6, 8.9; 14.5, 19.0; 1976 of 128 e4m3 channels
// 12.8, 15.7 (four: 21.7).  (Eight, of 333 keys, take what four do.)
int paged_waves(int64_t sequences, int64_t heads, int64_t kv_heads, int64_t longest)
{
    if (longest > 128)
        return 4;
    return sequences * kv_heads * tiles_of(heads, kv_heads) > 2 * device_compute_units() ? 1 : 2;
}

size_t paged_attention_bytes(int64_t d, int blocks)
{
    return (size_t)blocks * (32 * (size_t)(d + 2) * 4 + sizeof(Part));
}

hipError_t launch_paged_attention(const PagedAttention& a, hipStream_t stream)
{
    return a.cache.d == 64 ? launch<64>(a, stream) : a.cache.d == 128 ? launch<128>(a, stream) : launch<256>(a, stream);
}

}  // namespace quartz
