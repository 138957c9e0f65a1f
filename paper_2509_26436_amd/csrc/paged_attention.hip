// Attention of one new token a sequence over the pages of its cache:
//   o[b][h] = sum_j p_j v_j,  p = softmax_j(scale q[b][h] . k_j),
// j over the sequence's keys (the last `window` of them if that is set); a
// sequence without keys gives zeros.  Bound by the memory that holds the keys
// and values: each is read once and used by the `group` query heads that share
// it, up to 16 of them as the columns of one matrix tile.
//
// A block takes a run of split_keys keys of one (sequence, cache head); its
// four waves take 32 keys at a time.  No key or value passes through shared
// memory, because the matrix instructions' rows may be any keys and channels:
//   S^T = K Q^T: row 4 a + i of tile t is key 8 a + 4 t + i, so that the scores
//     a lane gets (one query, rows 4 g .. 4 g + 3 of two tiles) are keys 8 g ..
//     8 g + 7: exactly the 8 keys of its share of P^T in the next product;
//   O^T = V^T P^T: lane (m, g) reads channels (D/16) m .. + D/16 of keys 8 g ..
//     8 g + 7, whole rows of V over the 16 lanes, and turns the 8 x D/16 block
//     in registers; row m of tile t is channel (D/16) m + t, so that at the end
//     a lane holds D/16 neighbouring channels of its query.
// The softmax runs over the pass with a running maximum and sum in fp32 (base-2
// exponentials).  P is rounded to bf16 for the product, with a relative error of
// up to 2^-9 a weight as for the output itself, and the sum is that of the
// rounded weights (a row of ones beside V), so that weights add up to one.
// e4m3 keys and values are expanded to bf16, exactly, after the load; their
// scales go into the softmax scale and the output.
// Sequences longer than split_keys leave (maximum, sum, O) of every run in the
// workspace, and a second kernel joins them.
#include "quartz_internal.h"

namespace quartz {
namespace {

typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4;
constexpr int kKeys = 32;                        // keys of a wave's step
constexpr int kMostSplitKeys = 4096;
constexpr int kLeastPage = 8;
constexpr float kNoScore = -3.0e38f;             // a maximum below every score that counts

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

// the keys of a sequence that count: [first, n)
struct KeyRange {
    int n, first;
};
__device__ __forceinline__ KeyRange key_range(const PagedAttention& a, int64_t b)
{
    KeyRange r;
    r.n = min(max(a.lengths[b], 0), a.cache.table_pages << a.cache.page_shift);
    r.first = a.window > 0 ? max(0, r.n - a.window) : 0;
    return r;
}

template <int D, bool FP8>
__global__ __launch_bounds__(64 * kWaves) void paged_attention_kernel(const PagedAttention a, uint32_t tiles)
{
    constexpr int kSteps = D / 32;               // matrix steps over the channels
    constexpr int kTiles = D / 16;               // row tiles of O^T
    constexpr int kRow = D + 4;
    __shared__ float part[kWaves][16][kRow];
    __shared__ float part_m[kWaves][16], part_l[kWaves][16];
    __shared__ int32_t ids[kMostSplitKeys / kLeastPage + 1];

    const PagedCacheView& c = a.cache;
    const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t split = blockIdx.x % (uint32_t)a.splits, rest = blockIdx.x / (uint32_t)a.splits;
    const uint32_t part_of = rest % (c.heads * tiles);
    const int64_t b = rest / (c.heads * tiles);
    const int kv = part_of / tiles, tile = part_of % tiles;
    const int group = a.heads / c.heads, queries = min(16, group - 16 * tile);
    const int head0 = kv * group + 16 * tile;

    const KeyRange range = key_range(a, b);
    const int start = (range.first & ~(kKeys - 1)) + (int)split * a.split_keys;
    const int end = min(range.n, start + a.split_keys);
    if (start >= end && a.splits > 1)
        return;

    const int page0 = start >> c.page_shift;
    const int count = start < end ? ((end - 1) >> c.page_shift) - page0 + 1 : 0;
    for (int i = threadIdx.x; i < count; i += 64 * kWaves) {
        const int32_t id = c.table[b * c.table_stride + page0 + i];
        ids[i] = id >= 0 && id < c.pages ? id : -1;
    }

    // Q^T: lane (m, g) holds query m; step s holds the channels that the key
    // loads below put there
    v4u qf[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        const int channel = FP8 ? 64 * (s / 2) + 16 * g + 8 * (s & 1) : 32 * s + 8 * g;
        qf[s] = m < queries ? *reinterpret_cast<const v4u*>(a.q + b * a.q_token + (head0 + m) * a.q_head + channel)
                            : v4u{0, 0, 0, 0};
    }
    __syncthreads();

    const float scale = a.scale * 1.4426950408889634f * c.k_scale;
    v4f acc[kTiles] = {}, sum = {};
    float top = kNoScore;
    constexpr int kBytes = FP8 ? 1 : 2;
    const int64_t head_at = ((int64_t)kv << c.page_shift) * D;
    const uint8_t* keys = static_cast<const uint8_t*>(c.k) + head_at * kBytes;
    const uint8_t* values = static_cast<const uint8_t*>(c.v) + head_at * kBytes;
    const int mask = (1 << c.page_shift) - 1;

    for (int key0 = start + kKeys * wave; key0 < end; key0 += kKeys * kWaves) {
        const int kb = key0 + 8 * (m >> 2), vb = key0 + 8 * g;
        const int32_t kid = ids[(min(kb, end - 1) >> c.page_shift) - page0];
        const int32_t vid = vb < end ? ids[(vb >> c.page_shift) - page0] : -1;
        const uint8_t* kp = keys + ((int64_t)max(kid, 0) * c.page_stride + (int64_t)((kb & mask) + (m & 3)) * D) * kBytes;
        const uint8_t* vp = values + ((int64_t)max(vid, 0) * c.page_stride + (int64_t)(vb & mask) * D) * kBytes;
        v4u kf[2][kSteps];
        uint32_t vr[8][D / 32];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            if constexpr (FP8) {
#pragma unroll
                for (int s = 0; s < kSteps / 2; ++s) {
                    const v4u w = *reinterpret_cast<const v4u*>(kp + 4 * t * D + 64 * s + 16 * g);
                    kf[t][2 * s] = v4u{e4m3_pair(w[0], false), e4m3_pair(w[0], true), e4m3_pair(w[1], false), e4m3_pair(w[1], true)};
                    kf[t][2 * s + 1] = v4u{e4m3_pair(w[2], false), e4m3_pair(w[2], true), e4m3_pair(w[3], false), e4m3_pair(w[3], true)};
                }
            } else {
#pragma unroll
                for (int s = 0; s < kSteps; ++s)
                    kf[t][s] = *reinterpret_cast<const v4u*>(kp + (4 * t * D + 32 * s + 8 * g) * 2);
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint8_t* p = vp + (j * D + kTiles * m) * kBytes;
            if constexpr (FP8) {
                uint32_t w[D / 64];
                __builtin_memcpy(w, __builtin_assume_aligned(p, D / 16), D / 16);
#pragma unroll
                for (int i = 0; i < D / 64; ++i) {
                    vr[j][2 * i] = e4m3_pair(w[i], false);
                    vr[j][2 * i + 1] = e4m3_pair(w[i], true);
                }
            } else {
                __builtin_memcpy(vr[j], __builtin_assume_aligned(p, D == 64 ? 8 : 16), D / 8);
            }
        }

        v4f s0 = {}, s1 = {};
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            s0 = mfma(kf[0][s], qf[s], s0);
            s1 = mfma(kf[1][s], qf[s], s1);
        }
        float p[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            p[i] = s0[i] * scale;
            p[4 + i] = s1[i] * scale;
        }
        // keys outside the range and pages out of range: no weight, whatever
        // their places hold (a NaN there must not reach either product)
        if (key0 < range.first || key0 + kKeys > end || !__all(vid >= 0)) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bool counts = vid >= 0 && vb + j >= range.first && vb + j < end;
                p[j] = counts ? p[j] : -__builtin_inff();
#pragma unroll
                for (int i = 0; i < D / 32; ++i)
                    vr[j][i] = counts ? vr[j][i] : 0u;
            }
        }
        float most = fmaxf(fmaxf(fmaxf(p[0], p[1]), fmaxf(p[2], p[3])), fmaxf(fmaxf(p[4], p[5]), fmaxf(p[6], p[7])));
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
        for (int j = 0; j < 8; ++j)
            p[j] = __builtin_amdgcn_exp2f(p[j] - top);
        const v4u pf = {pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3]), pack_bf16(p[4], p[5]), pack_bf16(p[6], p[7])};
        const uint32_t one = 0x3F803F80u;
        sum = mfma(v4u{one, one, one, one}, pf, sum);
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            const uint32_t pick = t & 1 ? 0x07060302u : 0x05040100u;
            v4u vf;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                vf[j] = __builtin_amdgcn_perm(vr[2 * j + 1][t / 2], vr[2 * j][t / 2], pick);
            acc[t] = mfma(vf, pf, acc[t]);
        }
    }

    // the four waves' sums
    if (m < queries) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
                part[wave][m][kTiles * (4 * g + i) + t] = acc[t][i];
        if (g == 0) {
            part_m[wave][m] = top;
            part_l[wave][m] = sum[0];
        }
    }
    __syncthreads();
    const int64_t rows = c.sequences * a.heads;
    for (int at = threadIdx.x * 4; at < queries * D; at += 64 * kWaves * 4) {
        const int query = at / D, channel = at % D;
        float high = part_m[0][query];
#pragma unroll
        for (int w = 1; w < kWaves; ++w)
            high = fmaxf(high, part_m[w][query]);
        v4f o = {};
        float l = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float by = __builtin_amdgcn_exp2f(part_m[w][query] - high);
            o += *reinterpret_cast<const v4f*>(&part[w][query][channel]) * by;
            l += part_l[w][query] * by;
        }
        const int64_t head = head0 + query;
        if (a.splits == 1) {
            const float by = l == 0.0f ? 0.0f : c.v_scale / l;
            *reinterpret_cast<uint2*>(a.o + b * a.o_token + head * a.o_head + channel) =
                uint2{pack_bf16(o[0] * by, o[1] * by), pack_bf16(o[2] * by, o[3] * by)};
        } else {
            const int64_t row = (b * a.heads + head) * a.splits + split;
            *reinterpret_cast<v4f*>(a.workspace + row * D + channel) = o;
            if (channel == 0)
                *reinterpret_cast<f2*>(a.workspace + rows * a.splits * D + row * 2) = f2{high, l};
        }
    }
}

// A block joins the runs of one (sequence, head): each thread four channels of
// every 256 / (D / 4)-th run.
template <int D>
__global__ __launch_bounds__(256) void paged_join_kernel(const PagedAttention a)
{
    constexpr int kLanes = D / 4, kTeams = 256 / kLanes;
    __shared__ float high_of[4];
    __shared__ v4f part[kTeams][kLanes];
    __shared__ float part_l[kTeams];
    const int64_t b = blockIdx.x / (uint32_t)a.heads, head = blockIdx.x % (uint32_t)a.heads;
    const KeyRange range = key_range(a, b);
    const int from = range.first & ~(kKeys - 1);
    const int runs = (max(range.n - from, 0) + a.split_keys - 1) / a.split_keys;
    const int64_t row0 = (b * a.heads + head) * a.splits;
    const float* o = a.workspace + row0 * D;
    const f2* ml = reinterpret_cast<const f2*>(a.workspace + a.cache.sequences * a.heads * a.splits * D) + row0;

    float high = kNoScore;
    for (int i = threadIdx.x; i < runs; i += 256)
        high = fmaxf(high, ml[i][0]);
#pragma unroll
    for (int d = 32; d; d >>= 1)
        high = fmaxf(high, __shfl_xor(high, d));
    if ((threadIdx.x & 63) == 0)
        high_of[threadIdx.x >> 6] = high;
    __syncthreads();
    high = fmaxf(fmaxf(high_of[0], high_of[1]), fmaxf(high_of[2], high_of[3]));

    const int at = threadIdx.x % kLanes, team = threadIdx.x / kLanes;
    v4f s = {};
    float l = 0.0f;
    for (int i = team; i < runs; i += kTeams) {
        const f2 w = ml[i];
        const float by = __builtin_amdgcn_exp2f(w[0] - high);
        s += *reinterpret_cast<const v4f*>(o + (int64_t)i * D + 4 * at) * by;
        l += w[1] * by;
    }
    part[team][at] = s;
    if (at == 0)
        part_l[team] = l;
    __syncthreads();
    if (team != 0)
        return;
    for (int i = 1; i < kTeams; ++i) {
        s += part[i][at];
        l += part_l[i];
    }
    const float by = l == 0.0f ? 0.0f : a.cache.v_scale / l;
    *reinterpret_cast<uint2*>(a.o + b * a.o_token + head * a.o_head + 4 * at) =
        uint2{pack_bf16(s[0] * by, s[1] * by), pack_bf16(s[2] * by, s[3] * by)};
}

int tiles_of(int64_t heads, int64_t kv_heads) { return (int)((heads / kv_heads + 15) / 16); }

template <int D>
hipError_t launch(const PagedAttention& a, hipStream_t stream)
{
    const int tiles = tiles_of(a.heads, a.cache.heads);
    const uint32_t grid = (uint32_t)(a.cache.sequences * a.cache.heads * tiles * a.splits);
    if (a.cache.fp8)
        paged_attention_kernel<D, true><<<grid, 64 * kWaves, 0, stream>>>(a, tiles);
    else
        paged_attention_kernel<D, false><<<grid, 64 * kWaves, 0, stream>>>(a, tiles);
    if (a.splits > 1)
        paged_join_kernel<D><<<(uint32_t)(a.cache.sequences * a.heads), 256, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

PagedSplit paged_split(int64_t sequences, int64_t heads, int64_t kv_heads, int64_t d, int64_t longest)
{
    const int64_t parts = sequences * kv_heads * tiles_of(heads, kv_heads);
    int64_t keys = (longest * parts + 2047) / 2048;
    keys = (keys + 127) / 128 * 128;
    keys = keys < 128 ? 128 : keys > kMostSplitKeys ? kMostSplitKeys : keys;
    // a window's first key may lie inside a step
    const int64_t splits = (longest + kKeys - 1 + keys - 1) / keys;
    return {(int32_t)keys, (int32_t)(splits < 1 ? 1 : splits)};
}

size_t paged_attention_bytes(int64_t sequences, int64_t heads, int64_t d, const PagedSplit& s)
{
    return s.splits > 1 ? (size_t)(sequences * heads * s.splits) * (size_t)(d + 2) * 4 : 0;
}

hipError_t launch_paged_attention(const PagedAttention& a, hipStream_t stream)
{
    return a.cache.d == 64 ? launch<64>(a, stream) : a.cache.d == 128 ? launch<128>(a, stream) : launch<256>(a, stream);
}

}  // namespace quartz
