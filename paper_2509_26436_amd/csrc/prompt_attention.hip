// Attention of several new tokens a sequence over the pages of its cache (prompts
// and trees of drafted tokens):
//   o[i][h] = sum_j p_ij v_j,  p = softmax_j(b(scale q[i][h] . k_j)),
// b a cap (cap tanh(s / cap)) and a bias (- slope |position_i - j|), j over the
// keys that token i sees.  A row is one query head of one token; the heads that
// share a cache head are rows of one list, token after token, so that a block
// reads its keys and values once for all of them.
//
// A block takes a tile of 32 RW rows: RW waves of 32 rows, times KW waves that
// take the keys of a step in turn where there are few rows.  Keys and values pass
// through registers into shared memory a step ahead (the pages' rows are gathered
// on the way; e4m3 is expanded, exactly).
//   S^T = K Q^T (32 x 32 x 16 instructions): the rows of K lie in an order in which
//     the 16 scores that a lane gets, of one query, are two runs of 8 keys: its
//     share of P^T in the next product, without an exchange.
//   O^T = V^T P^T: V^T comes out of shared memory by transposing reads.
// The softmax runs along with a running maximum (kept while weights are at most 2^8
// above one: moved at every step 8 ragged prompts take 188 us for 173) and fp32 sums.
//
// P enters the product in 16 bits.  In fp16, times 2^7, a weight is off by 2^-11 of
// itself down to 2^-21 of the largest one, where bf16 would leave 2^-8, and V is
// turned to fp16, times 2^7, on its way into shared memory, exactly: zero or
// 2^-24 <= |v| < 2^9 (e4m3: any number).  A step with another value keeps bf16
// values and takes the weights in two bf16 parts (2^-16), and counts infinities and
// NaN apart, for the rows that see them only: a weight of zero times either would
// reach rows that do not.  All steps so: 969 us for 645 (8192 tokens of 32 heads of 128
// channels).  O's sums are of up to 2^22 times a value and key, so a block that meets a
// value of 2^64 or more starts over: all its steps are such then, and the weights of n
// keys at most 1 / n, which no value is too large for (1110 us).
//
// What bounds it: long prompts the issue of instructions.  8192 tokens of 32 heads take
// 641 us, 858 TFLOP/s, where a large matrix product of the library reaches 1230; the
// matrix unit is busy for 36 % of the cycles.  A step of 64 keys and 32 rows
// has 32 products (36 cycles each, 16 of which keep vector instructions out) beside some
// 250 vector instructions (16 maxima, 32 products, 32 exponentials, 16 roundings, 16 sums,
// 64 for the values' turn to fp16), and its two waves a SIMD, which a barrier a step
// holds together, are in the same part of it at a time.  Trees over long caches are
// bound by the memory (128 of 2 to 7 nodes over bf16 keys 4.1 TB/s), short calls by
// the latencies of starts, pages and keys.
#include <algorithm>
#include <cfloat>

#include "quartz_internal.h"

namespace quartz {
namespace {

typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef unsigned short us2 __attribute__((ext_vector_type(2)));

constexpr float kNoScore = -FLT_MAX;             // a maximum no score is below, finite
constexpr float kSlack = 8.0f;                   // scores above the maximum before it moves (log2)
// Maxima past which a step's scores are rounded as the maximum was before it is taken off
// them.  Below, scores go into the exponential with their factor in one instruction, off by
// the roundings of the maximum, less than 2^-3; past 2^24 those could pass what fp16 holds.
constexpr float kLarge = 0x1p20f;
constexpr int kNoKey = 1 << 30;                  // behind all of a sequence's
constexpr float kWeight = 7.0f;                  // weights are held times 2^7
constexpr uint32_t kValue = 7;                   // values in fp16 times 2^7
constexpr uint32_t kLeast = (127 - 24) << 7, kMost = (127 + 9) << 7;   // bf16 magnitudes that fp16 takes
constexpr float kUnits = 0x1p-7f;                // of O over the weights' sum
constexpr uint32_t kHuge = (127 + 64) << 7;      // bf16 magnitudes whose sums could pass fp32's range

// Keys that a wave takes of a step, and keys of a step.  Where the memory bounds the
// call larger steps keep more of it on the way: 32 sequences of 5 to 26 nodes over 129
// to 4096 e4m3 keys 81.3 us with 32 keys a wave, 73.5 with 64; 9 to 16 nodes over as
// many bf16 keys of 64 channels 62.6, 53.1, of 128 (whose steps are in the registers
// then) 90.0, 110.8.
constexpr int wave_keys(int d, bool fp8, int kw)
{
    return (kw == 1 && d < 256) || (kw == 2 && (d == 64 || (d == 128 && fp8))) ? 64 : 32;
}
constexpr int step_keys(int d, bool fp8, int kw) { return kw * wave_keys(d, fp8, kw); }
// steps in shared memory
constexpr int buffers(int kw) { return kw == 1 ? 2 : 1; }

// Rows of shared memory: 16 bytes (V: 64, for the transposing reads) past the
// channels, so that the rows an instruction reads lie in different banks.
constexpr int k_pitch(int d) { return 2 * d + 16; }
constexpr int v_pitch(int d) { return 2 * d + 64; }
constexpr int buffer_bytes(int d, bool fp8, int kw) { return step_keys(d, fp8, kw) * (k_pitch(d) + v_pitch(d)); }
constexpr int merge_bytes(int d, int rw, int kw) { return kw == 1 ? 0 : rw * kw * 32 * (d + 4 + 2) * 4; }
constexpr int shared_bytes(int d, bool fp8, int rw, int kw)
{
    return std::max(buffers(kw) * buffer_bytes(d, fp8, kw), merge_bytes(d, rw, kw));
}
// Blocks of four waves that a compute unit's registers hold.  One row of waves over bf16
// keys of 128 channels wants all of them: 128 sequences of 2 to 7 nodes over 1000 to 4096
// keys 346 us with two blocks, 326 with one (4.1 TB/s; e4m3, which does not, 154, 228).
constexpr int blocks_fit(int d, bool fp8, int rw) { return d == 256 || (d == 128 && !fp8 && rw == 1) ? 1 : 2; }

__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{a, b}, bf2));
}

__device__ __forceinline__ uint2 output(v4f o) { return uint2{pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3])}; }

__device__ __forceinline__ uint32_t e4m3_bf16(uint32_t w, bool high)
{
    return __builtin_bit_cast(uint32_t, high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true)
                                             : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false));
}

__device__ __forceinline__ uint32_t e4m3_half(uint32_t w, bool high)
{
    return __builtin_bit_cast(uint32_t, high ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 128.0f, true)
                                             : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 128.0f, false));
}

// the other half wave's value, lanes l ^ 32
__device__ __forceinline__ f2 halves(float v)
{
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return f2{__uint_as_float(a[0]), __uint_as_float(a[1])};
}

__device__ __forceinline__ v16f mfma_bf16(v4u a, v4u b, v16f c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8, a), __builtin_bit_cast(bf8, b), c, 0, 0, 0);
}

__device__ __forceinline__ v16f mfma_half(v4u a, v4u b, v16f c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
}

// four keys of one channel each, from 4 keys x 16 channels of the 16 lanes around
typedef __attribute__((address_space(3))) const uint8_t* local_ptr;
__device__ __forceinline__ v2u transposed(local_ptr p)
{
    return __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)p));
}

// A value times a weight of a row that sees it: infinities stay, also where the weight is below
// fp32's numbers (of two NaN and a number the median is the number).
__device__ __forceinline__ float weighed(float v, float by)
{
    const float w = v * by;
    return __builtin_amdgcn_fmed3f(w, w, v);
}
__device__ __forceinline__ v4f weighed(v4f v, float by)
{
    return v4f{weighed(v[0], by), weighed(v[1], by), weighed(v[2], by), weighed(v[3], by)};
}

// the lowest n of 8 bits
__device__ __forceinline__ uint32_t below(int n) { return (1u << min(max(n, 0), 8)) - 1; }

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Parts of a tile's keys at most, and more than which teams of threads join: 8 nodes of
// 8 heads over 100000 keys 60.2 us with 64 parts that a thread joins one after the
// other, 36.5 with 128 and 29.2 with 256 that teams do; over 8000 e4m3 keys of two
// cache heads 18.3 and 14.9.
constexpr int64_t kMostParts = 256;
constexpr int kManyParts = 16;

// ---- the list of tiles

// rows of tile `index`: token `first` + r / group, head r % group for r in [row0, rows)
struct Tile {
    int first;                  // the sequence's first token
    int b, count, row0, rows;   // sequence, its tokens, this tile's rows of tokens x group
    int length, prefix;         // of its keys
};

// Tiles of all sequences one after the other, found by scanning their starts, which
// are taken as they are as long as they stay in [0, tokens] and do not fall.
__device__ __forceinline__ bool find_tile(const PromptAttention& a, int64_t index, int group, int rows, Tile& t)
{
    const int lane = threadIdx.x & 63;
    int64_t behind = 0;
    for (int64_t b0 = 0; b0 < a.cache.sequences; b0 += 64) {
        const int64_t b = b0 + lane;
        int64_t s0 = 0, n = 0;
        int length = 0, prefix = 0;
        if (b < a.cache.sequences) {
            length = a.lengths[b];
            prefix = a.prefix ? a.prefix[b] : 0;
            s0 = min(max((int64_t)a.starts[b], (int64_t)0), a.tokens);
            n = min(max((int64_t)a.starts[b + 1], s0), a.tokens) - s0;
        }
        const int mine = (int)((n * group + rows - 1) / rows);       // 2^30 rows in all
        int up = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int other = __shfl_up(up, d);
            up += lane >= d ? other : 0;
        }
        const uint64_t past = __ballot(index < behind + up);
        if (past != 0) {
            const int at = __ffsll((unsigned long long)past) - 1;
            const auto of = [&](int v) { return __builtin_amdgcn_readlane(v, at); };
            t.b = uniform((int)b0) + at;
            t.first = of((int)s0);
            t.count = of((int)n);
            t.row0 = (int)(index - behind - of(up - mine)) * rows;
            t.rows = min(rows, t.count * group - t.row0);
            t.length = (int)min(max((int64_t)of(length), (int64_t)0), (int64_t)a.cache.table_pages << a.cache.page_shift);
            t.prefix = min(max(of(prefix), 0), t.length);
            return true;
        }
        behind += __builtin_amdgcn_readlane(up, 63);
    }
    return false;
}

// What token i of a sequence sees: keys in [lo, hi) and those below pre; of a tree
// its newest places by the token's bits.
struct Sight {
    int lo, hi, pre;
};
__device__ __forceinline__ Sight sight_of(const PromptAttention& a, const Tile& t, int i)
{
    const int64_t end = (int64_t)t.length - t.count + i + 1;        // behind its own position
    Sight s;
    s.pre = t.prefix;
    if (a.tree) {
        s.hi = t.length;
        s.lo = 0;
    } else {
        s.hi = (int)min(max(end, (int64_t)0), (int64_t)t.length);
        s.lo = a.window > 0 ? (int)max(end - a.window, (int64_t)0) : 0;
    }
    return s;
}

// the keys that a tile's rows see, [from, to), in `count` parts of `unit`
struct Keys {
    int from, to, behind_gap, unit, count;
};
__device__ __forceinline__ Keys keys_of(const PromptAttention& a, const Tile& t, int group, int step)
{
    const Sight s0 = sight_of(a, t, t.row0 / group), s1 = sight_of(a, t, (t.row0 + t.rows - 1) / group);
    Keys k;
    k.to = max(s1.hi, s0.pre);
    k.behind_gap = s0.lo & ~(step - 1);
    k.from = s0.pre > 0 ? 0 : k.behind_gap;
    const int span = max(0, k.to - k.from);
    k.unit = max(a.unit, ((span + a.splits - 1) / a.splits + step - 1) & ~(step - 1));
    k.count = (span + k.unit - 1) / k.unit;
    return k;
}

__device__ __forceinline__ float* parts_o(const PromptAttention& a, int64_t slot, int rows, int d)
{
    return a.workspace + slot * rows * (d + 2);
}

template <int D, bool FP8, int RW, int KW>
__global__ __launch_bounds__(64 * RW * KW, blocks_fit(D, FP8, RW)) void prompt_attention_kernel(const PromptAttention a)
{
    constexpr int kThreads = 64 * RW * KW, kRows = 32 * RW;
    constexpr int kWaveKeys = wave_keys(D, FP8, KW), kStep = step_keys(D, FP8, KW), kHalves = kWaveKeys / 32;
    constexpr int kBuffers = buffers(KW);
    constexpr int kSteps = D / 16, kTiles = D / 32;
    constexpr int kBytes = FP8 ? 1 : 2;
    constexpr int kChunks = D * kBytes / 16;                 // 16-byte pieces of a key
    constexpr int kAll = kStep * kChunks, kMine = (kAll + kThreads - 1) / kThreads;
    __shared__ __align__(16) uint8_t shared[shared_bytes(D, FP8, RW, KW)];
    // steps whose keys lack pages, whose values need bf16, and of these the ones that hold infinities or
    // NaN, or huge values (or either): their numbers
    __shared__ __align__(16) int marks[kBuffers][4];

    const PagedCacheView& c = a.cache;
    const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rw = wave % RW, kw = wave / RW;
    const int group = a.heads / c.heads;
    const int kv = (int)(blockIdx.x % (uint32_t)c.heads);
    const int64_t rest = blockIdx.x / (uint32_t)c.heads;
    const int part = (int)(rest % a.splits);
    // a sequence's last tiles, which see the most keys, first
    const int64_t index = a.tiles - 1 - rest / a.splits;
    Tile tile;
    if (!find_tile(a, index, group, kRows, tile))
        return;
    const Keys keys = keys_of(a, tile, group, kStep);
    if (part >= max(keys.count, 1))
        return;
    const int first_key = keys.from + part * keys.unit;
    const int end_key = min(keys.to, first_key + keys.unit);

    // ---- this lane's row
    const int row = 32 * rw + n;
    const bool live = row < tile.rows;
    const int at_row = tile.row0 + min(row, tile.rows - 1);
    const int token = at_row / group, head = kv * group + at_row % group;
    Sight sight = sight_of(a, tile, token);
    const int base = tile.length - tile.count;               // of a tree's nodes; may be negative
    const int position = base + token;
    const uint64_t* bits = a.tree ? a.tree + (int64_t)(tile.first + token) * a.tree_token : nullptr;
    const float slope = a.slopes ? a.slopes[head] * 1.44269504f : 0.0f;
    // what all rows of the wave see without looking, and what any of them may
    int all_hi = a.tree ? base : sight.hi, all_lo = sight.lo, any_hi = max(sight.hi, sight.pre), any_lo = sight.lo;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        all_hi = min(all_hi, __shfl_xor(all_hi, d));
        all_lo = max(all_lo, __shfl_xor(all_lo, d));
        any_hi = max(any_hi, __shfl_xor(any_hi, d));
        any_lo = min(any_lo, __shfl_xor(any_lo, d));
    }
    all_hi = __builtin_amdgcn_readfirstlane(all_hi);
    all_lo = __builtin_amdgcn_readfirstlane(all_lo);
    any_hi = __builtin_amdgcn_readfirstlane(any_hi);
    any_lo = __builtin_amdgcn_readfirstlane(any_lo);

    v4u qf[kSteps];
    {
        const uint16_t* q = a.q + (int64_t)(tile.first + token) * a.q_token + (int64_t)head * a.q_head + 8 * h;
        const uint32_t sign = a.negate ? 0x80008000u : 0u;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            qf[s] = live ? *reinterpret_cast<const v4u*>(q + 16 * s) : v4u{0, 0, 0, 0};
            qf[s] ^= v4u{sign, sign, sign, sign};
        }
    }

    // ---- keys and values into shared memory, a step ahead
    const int mask = (1 << c.page_shift) - 1, last_page = c.table_pages - 1;
    const int64_t head_at = ((int64_t)kv << c.page_shift) * D;
    const uint8_t* k_at = static_cast<const uint8_t*>(c.k) + head_at * kBytes;
    const uint8_t* v_at = static_cast<const uint8_t*>(c.v) + head_at * kBytes;
    const int32_t* table = c.table + (int64_t)tile.b * c.table_stride;
    const bool stages = kAll >= kThreads || (int)threadIdx.x < kAll;
    int32_t pages[kMine];
    uint32_t counts = 0, holes = 0;
    v4u kr[kMine], vr[kMine];
    auto key_of = [&](int i) { return (int)(threadIdx.x + i * kThreads) / kChunks; };
    const int chunk = (int)threadIdx.x % kChunks;
    auto find = [&](int key0) {
#pragma unroll
        for (int i = 0; i < kMine; ++i)
            pages[i] = table[min((key0 + key_of(i)) >> c.page_shift, last_page)];
    };
    auto fetch = [&](int key0) {
        counts = holes = 0;
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int key = key0 + key_of(i);
            const bool is_page = pages[i] >= 0 && pages[i] < c.pages;
            counts |= (is_page && key < tile.length ? 1u : 0u) << i;
            holes |= !is_page && key < tile.length ? 1u : 0u;
            const int64_t at = ((is_page ? pages[i] : 0) * c.page_stride + (int64_t)(key & mask) * D) * kBytes + 16 * chunk;
            if (stages) {
                kr[i] = *reinterpret_cast<const v4u*>(k_at + at);
                vr[i] = *reinterpret_cast<const v4u*>(v_at + at);
            }
        }
    };
    auto k_row = [&](uint8_t* buffer, int key) {
        return buffer + ((key & ~12) | (key & 4) << 1 | (key & 8) >> 1) * k_pitch(D);
    };
    auto v_row = [&](uint8_t* buffer, int key) { return buffer + kStep * k_pitch(D) + key * v_pitch(D); };
    // stores what fetch() got; `found` marks the buffer's step where values need bf16
    auto store = [&](int slot, int found) {
        uint8_t* buffer = shared + slot * buffer_bytes(D, FP8, KW);
        uint32_t out = 0;                                    // bits of e4m3 NaN
        us2 least = {0xFFFF, 0xFFFF}, most = {0, 0};
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            if (!stages)
                break;
            const uint32_t keep = counts >> i & 1 ? ~0u : 0u;
            vr[i] &= v4u{keep, keep, keep, keep};
            uint8_t *kp = k_row(buffer, key_of(i)), *vp = v_row(buffer, key_of(i));
            if constexpr (FP8) {
                v4u k0, k1, v0, v1;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    k0[2 * j] = e4m3_bf16(kr[i][j], false);
                    k0[2 * j + 1] = e4m3_bf16(kr[i][j], true);
                    k1[2 * j] = e4m3_bf16(kr[i][2 + j], false);
                    k1[2 * j + 1] = e4m3_bf16(kr[i][2 + j], true);
                    v0[2 * j] = e4m3_half(vr[i][j], false);
                    v0[2 * j + 1] = e4m3_half(vr[i][j], true);
                    v1[2 * j] = e4m3_half(vr[i][2 + j], false);
                    v1[2 * j + 1] = e4m3_half(vr[i][2 + j], true);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    out |= (vr[i][j] & 0x7F7F7F7Fu) + 0x01010101u;
                *reinterpret_cast<v4u*>(kp + 32 * chunk) = k0;
                *reinterpret_cast<v4u*>(kp + 32 * chunk + 16) = k1;
                *reinterpret_cast<v4u*>(vp + 32 * chunk) = v0;
                *reinterpret_cast<v4u*>(vp + 32 * chunk + 16) = v1;
            } else {
                v4u v;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const us2 m = __builtin_bit_cast(us2, vr[i][j] & 0x7FFF7FFFu);
                    least = __builtin_elementwise_min(least, m - us2{1, 1});     // zero is none
                    most = __builtin_elementwise_max(most, m);
                    const uint32_t w = vr[i][j] + (kValue << 23 | kValue << 7);
                    v[j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(__uint_as_float(w << 16),
                                                                                  __uint_as_float(w & 0xFFFF0000u)));
                }
                *reinterpret_cast<v4u*>(kp + 16 * chunk) = kr[i];
                *reinterpret_cast<v4u*>(vp + 16 * chunk) = v;
            }
        }
        bool slow, special, huge = false;
        if constexpr (FP8) {
            slow = special = (out & 0x80808080u) != 0;
        } else {
            const uint32_t top = max(most[0], most[1]);
            special = top >= 0x7F80u;
            slow = top >= kMost || min(least[0], least[1]) < kLeast - 1;
            huge = top >= kHuge;
        }
        if (holes)
            marks[slot][0] = found;
        if (slow) {
            marks[slot][1] = found;
            if (special)
                marks[slot][2] = found;
            if (huge)
                marks[slot][3] = found;
        }
    };
    auto store_values = [&](int slot) {                      // as bf16
        uint8_t* buffer = shared + slot * buffer_bytes(D, FP8, KW);
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            if (!stages)
                break;
            uint8_t* vp = v_row(buffer, key_of(i));
            if constexpr (FP8) {
                v4u v0, v1;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    v0[2 * j] = e4m3_bf16(vr[i][j], false);
                    v0[2 * j + 1] = e4m3_bf16(vr[i][j], true);
                    v1[2 * j] = e4m3_bf16(vr[i][2 + j], false);
                    v1[2 * j + 1] = e4m3_bf16(vr[i][2 + j], true);
                }
                *reinterpret_cast<v4u*>(vp + 32 * chunk) = v0;
                *reinterpret_cast<v4u*>(vp + 32 * chunk + 16) = v1;
            } else {
                *reinterpret_cast<v4u*>(vp + 16 * chunk) = vr[i];
            }
        }
    };
    // the keys between the prefix and the windows are nobody's
    auto behind = [&](int key0) {
        const int next = key0 + kStep;
        return next >= sight.pre && next < keys.behind_gap ? keys.behind_gap : next;
    };

    v16f acc[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
        acc[t] = v16f{};
    float top = kNoScore, sum = 0.0f;
    bool large = true;                                       // a row's maximum is past kLarge, or none yet
    // A value is huge: the weights of fewer than 2^power keys are at most 2^-power in the product, and the
    // maximum moves at once.
    bool huge = false;
    const int power = 32 - __clz(max(end_key - first_key, 1));
    const float low = __uint_as_float(uniform(__float_as_uint((float)(-7 - power))));

    // one step's product of a wave with its 32 or 64 keys
    auto compute = [&](int slot, int key0, bool slow, bool special, bool holed) {
        const uint8_t* buffer = shared + slot * buffer_bytes(D, FP8, KW);
        const int mine = kw * kWaveKeys;
        key0 += mine;
        if (key0 >= any_hi || (key0 + kWaveKeys <= any_lo && key0 >= sight.pre))
            return;
        v16f s[kHalves];
        // reads of keys go kAhead instructions before the product that takes them
        const local_ptr kp = (local_ptr)buffer + (mine + n) * k_pitch(D) + 16 * h;
        constexpr int kProducts = kHalves * kSteps, kAhead = kProducts < 8 ? kProducts : 8;
        v4u ring[kAhead];
        auto key = [&](int j) {
            return *(__attribute__((address_space(3))) const v4u*)(kp + 32 * (j % kHalves) * k_pitch(D) + 32 * (j / kHalves));
        };
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            ring[j] = key(j);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < kProducts; ++j) {
            const int x = j % kHalves, i = j / kHalves;
            s[x] = mfma_bf16(ring[j % kAhead], qf[i], i == 0 ? v16f{} : s[x]);
            if (j + kAhead < kProducts)
                ring[j % kAhead] = key(j + kAhead);
            __builtin_amdgcn_sched_barrier(0);
        }
        const bool whole = !holed && ((key0 >= all_lo && key0 + kWaveKeys <= all_hi) || key0 + kWaveKeys <= sight.pre);
        uint32_t seen = 0xFFFFFFFFu;
        float most = -__builtin_inff(), by = a.scale;
        if (!whole || a.cap > 0.0f || a.slopes) {
            if (a.cap > 0.0f) {
                // cap tanh(y) = cap - 2 cap / (exp(2 y) + 1), in units of log2
#pragma unroll
                for (int x = 0; x < kHalves; ++x)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        s[x][e] = __builtin_fmaf(-2.0f * a.cap, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(s[x][e] * a.scale) + 1.0f), a.cap);
            } else {
#pragma unroll
                for (int x = 0; x < kHalves; ++x)
                    s[x] *= a.scale;
            }
            by = 1.0f;
            if (a.slopes) {
                const float far = (float)(key0 + 8 * h - position);
#pragma unroll
                for (int x = 0; x < kHalves; ++x)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        s[x][e] = __builtin_fmaf(-slope, __builtin_fabsf(far + (float)(32 * x + 16 * (e >> 3) + (e & 7))), s[x][e]);
            }
            if (!whole) {
#pragma unroll
                for (int x = 0; x < kHalves; ++x)
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        const int run = key0 + 32 * x + 16 * t + 8 * h;          // 8 keys of one page
                        uint32_t see;
                        if (a.tree) {
                            // the words around the run's first node; the past is all ones
                            const int node = run - base, first = node >> 6, shift = node & 63;
                            const uint64_t w0 = bits[min(max(first, 0), a.tree_words - 1)];
                            const uint64_t w1 = bits[min(max(first + 1, 0), a.tree_words - 1)];
                            const uint64_t lo = first < 0 ? ~0ull : first < a.tree_words ? w0 : 0;
                            const uint64_t hi = first + 1 < 0 ? ~0ull : first + 1 < a.tree_words ? w1 : 0;
                            see = (uint32_t)(lo >> shift | hi << 1 << (63 - shift)) & below(sight.hi - run);
                        } else {
                            see = (below(sight.hi - run) & ~below(sight.lo - run)) | below(sight.pre - run);
                        }
                        if (holed) {
                            const int32_t page = table[min(run >> c.page_shift, last_page)];
                            see = page >= 0 && page < c.pages ? see : 0u;
                        }
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            s[x][8 * t + j] = see >> j & 1 ? s[x][8 * t + j] : -__builtin_inff();
                        const int at = 16 * x + 8 * t;
                        seen = (seen & ~(0xFFu << at)) | see << at;
                    }
            }
        }
#pragma unroll
        for (int x = 0; x < kHalves; ++x)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                most = fmaxf(most, s[x][e]);
        most *= by;
        const f2 both = halves(most);
        most = fmaxf(both[0], both[1]);
        if (__any(most - top > (huge ? 0.0f : kSlack))) {
            const float next = fmaxf(most, top);
            const float keep = __builtin_amdgcn_exp2f(top - next);
            top = next;
            large = __any(__builtin_fabsf(top) > kLarge);
            sum *= keep;
            // a loop of none or one (as for the slow product, below)
            int infinities = !FP8 && huge ? 1 : 0;
            asm volatile("" : "+s"(infinities));
#pragma unroll 1
            for (; infinities > 0; --infinities)
#pragma unroll
                for (int t = 0; t < kTiles; ++t)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        acc[t][e] = weighed(acc[t][e], keep);
            const float rest = !FP8 && huge ? 1.0f : keep;
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
                acc[t] *= rest;
        }
        const float unit = huge ? low : kWeight;
        float off = unit - top;
        if (large) {
#pragma unroll
            for (int x = 0; x < kHalves; ++x)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    s[x][e] = s[x][e] * by - top;
            by = 1.0f;
            off = unit;
        }
#pragma unroll
        for (int x = 0; x < kHalves; ++x)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                s[x][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[x][e], by, off));
        // V^T: 4 keys x 4 channels of a lane, whose rows are channels 16 h' + 4 a + i
        const int g = lane >> 4 & 1, piece = lane & 3;
        const local_ptr vp = (local_ptr)buffer + kStep * k_pitch(D) + (mine + 8 * h + (lane >> 2 & 3)) * v_pitch(D) +
                             2 * (16 * (piece & 1) + 4 * (2 * g + (piece >> 1)));
        auto values = [&](local_ptr p, int tile) {
            const v2u lo = transposed(p + 64 * tile), hi = transposed(p + 64 * tile + 4 * v_pitch(D));
            return v4u{lo[0], lo[1], hi[0], hi[1]};
        };
        if (!slow) {
            v4u pp[2 * kHalves];
#pragma unroll
            for (int x = 0; x < kHalves; ++x)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    v4u& p = pp[2 * x + t];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const h2 two = __builtin_convertvector(f2{s[x][8 * t + 2 * j], s[x][8 * t + 2 * j + 1]}, h2);
                        sum = __builtin_amdgcn_fdot2(two, h2{1, 1}, sum, false);
                        p[j] = __builtin_bit_cast(uint32_t, two);
                    }
                }
            // reads of values go as far ahead
            constexpr int kProducts = 2 * kHalves * kTiles, kAhead = kProducts < 8 ? kProducts : 8;
            v4u ring[kAhead];
            auto value = [&](int j) { return values(vp + 16 * (j / kTiles) * v_pitch(D), j % kTiles); };
    #pragma unroll
            for (int j = 0; j < kAhead; ++j)
                ring[j] = value(j);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < kProducts; ++j) {
                acc[j % kTiles] = mfma_half(ring[j % kAhead], pp[j / kTiles], acc[j % kTiles]);
                if (j + kAhead < kProducts)
                    ring[j % kAhead] = value(j + kAhead);
                __builtin_amdgcn_sched_barrier(0);
            }
            }
        // 16 keys at a time, in a loop: few steps need it.  Its count is opaque, since as the other
        // branch of the above it would have a second set of O's registers.
        int runs = slow ? 2 * kHalves : 0;
        asm volatile("" : "+s"(runs));
#pragma unroll 1
        for (int run = 0; run < runs; ++run) {
            float w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                w[j] = s[0][j];
#pragma unroll
            for (int r = 1; r < 2 * kHalves; ++r)
                if (run == r)
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        w[j] = s[r / 2][8 * (r % 2) + j];
            v4u p, more;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                sum += w[2 * j] + w[2 * j + 1];
                // the values lack their factor of 2^7
                const float w0 = w[2 * j] * 0x1p7f, w1 = w[2 * j + 1] * 0x1p7f;
                const uint32_t two = pack_bf16(w0, w1);
                p[j] = two;
                more[j] = pack_bf16(w0 - __uint_as_float(two << 16), w1 - __uint_as_float(two & 0xFFFF0000u));
            }
            const local_ptr at = vp + 16 * run * v_pitch(D);
#pragma unroll
            for (int i = 0; i < kTiles; ++i) {
                v4u v = values(at, i);
                if (special)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t w = v[j];
                        v[j] = ((w & 0x7F80u) == 0x7F80u ? 0 : w & 0xFFFFu) |
                               ((w & 0x7F800000u) == 0x7F800000u ? 0 : w & 0xFFFF0000u);
                    }
                acc[i] = mfma_bf16(v, more, mfma_bf16(v, p, acc[i]));
            }
            if (!special)
                continue;
            // infinities of either sign and NaN, counted over the keys that the row sees
            v4u sees;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t two = seen >> (8 * run + 2 * j);
                sees[j] = (two & 1 ? 0x3F80u : 0u) | (two & 2 ? 0x3F800000u : 0u);
            }
#pragma unroll 1
            for (int kind = 0; kind < 3; ++kind) {
                const uint32_t least = kind == 0 ? 0x7F80u : kind == 1 ? 0xFF80u : 0x7F81u;
                const uint32_t last = kind == 2 ? 0x7FFFu : least, bits = kind == 2 ? 0x7FFFu : 0xFFFFu;
                const float what = kind == 0 ? __builtin_inff() : kind == 1 ? -__builtin_inff() : __builtin_nanf("");
                auto is = [&](uint32_t v) { return (v & bits) >= least && (v & bits) <= last; };
#pragma unroll
                for (int i = 0; i < kTiles; ++i) {
                    v4u v = values(at, i);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t w = v[j];
                        v[j] = (is(w & 0xFFFFu) ? 0x3F80u : 0u) | (is(w >> 16) ? 0x3F800000u : 0u);
                    }
                    const v16f found = mfma_bf16(v, sees, v16f{});
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        acc[i][e] += found[e] > 0.0f ? what : 0.0f;
                }
            }
        }
    };

    if (first_key < end_key) {
        for (int i = threadIdx.x; i < 4 * kBuffers; i += kThreads)
            (&marks[0][0])[i] = 0;
        find(first_key);
        fetch(first_key);
        find(behind(first_key));
        __syncthreads();
        store(0, 1);
        int slot = 0, found = 1;
        for (int key0 = first_key; key0 < end_key; ++found) {
            __syncthreads();
            const int4 mark = *reinterpret_cast<const int4*>(marks[slot]);
            const bool holed = uniform(mark.x) == found, special = uniform(mark.z) == found;
            bool slow = uniform(mark.y) == found;
            int next = behind(key0);
            if (huge | slow) {
                slow = true;
                if (!FP8 && !huge & (uniform(mark.w) == found)) {
                    // the block starts over; the first maximum of a row takes what the row has to nothing
                    huge = large = true;
                    top = kNoScore;
                    sum = 0.0f;
                    key0 = kNoKey;
                    next = first_key;
                    find(next);
                }
                store_values(slot);
                __syncthreads();
            }
            if (next < end_key) {
                fetch(next);
                find(behind(next));
            }
            compute(slot, key0, slow, special, holed);
            if (next < end_key) {
                if (kBuffers == 1)
                    __syncthreads();
                slot = kBuffers == 1 ? 0 : slot ^ 1;
                store(slot, found + 1);
            }
            key0 = next;
        }
    }

    // ---- the sums of the halves, then of the waves that took other keys
    {
        const f2 both = halves(sum);
        sum = both[0] + both[1];
    }
    float* const slots = parts_o(a, (index * c.heads + kv) * a.splits + part, kRows, D);
    const bool last = keys.count <= 1;
    const float weight = huge ? __builtin_amdgcn_ldexpf(0x1p14f, power) : 1.0f;
    // a part leaves its mean and the sum of its weights times 2^7
    auto write = [&](int row, int channel, v4f o, float top, float sum) {
        o *= sum == 0.0f ? 0.0f : kUnits / sum;
        if (last) {
            const int at = tile.row0 + row;
            uint16_t* to = a.o + (int64_t)(tile.first + at / group) * a.o_token + (int64_t)(kv * group + at % group) * a.o_head + channel;
            *reinterpret_cast<uint2*>(to) = output(o * c.v_scale);
        } else {
            *reinterpret_cast<v4f*>(slots + (int64_t)row * D + channel) = o;
            if (channel == 0)
                *reinterpret_cast<f2*>(slots + (int64_t)kRows * D + 2 * row) = f2{top, sum * weight};
        }
    };
    if constexpr (KW == 1) {
        if (live)
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
                for (int e = 0; e < 16; e += 4)
                    write(row, 32 * t + 16 * h + e, v4f{acc[t][e], acc[t][e + 1], acc[t][e + 2], acc[t][e + 3]}, top, sum);
    } else {
        constexpr int kRow = D + 4;
        __syncthreads();                                     // the last step's values have been read
        float* mine = reinterpret_cast<float*>(shared) + wave * 32 * (kRow + 2);
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                *reinterpret_cast<v4f*>(mine + n * kRow + 32 * t + 16 * h + e) = v4f{acc[t][e], acc[t][e + 1], acc[t][e + 2], acc[t][e + 3]};
        if (h == 0)
            *reinterpret_cast<f2*>(mine + 32 * kRow + 2 * n) = f2{top, sum};
        __syncthreads();
        for (int i = 4 * threadIdx.x; i < tile.rows * D; i += 4 * kThreads) {
            const int row = i / D, channel = i % D;
            float high = kNoScore;
            const float* from[KW];
            f2 ml[KW];
#pragma unroll
            for (int w = 0; w < KW; ++w) {
                from[w] = reinterpret_cast<const float*>(shared) + (w * RW + row / 32) * 32 * (kRow + 2);
                ml[w] = *reinterpret_cast<const f2*>(from[w] + 32 * kRow + 2 * (row % 32));
                high = fmaxf(high, ml[w][0]);
            }
            v4f o = {};
            float l = 0.0f;
#pragma unroll
            for (int w = 0; w < KW; ++w) {
                const float by = __builtin_amdgcn_exp2f(ml[w][0] - high);
                const v4f part = *reinterpret_cast<const v4f*>(from[w] + (row % 32) * kRow + channel);
                o += FP8 ? part * by : weighed(part, by);
                l += ml[w][1] * by;
            }
            write(row, channel, o, high, l);
        }
    }
}

// Joins the parts of tiles whose keys several blocks took: the mean of their means, a
// mean at every step, which no value is too large for.  A thread has four channels of a
// row; TEAMS: of every kTeams-th part of it, which meet in shared memory.
template <int D, int ROWS, bool TEAMS>
__global__ __launch_bounds__(256) void prompt_join_kernel(const PromptAttention a, int step)
{
    constexpr int kLanes = D / 4, kTeams = 256 / kLanes;
    const PagedCacheView& c = a.cache;
    const int group = a.heads / c.heads, kv = (int)(blockIdx.x % (uint32_t)c.heads);
    const int64_t index = blockIdx.x / (uint32_t)c.heads;
    Tile tile;
    if (!find_tile(a, index, group, ROWS, tile))
        return;
    const int team = (int)threadIdx.x / kLanes, lane = (int)threadIdx.x % kLanes, channel = 4 * lane;
    const int row = TEAMS ? blockIdx.y : blockIdx.y * kTeams + team;
    const Keys keys = keys_of(a, tile, group, step);
    if (row >= tile.rows || keys.count <= 1)
        return;                                  // with TEAMS the whole block
    v4f o = {};
    float high = kNoScore, l = 0.0f;
#pragma unroll 4
    for (int i = TEAMS ? team : 0; i < keys.count; i += TEAMS ? kTeams : 1) {
        const float* from = parts_o(a, (index * c.heads + kv) * a.splits + i, ROWS, D);
        const f2 ml = *reinterpret_cast<const f2*>(from + (int64_t)ROWS * D + 2 * row);
        const v4f part = *reinterpret_cast<const v4f*>(from + (int64_t)row * D + channel);
        const float next = fmaxf(high, ml[0]);
        const float old = l * __builtin_amdgcn_exp2f(high - next), more = ml[1] * __builtin_amdgcn_exp2f(ml[0] - next);
        l = old + more;
        const float by = l == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(l);
        o = weighed(o, old * by) + weighed(part, more * by);
        high = next;
    }
    if constexpr (TEAMS) {
        __shared__ v4f sums[kTeams][kLanes];
        __shared__ float tops[kTeams], weights[kTeams];
        sums[team][lane] = o;
        if (lane == 0) {
            tops[team] = high;
            weights[team] = l;
        }
        __syncthreads();
        if (team != 0)
            return;
#pragma unroll
        for (int i = 1; i < kTeams; ++i)
            high = fmaxf(high, tops[i]);
        l = 0.0f;
#pragma unroll
        for (int i = 0; i < kTeams; ++i)
            l += weights[i] * __builtin_amdgcn_exp2f(tops[i] - high);
        const float by = l == 0.0f ? 0.0f : 1.0f / l;
        o = v4f{};
#pragma unroll
        for (int i = 0; i < kTeams; ++i)
            o += weighed(sums[i][lane], weights[i] * __builtin_amdgcn_exp2f(tops[i] - high) * by);
    }
    const int at = tile.row0 + row;
    uint16_t* to = a.o + (int64_t)(tile.first + at / group) * a.o_token + (int64_t)(kv * group + at % group) * a.o_head + channel;
    *reinterpret_cast<uint2*>(to) = output(o * c.v_scale);
}

template <int D, bool FP8, int RW, int KW>
hipError_t launch(const PromptAttention& a, hipStream_t stream)
{
    const uint32_t grid = (uint32_t)(a.tiles * a.splits * a.cache.heads);
    prompt_attention_kernel<D, FP8, RW, KW><<<grid, 64 * RW * KW, 0, stream>>>(a);
    if (a.splits > 1) {
        const uint32_t tiles = (uint32_t)(a.tiles * a.cache.heads), rows = 32 * RW;
        constexpr int kStep = step_keys(D, FP8, KW);
        if (a.splits > kManyParts)
            prompt_join_kernel<D, 32 * RW, true><<<dim3(tiles, rows), 256, 0, stream>>>(a, kStep);
        else
            prompt_join_kernel<D, 32 * RW, false><<<dim3(tiles, rows / (1024 / D)), 256, 0, stream>>>(a, kStep);
    }
    return hipGetLastError();
}

template <int D, bool FP8>
hipError_t launch(const PromptAttention& a, hipStream_t stream)
{
    switch (a.rows) {
    case 32:
        if constexpr (D < 256)
            return launch<D, FP8, 1, 4>(a, stream);
        return hipErrorInvalidValue;
    case 64:
        return launch<D, FP8, 2, 2>(a, stream);
    case 128:
        return launch<D, FP8, 4, 1>(a, stream);
    default:
        if constexpr (D < 256)
            return launch<D, FP8, 8, 1>(a, stream);
        return hipErrorInvalidValue;
    }
}

template <int D>
hipError_t launch(const PromptAttention& a, hipStream_t stream)
{
    return a.cache.fp8 ? launch<D, true>(a, stream) : launch<D, false>(a, stream);
}

}  // namespace

PromptShape prompt_shape(int64_t tokens, int64_t sequences, int64_t heads, int64_t kv_heads, int64_t d, int64_t longest)
{
    const int64_t group = heads / kv_heads, rows = tokens * group;
    const int64_t each = (rows + sequences - 1) / sequences;
    PromptShape s;
    // As many rows as a sequence has, since a tile reads all of its keys and turns their
    // values: 8192 tokens of 32 heads 650 us with 256 rows, 750 with 128, 8 ragged prompts
    // over e4m3 169, 184; 1 to 8 drafted tokens of 32 heads 14.8 with 32 rows, 15.5 with 64,
    // 20.7 with 128.  (256 channels: 128 rows are a block's registers, 32 would be too few
    // for what is on its way.)
    s.rows = each <= 32 && d < 256 ? 32 : each <= 64 ? 64 : each <= 128 || d == 256 ? 128 : 256;
    s.tiles = rows / s.rows + std::min(sequences, tokens);
    // Parts of at least four steps or so; short sequences are one: 1000 tokens of 8 heads
    // 27.3 us with 256 keys a part, 33.1 with 512; 1 to 8 tokens over 341 keys 15.1 in two
    // parts, 13.6 in one.
    s.unit = longest > 512 ? 256 : 512;
    // As many as the device holds at once (tiles counted as if all sequences were alike, and
    // as long as the table is wide; blocks of 32 rows over bf16 keys of 128 channels, which
    // have a compute unit's registers each, go in two rounds): 64 nodes of 64 heads over
    // 131000 keys 357 us with 16 parts of each of 16 tiles, 389 with 32, 485 with 22, which
    // leave a second round that is almost empty.
    const int64_t resident = device_compute_units() * (s.rows == 256 || d == 256 ? 1 : 2);
    const int64_t parts = std::min(sequences, tokens) * ((each + s.rows - 1) / s.rows) * kv_heads;
    const int64_t units = std::min((longest + s.unit - 1) / s.unit, kMostParts);
    s.splits = (int)std::max<int64_t>(1, std::min(resident / parts, units));
    // More of them, four times as many at most, where that leaves compute units without a
    // tile: rounds of blocks beside what a join reads and writes.  64 keys take a block some
    // 2.2 us, in the middle of the kernels' own 1.5 (64 rows, e4m3 keys of 128 channels), 2.0
    // (64 channels), 2.5 (256 rows of 128) and 6.7 (256 channels).  17 trees of 24 to 48 nodes
    // over 3200 to 6000 e4m3 keys (136 tiles of 256 rows) 185 us in one part each, 130 so.
    if (parts < resident) {
        const auto expected = [&](int64_t splits) {
            const int64_t rounds = (parts * splits + resident - 1) / resident;
            return (double)rounds / splits * longest * (2.2 / 64) +
                   (splits > 1 ? 5.0 + (double)parts * splits * s.rows * (d + 2) * 8 / 5e6 : 0.0);
        };
        const int64_t most = std::min<int64_t>(units, 4 * s.splits);
        for (int64_t splits = s.splits + 1; splits <= most; ++splits)
            if (expected(splits) < expected(s.splits))
                s.splits = (int)splits;
    }
    return s;
}

size_t prompt_attention_bytes(const PromptShape& s, int64_t kv_heads, int64_t d)
{
    return s.splits == 1 ? 0 : (size_t)s.tiles * kv_heads * s.splits * s.rows * (d + 2) * 4;
}

hipError_t launch_prompt_attention(const PromptAttention& a, hipStream_t stream)
{
    return a.cache.d == 64 ? launch<64>(a, stream) : a.cache.d == 128 ? launch<128>(a, stream) : launch<256>(a, stream);
}

}  // namespace quartz
