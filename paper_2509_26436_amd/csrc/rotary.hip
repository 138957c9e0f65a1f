// Rotary positions, and the paged cache's append, which rotates keys on the way.
//
// Pair i of a head's first `rot` channels at position p is turned by the angle
// of p f_i turns: (a, b) -> (a cos - b sin, b cos + a sin) times a magnitude.
// f_i is a fixed-point fraction of a turn in units of 2^-64, so that p f_i
// modulo one turn is the 64-bit product that wraps: exact for every position,
// where an fp32 angle at position 2^20 would be off by up to 0.06.  The top 32
// bits, as a signed fraction of a turn, go to the sine and cosine instructions,
// which take turns (largest error over a turn's 2^16 steps: 1.2e-7).
//
// A unit is 16 channels of one head: eight pairs of two 16-byte vectors
// (rotated: channels 8 u and rot / 2 + 8 u for the half layout, 16 u and 16 u
// + 8 for the interleaved one; the other channels are copied 16 at a time).
// A thread keeps its unit's eight sines and cosines over several heads.  Both
// kernels are bound by memory traffic, two vectors in, two out a unit, past a start
// of some 5 us in which each thread waits for its position, page and rows in turn:
// keys and values of 4612 tokens of 8 x 128 take 12.8 us into a bf16 cache (37.8 MB)
// and 11.0 into an e4m3 one (28.3 MB), of 18448 tokens 35.4 and 27.9, 5.0 TB/s more
// in either.  V = 2 and V = 1 are
// the same with pairs of channels and single ones in place of vectors, for
// strides, alignments and numbers of channels that are no multiples of 8 (16),
// or of 2 (4).
#include "quartz_internal.h"

namespace quartz {
namespace {

typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef float f2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
constexpr int kHeadsPerThread = 4;

template <int V>
__device__ __forceinline__ void load(const uint16_t* p, float (&v)[V])
{
    if constexpr (V == 8) {
        const uint4 w = *reinterpret_cast<const uint4*>(p);
        const uint32_t d[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(d[i] << 16);
            v[2 * i + 1] = __uint_as_float(d[i] & 0xFFFF0000u);
        }
    } else if constexpr (V == 2) {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(p);
        v[0] = __uint_as_float(w << 16);
        v[1] = __uint_as_float(w & 0xFFFF0000u);
    } else {
        v[0] = __uint_as_float((uint32_t)*p << 16);
    }
}

template <int V>
__device__ __forceinline__ void store(uint16_t* p, const float (&v)[V])
{
    if constexpr (V == 8) {
        uint32_t d[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            d[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{v[2 * i], v[2 * i + 1]}, bf2));
        *reinterpret_cast<uint4*>(p) = uint4{d[0], d[1], d[2], d[3]};
    } else if constexpr (V == 2) {
        *reinterpret_cast<uint32_t*>(p) = __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{v[0], v[1]}, bf2));
    } else {
        *p = __builtin_bit_cast(uint16_t, (__bf16)v[0]);
    }
}

// x / scale from inverse = 1 / scale: the product, corrected by its remainder,
// which the second operation forms without an error.  A quotient that fp32 holds
// comes out as it is, so that a tie of the rounding to the cache's type is one.
// The compiler's division has twice the instructions, and bound an e4m3 append by
// them (4612 tokens of 8 x 128, one call's rows in the caches: 12.0 us with it, 8.9
// so).  An infinite
// product has no remainder; where the quotient is clamped at 448 (LOW) the product
// is at 1024, and x itself brings infinities and NaN back.
template <bool LOW>
__device__ __forceinline__ float quotient(float x, float scale, float inverse)
{
    float q = x * inverse;
    if constexpr (LOW)
        q = __builtin_amdgcn_fmed3f(q, -1024.0f, 1024.0f);
    // signs so that a zero keeps its own
    const float better = __builtin_fmaf(__builtin_fmaf(q, scale, -x), -inverse, q);
    return LOW || better == better ? better : q;
}

// e4m3, round to nearest even, saturating at 448; NaN stays NaN
__device__ __forceinline__ float e4m3_range(float v)
{
    return __builtin_elementwise_minimum(__builtin_elementwise_maximum(v, -448.0f), 448.0f);
}

__device__ __forceinline__ uint2 e4m3_eight(const float (&v)[8])
{
    uint32_t d[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_range(v[4 * i]), e4m3_range(v[4 * i + 1]), 0, false);
        d[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(e4m3_range(v[4 * i + 2]), e4m3_range(v[4 * i + 3]), w, true);
    }
    return uint2{d[0], d[1]};
}

template <int V>
__device__ __forceinline__ void store(uint8_t* p, const float (&v)[V])
{
    if constexpr (V == 2) {
        *reinterpret_cast<uint16_t*>(p) =
            (uint16_t)__builtin_amdgcn_cvt_pk_fp8_f32(e4m3_range(v[0]), e4m3_range(v[1]), 0, false);
    } else {
        *p = (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(e4m3_range(v[0]), 0.0f, 0, false);
    }
}

// The channels of unit u (two runs of V), and the sines and cosines of its pairs.
template <int V>
struct Unit {
    int at0, at1;
    bool turned;
    float cos[V], sin[V];
};

template <int V>
__device__ __forceinline__ Unit<V> make_unit(int u, int rot, bool interleaved, int32_t position,
                                             const int64_t* freqs, float magnitude, bool inverse)
{
    Unit<V> w;
    const int turned = rot / (2 * V);
    w.turned = u < turned;
    if (!w.turned) {
        w.at0 = 2 * V * u;
        w.at1 = w.at0 + V;
        return w;
    }
    w.at0 = interleaved ? 2 * V * u : V * u;
    w.at1 = interleaved ? w.at0 + V : w.at0 + rot / 2;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const uint64_t turn = (uint64_t)freqs[V * u + i] * (uint64_t)(int64_t)position;
        const float t = (float)(int32_t)(turn >> 32) * 0x1p-32f;
        w.cos[i] = __builtin_amdgcn_cosf(t) * magnitude;
        const float s = __builtin_amdgcn_sinf(t) * magnitude;
        w.sin[i] = inverse ? -s : s;
    }
    return w;
}

// a: the run at at0, b: the run at at1
template <int V>
__device__ __forceinline__ void turn(const Unit<V>& w, bool interleaved, float (&a)[V], float (&b)[V])
{
    if (!w.turned)
        return;
    if (!interleaved || V == 1) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float x = a[i], y = b[i];
            a[i] = __builtin_fmaf(-y, w.sin[i], x * w.cos[i]);
            b[i] = __builtin_fmaf(x, w.sin[i], y * w.cos[i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float(&c)[V] = i < V / 2 ? a : b;
            constexpr int half = V / 2;
            const int j = 2 * (i % (half ? half : 1));
            const float x = c[j], y = c[j + 1];
            c[j] = __builtin_fmaf(-y, w.sin[i], x * w.cos[i]);
            c[j + 1] = __builtin_fmaf(x, w.sin[i], y * w.cos[i]);
        }
    }
}

// `units` of a head; heads are taken kHeadsPerThread by kHeadsPerThread.  In
// place (copy == false) only the turned units are visited.
template <int V>
__global__ __launch_bounds__(kThreads) void rotary_kernel(const Rotary a, uint32_t units, uint32_t groups)
{
    const uint32_t id = blockIdx.x * kThreads + threadIdx.x;
    const uint32_t rest = id / units, u = id - rest * units;
    const uint32_t token = rest / groups, group = rest - token * groups;
    if (token >= a.tokens)
        return;
    const Unit<V> w = make_unit<V>((int)u, a.rot, a.interleaved, a.positions[token], a.freqs, a.magnitude,
                                   a.inverse);
    const uint16_t* x = a.x + (int64_t)token * a.x_token;
    uint16_t* y = a.y + (int64_t)token * a.y_token;
    const int first = (int)group * kHeadsPerThread;
    float v0[kHeadsPerThread][V], v1[kHeadsPerThread][V];
#pragma unroll
    for (int i = 0; i < kHeadsPerThread; ++i) {
        const int64_t at = (int64_t)min(first + i, a.heads - 1) * a.x_head;
        load<V>(x + at + w.at0, v0[i]);
        load<V>(x + at + w.at1, v1[i]);
    }
#pragma unroll
    for (int i = 0; i < kHeadsPerThread; ++i) {
        if (first + i >= a.heads)
            return;
        turn<V>(w, a.interleaved, v0[i], v1[i]);
        const int64_t at = (int64_t)(first + i) * a.y_head;
        store<V>(y + at + w.at0, v0[i]);
        store<V>(y + at + w.at1, v1[i]);
    }
}

// Keys and values of new tokens into the pages of their sequences; the keys
// turned on the way.  A token without a place (a sequence or a position out of
// range, a page out of range) is skipped.
template <typename T, int V>
__global__ __launch_bounds__(kThreads) void paged_append_kernel(const PagedAppend a, uint32_t units,
                                                                uint32_t groups)
{
    const uint32_t id = blockIdx.x * kThreads + threadIdx.x;
    uint32_t rest = id / units;
    const uint32_t u = id - rest * units;
    const uint32_t part = rest / groups, group = rest - part * groups;
    const uint32_t token = part >> 1;
    const bool values = part & 1;
    if (token >= a.tokens)
        return;
    const PagedCacheView& c = a.cache;
    const int32_t position = a.positions[token];
    const int64_t sequence = a.sequences ? (int64_t)a.sequences[token] : (int64_t)token;
    if (sequence < 0 || sequence >= c.sequences || position < 0 ||
        (position >> c.page_shift) >= c.table_pages)
        return;
    const int32_t page = c.table[sequence * c.table_stride + (position >> c.page_shift)];
    if (page < 0 || page >= c.pages)
        return;
    const Unit<V> w = make_unit<V>((int)u, values ? 0 : a.rot, a.interleaved, position, a.freqs, a.magnitude, false);
    T* y = static_cast<T*>(values ? c.v : c.k) + page * c.page_stride +
           (int64_t)(position & ((1 << c.page_shift) - 1)) * c.d;
    const int64_t y_head = (int64_t)c.d << c.page_shift;
    const float scale = values ? c.v_scale : c.k_scale, inverse = 1.0f / scale;
    const uint16_t* x = (values ? a.v : a.k) + (int64_t)token * (values ? a.v_token : a.k_token);
    const int64_t x_head = values ? a.v_head : a.k_head;
    const int first = (int)group * kHeadsPerThread;
    float v0[kHeadsPerThread][V], v1[kHeadsPerThread][V];
#pragma unroll
    for (int i = 0; i < kHeadsPerThread; ++i) {
        const int64_t at = (int64_t)min(first + i, c.heads - 1) * x_head;
        load<V>(x + at + w.at0, v0[i]);
        load<V>(x + at + w.at1, v1[i]);
    }
#pragma unroll
    for (int i = 0; i < kHeadsPerThread; ++i) {
        if (first + i >= c.heads)
            return;
        turn<V>(w, a.interleaved, v0[i], v1[i]);
        if (scale != 1.0f) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                v0[i][j] = quotient<sizeof(T) == 1>(v0[i][j], scale, inverse);
                v1[i][j] = quotient<sizeof(T) == 1>(v1[i][j], scale, inverse);
            }
        }
        T* to = y + (first + i) * y_head;
        if constexpr (V == 8 && sizeof(T) == 1) {
            const uint2 d0 = e4m3_eight(v0[i]), d1 = e4m3_eight(v1[i]);
            if (w.at1 == w.at0 + V) {            // a run of 16: one store
                *reinterpret_cast<uint4*>(to + w.at0) = uint4{d0.x, d0.y, d1.x, d1.y};
            } else {
                *reinterpret_cast<uint2*>(to + w.at0) = d0;
                *reinterpret_cast<uint2*>(to + w.at1) = d1;
            }
        } else {
            store<V>(to + w.at0, v0[i]);
            store<V>(to + w.at1, v1[i]);
        }
    }
}

// Channels of a vector: the most of 8, 2 and 1 that pairs, heads, strides and
// pointers allow (4608 tokens of 32 x 128, all turned: 14.2 us with 8; 20 of them
// turned: 15.4 us with 2, 21.6 with 1).
int vector_of(int d, int rot, uintptr_t pointers, int64_t strides)
{
    for (int v : {8, 2})
        if (d % (2 * v) == 0 && rot % (2 * v) == 0 && pointers % (2 * v) == 0 && (strides & (v - 1)) == 0)
            return v;
    return 1;
}

uint32_t blocks_of(int64_t threads) { return (uint32_t)((threads + kThreads - 1) / kThreads); }

}  // namespace

hipError_t launch_rotary(const Rotary& a, hipStream_t stream)
{
    const int64_t groups = (a.heads + kHeadsPerThread - 1) / kHeadsPerThread;
    const bool in_place = a.x == a.y;
    const int channels = in_place ? a.rot : a.d;
    const int64_t strides = a.x_token | a.x_head | a.y_token | a.y_head;
    const int v = vector_of(a.d, a.rot, reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.y), strides);
    const int64_t units = channels / (2 * v);
    if (units == 0)
        return hipSuccess;
    const uint32_t grid = blocks_of(a.tokens * groups * units);
    if (v == 8)
        rotary_kernel<8><<<grid, kThreads, 0, stream>>>(a, (uint32_t)units, (uint32_t)groups);
    else if (v == 2)
        rotary_kernel<2><<<grid, kThreads, 0, stream>>>(a, (uint32_t)units, (uint32_t)groups);
    else
        rotary_kernel<1><<<grid, kThreads, 0, stream>>>(a, (uint32_t)units, (uint32_t)groups);
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_append(const PagedAppend& a, hipStream_t stream)
{
    const int64_t groups = (a.cache.heads + kHeadsPerThread - 1) / kHeadsPerThread;
    const int v = vector_of(a.cache.d, a.rot, reinterpret_cast<uintptr_t>(a.k) | reinterpret_cast<uintptr_t>(a.v),
                            a.k_token | a.k_head | a.v_token | a.v_head);
    const int64_t units = a.cache.d / (2 * v);
    const uint32_t grid = blocks_of(a.tokens * 2 * groups * units);
    if (v == 8)
        paged_append_kernel<T, 8><<<grid, kThreads, 0, stream>>>(a, (uint32_t)units, (uint32_t)groups);
    else if (v == 2)
        paged_append_kernel<T, 2><<<grid, kThreads, 0, stream>>>(a, (uint32_t)units, (uint32_t)groups);
    else
        paged_append_kernel<T, 1><<<grid, kThreads, 0, stream>>>(a, (uint32_t)units, (uint32_t)groups);
    return hipGetLastError();
}

hipError_t launch_paged_append(const PagedAppend& a, hipStream_t stream)
{
    return a.cache.fp8 ? launch_append<uint8_t>(a, stream) : launch_append<uint16_t>(a, stream);
}

}  // namespace quartz
