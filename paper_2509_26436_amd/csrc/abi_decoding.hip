// C-ABI entry points of the decoding step: MXFP4 quantization and linear layer,
// rotary positions, paged cache and attention.  Host-side validation, then the
// launch on the caller's stream; include/quartz.h has the contract of each.
#include <algorithm>
#include <cfloat>
#include <cmath>

#include "abi_checks.h"
#include "mxfp4.h"
#include "quartz.h"
#include "quartz_internal.h"

using namespace quartz;

namespace {

// blocks of 512 threads whose grid stays below 2^32 threads
constexpr int64_t kMaxBlocks512 = (int64_t(1) << 23) - 1;
// elements of one rotary (append) call: below 2^32 threads of one pair each
constexpr int64_t kMaxRotary = int64_t(1) << 32;
constexpr int64_t kMaxAppend = int64_t(1) << 31;
// positions of one sequence's pages
constexpr int64_t kMaxPositions = int64_t(1) << 30;
constexpr int64_t kMaxStride = int64_t(1) << 40;
// attention's v_scale: over a sum of weights of up to kMaxPositions still normal
constexpr float kMinValueScale = 0x1p-96f;

bool layout_ok(int32_t layout) { return layout == QUARTZ_ROTARY_HALF || layout == QUARTZ_ROTARY_INTERLEAVED; }

bool stride_ok(int64_t s) { return s >= -kMaxStride && s <= kMaxStride; }

// a * b <= most for a, b >= 0
bool product_ok(int64_t a, int64_t b, int64_t most) { return b == 0 || a <= most / b; }

quartz_status mx_linear_checks(int64_t M, int64_t N, int64_t K, int64_t ldy, int32_t epilogue)
{
    if (epilogue != QUARTZ_EPI_NONE && epilogue != QUARTZ_EPI_GELU_TANH)
        return QUARTZ_ERR_UNSUPPORTED;
    if (K <= 0 || !size_ok(M, K) || !size_ok(N, K) || ldy < N || ldy > kMaxLd ||
        !product_ok((M + 255) / 256, (N + 255) / 256, kMaxBlocks512))
        return QUARTZ_ERR_SHAPE;
    return QUARTZ_OK;
}

struct MxWorkspace {
    size_t scales, total;      // codes first
};
MxWorkspace mx_workspace(int64_t M, int64_t K)
{
    MxWorkspace w;
    w.scales = ((size_t)mx_code_bytes(M, K) + 255) / 256 * 256;
    w.total = w.scales + (size_t)mx_scale_bytes(M, K);
    return w;
}

// the cache and its table; the pointers are looked at only if `used`
quartz_status cache_checks(const PagedCacheView& c, int64_t page_size, int32_t type, bool used)
{
    if (type != QUARTZ_CACHE_BF16 && type != QUARTZ_CACHE_E4M3)
        return QUARTZ_ERR_UNSUPPORTED;
    if (c.d != 64 && c.d != 128 && c.d != 256)
        return QUARTZ_ERR_UNSUPPORTED;
    if (!(c.k_scale >= FLT_MIN) || !(c.v_scale >= FLT_MIN) || !std::isfinite(c.k_scale) ||
        !std::isfinite(c.v_scale))
        return QUARTZ_ERR_UNSUPPORTED;
    if (page_size < 8 || page_size > 4096 || (page_size & (page_size - 1)) != 0)
        return QUARTZ_ERR_UNSUPPORTED;
    if (c.pages <= 0 || c.pages > INT32_MAX || c.table_pages < 0 || c.sequences < 0 ||
        c.table_stride < c.table_pages || c.table_stride > kMaxStride || c.page_stride > kMaxStride ||
        c.page_stride < (int64_t)c.heads * page_size * c.d || c.table_pages > kMaxPositions / page_size)
        return QUARTZ_ERR_SHAPE;
    if (!used)
        return QUARTZ_OK;
    if (!c.k || !c.v || (!c.table && c.table_pages > 0))
        return QUARTZ_ERR_NULL;
    if (!aligned16(c.k) || !aligned16(c.v) || !aligned(c.table, 4) || c.page_stride % (c.fp8 ? 16 : 8) != 0)
        return QUARTZ_ERR_ALIGN;
    return QUARTZ_OK;
}

int shift_of(int64_t page_size)
{
    int s = 0;
    while (s < 12 && (int64_t(1) << s) < page_size)
        ++s;
    return s;
}

}  // namespace

extern "C" {

quartz_status quartz_mxfp4_quantize(const void* x_bf16, int64_t M, int64_t K, int64_t ldx, uint8_t* codes,
                                    uint8_t* scales, hipStream_t stream)
{
    if (!size_ok(M, K) || ldx < K || ldx > kMaxLd)
        return QUARTZ_ERR_SHAPE;
    if (ldx % 8 != 0)
        return QUARTZ_ERR_ALIGN;
    if (M == 0 || K == 0)
        return QUARTZ_OK;
    if (!x_bf16 || !codes || !scales)
        return QUARTZ_ERR_NULL;
    if (!aligned16(x_bf16) || !aligned16(codes) || !aligned16(scales))
        return QUARTZ_ERR_ALIGN;
    return from_hip(launch_mxfp4_quantize(static_cast<const uint16_t*>(x_bf16), M, K, ldx, codes, scales, stream));
}

quartz_status quartz_mxfp4_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t M, int64_t K,
                                      void* y_bf16, int64_t ldy, hipStream_t stream)
{
    if (!size_ok(M, K) || ldy < K || ldy > kMaxLd)
        return QUARTZ_ERR_SHAPE;
    if (ldy % 8 != 0)
        return QUARTZ_ERR_ALIGN;
    if (M == 0 || K == 0)
        return QUARTZ_OK;
    if (!codes || !scales || !y_bf16)
        return QUARTZ_ERR_NULL;
    if (!aligned16(y_bf16) || !aligned16(codes) || !aligned16(scales))
        return QUARTZ_ERR_ALIGN;
    return from_hip(launch_mxfp4_dequantize(codes, scales, M, K, static_cast<uint16_t*>(y_bf16), ldy, stream));
}

quartz_status quartz_mxfp4_linear(const uint8_t* a_codes, const uint8_t* a_scales, const uint8_t* w_codes,
                                  const uint8_t* w_scales, const void* bias_bf16, void* y_bf16, int64_t M,
                                  int64_t N, int64_t K, int64_t ldy, int32_t epilogue, hipStream_t stream)
{
    const quartz_status st = mx_linear_checks(M, N, K, ldy, epilogue);
    if (st != QUARTZ_OK || M == 0 || N == 0)
        return st;
    if (!a_codes || !a_scales || !w_codes || !w_scales || !y_bf16)
        return QUARTZ_ERR_NULL;
    if (!aligned16(a_codes) || !aligned16(a_scales) || !aligned16(w_codes) || !aligned16(w_scales) ||
        !aligned16(y_bf16) || !aligned16(bias_bf16))
        return QUARTZ_ERR_ALIGN;
    return from_hip(launch_mxfp4_linear({nullptr, 0, a_codes, a_scales, w_codes, w_scales,
                                         static_cast<const uint16_t*>(bias_bf16), static_cast<uint16_t*>(y_bf16),
                                         M, N, K, ldy, epilogue == QUARTZ_EPI_GELU_TANH},
                                        stream));
}

size_t quartz_mxfp4_linear_workspace_bytes(int64_t M, int64_t K)
{
    if (M <= 0 || K <= 0 || !size_ok(M, K) || mxfp4_fuses(M, K))
        return 0;
    return mx_workspace(M, K).total;
}

quartz_status quartz_mxfp4_linear_bf16(const void* x_bf16, int64_t ldx, const uint8_t* w_codes,
                                       const uint8_t* w_scales, const void* bias_bf16, void* y_bf16, int64_t M,
                                       int64_t N, int64_t K, int64_t ldy, int32_t epilogue, void* workspace,
                                       size_t workspace_bytes, hipStream_t stream)
{
    const quartz_status st = mx_linear_checks(M, N, K, ldy, epilogue);
    if (st != QUARTZ_OK)
        return st;
    if (ldx < K || ldx > kMaxLd)
        return QUARTZ_ERR_SHAPE;
    if (ldx % 8 != 0)
        return QUARTZ_ERR_ALIGN;
    if (M == 0 || N == 0)
        return QUARTZ_OK;
    const bool fused = mxfp4_fuses(M, K);
    if (!x_bf16 || !w_codes || !w_scales || !y_bf16)
        return QUARTZ_ERR_NULL;
    if (!aligned16(x_bf16) || !aligned16(w_codes) || !aligned16(w_scales) || !aligned16(y_bf16) ||
        !aligned16(bias_bf16) || !aligned16(workspace))
        return QUARTZ_ERR_ALIGN;
    MxLinear a{static_cast<const uint16_t*>(x_bf16), ldx, nullptr, nullptr, w_codes, w_scales,
               static_cast<const uint16_t*>(bias_bf16), static_cast<uint16_t*>(y_bf16), M, N, K, ldy,
               epilogue == QUARTZ_EPI_GELU_TANH};
    if (!fused) {
        const MxWorkspace w = mx_workspace(M, K);
        if (!workspace || workspace_bytes < w.total)
            return QUARTZ_ERR_WORKSPACE;
        uint8_t* codes = static_cast<uint8_t*>(workspace);
        const hipError_t e = launch_mxfp4_quantize(a.x, M, K, ldx, codes, codes + w.scales, stream);
        if (e != hipSuccess)
            return from_hip(e);
        a.x = nullptr;
        a.x_codes = codes;
        a.x_scales = codes + w.scales;
    }
    return from_hip(launch_mxfp4_linear(a, stream));
}

quartz_status quartz_mxfp4_linear_kernel(int64_t M, int64_t N, int64_t K, int32_t* kernel)
{
    if (M <= 0 || N <= 0)
        return QUARTZ_ERR_SHAPE;
    const quartz_status st = mx_linear_checks(M, N, K, N, QUARTZ_EPI_NONE);
    if (st != QUARTZ_OK)
        return st;
    if (!kernel)
        return QUARTZ_ERR_NULL;
    const MxShape s = mxfp4_shape(M, N, K);
    const int unit = s.tiled ? 64 : 16;
    kernel[0] = s.tiled ? QUARTZ_MX_TILED : QUARTZ_MX_DIRECT;
    kernel[1] = unit * s.tm;
    kernel[2] = unit * s.tn;
    kernel[3] = mxfp4_fuses(M, K);
    return QUARTZ_OK;
}

quartz_status quartz_rotary_frequencies(int64_t rot, double base, int32_t scaling, double factor, double low,
                                        double high, double original, int64_t* freqs)
{
    if (scaling != QUARTZ_ROTARY_LINEAR && scaling != QUARTZ_ROTARY_BASE && scaling != QUARTZ_ROTARY_PARTS)
        return QUARTZ_ERR_UNSUPPORTED;
    if (rot < 0 || rot % 2 != 0 || rot > kMaxK)
        return QUARTZ_ERR_SHAPE;
    if (!(base >= 1.0) || !std::isfinite(base) || !(factor >= 1.0) || !std::isfinite(factor))
        return QUARTZ_ERR_UNSUPPORTED;
    if (scaling == QUARTZ_ROTARY_PARTS &&
        (!(low < high) || !std::isfinite(low) || !std::isfinite(high) || !(original > 0.0) ||
         !std::isfinite(original)))
        return QUARTZ_ERR_UNSUPPORTED;
    if (rot > 0 && !freqs)
        return QUARTZ_ERR_NULL;
    const long double two_pi = 6.283185307179586476925286766559005768L;
    if (scaling == QUARTZ_ROTARY_BASE && rot > 2)
        base = (double)((long double)base * std::pow((long double)factor, (long double)rot / (rot - 2)));
    for (int64_t i = 0; i < rot / 2; ++i) {
        long double turns = std::pow((long double)base, -2.0L * i / rot) / two_pi;
        if (scaling == QUARTZ_ROTARY_LINEAR) {
            turns /= factor;
        } else if (scaling == QUARTZ_ROTARY_PARTS) {
            long double keep = ((long double)original * turns - low) / ((long double)high - low);
            keep = keep < 0.0L ? 0.0L : keep > 1.0L ? 1.0L : keep;
            turns = turns * keep + turns / factor * (1.0L - keep);
        }
        // at most 1 / (2 pi) of a turn: below 2^63
        freqs[i] = (int64_t)std::llrint(turns * 18446744073709551616.0L);
    }
    return QUARTZ_OK;
}

quartz_status quartz_rotary(const void* x_bf16, void* y_bf16, int64_t tokens, int64_t heads, int64_t d,
                            int64_t rot, int64_t x_token, int64_t x_head, int64_t y_token, int64_t y_head,
                            const int32_t* positions, const int64_t* freqs, int32_t layout, int32_t inverse,
                            float magnitude, hipStream_t stream)
{
    if (!layout_ok(layout) || !std::isfinite(magnitude))
        return QUARTZ_ERR_UNSUPPORTED;
    if (tokens < 0 || heads < 0 || d <= 0 || d % 2 != 0 || d > kMaxK || rot < 0 || rot > d || rot % 2 != 0 ||
        tokens > kMaxRotary || heads > kMaxK || !product_ok(heads * d, tokens, kMaxRotary) ||
        !stride_ok(x_token) || !stride_ok(x_head) || !stride_ok(y_token) || !stride_ok(y_head))
        return QUARTZ_ERR_SHAPE;
    if (tokens == 0 || heads == 0)
        return QUARTZ_OK;
    if (!x_bf16 || !y_bf16 || !positions || (!freqs && rot > 0))
        return QUARTZ_ERR_NULL;
    if (!aligned(x_bf16, 2) || !aligned(y_bf16, 2) || !aligned(positions, 4) || !aligned(freqs, 8))
        return QUARTZ_ERR_ALIGN;
    if (x_bf16 == y_bf16 && (x_token != y_token || x_head != y_head))
        return QUARTZ_ERR_SHAPE;       // in place: the same elements
    return from_hip(launch_rotary({static_cast<const uint16_t*>(x_bf16), static_cast<uint16_t*>(y_bf16), tokens,
                                   (int32_t)heads, (int32_t)d, (int32_t)rot, x_token, x_head, y_token, y_head,
                                   positions, freqs, layout == QUARTZ_ROTARY_INTERLEAVED, inverse != 0, magnitude},
                                  stream));
}

quartz_status quartz_paged_append(const void* k_bf16, const void* v_bf16, int64_t tokens, int64_t heads, int64_t d,
                                  int64_t k_token, int64_t k_head, int64_t v_token, int64_t v_head,
                                  const int32_t* positions, const int32_t* sequences, const int64_t* freqs,
                                  int64_t rot, int32_t layout, float magnitude, void* k_cache, void* v_cache,
                                  int32_t cache_type, float k_scale, float v_scale, int64_t pages,
                                  int64_t page_size, int64_t page_stride, const int32_t* table,
                                  int64_t table_rows, int64_t table_pages, int64_t table_stride,
                                  hipStream_t stream)
{
    if (!layout_ok(layout) || !std::isfinite(magnitude))
        return QUARTZ_ERR_UNSUPPORTED;
    if (tokens < 0 || tokens > kMaxAppend || heads <= 0 || heads > kMaxK || d <= 0 || d > kMaxK || rot < 0 ||
        rot > d || rot % 2 != 0 || !product_ok(heads * d, tokens, kMaxAppend) || !stride_ok(k_token) ||
        !stride_ok(k_head) || !stride_ok(v_token) || !stride_ok(v_head) || table_pages < 0 ||
        table_pages > kMaxPositions)
        return QUARTZ_ERR_SHAPE;
    PagedAppend a{};
    a.cache = {k_cache, v_cache, pages, page_stride, (int32_t)heads, (int32_t)d, shift_of(page_size),
               cache_type == QUARTZ_CACHE_E4M3, k_scale, v_scale, table, table_rows, table_stride,
               (int32_t)table_pages};
    const quartz_status st = cache_checks(a.cache, page_size, cache_type, tokens > 0);
    if (st != QUARTZ_OK || tokens == 0)
        return st;
    if (!k_bf16 || !v_bf16 || !positions || (!freqs && rot > 0))
        return QUARTZ_ERR_NULL;
    if (!aligned(k_bf16, 2) || !aligned(v_bf16, 2) || !aligned(positions, 4) || !aligned(sequences, 4) ||
        !aligned(freqs, 8))
        return QUARTZ_ERR_ALIGN;
    if (table_rows == 0 || table_pages == 0)
        return QUARTZ_OK;              // no token has a place
    a.k = static_cast<const uint16_t*>(k_bf16);
    a.v = static_cast<const uint16_t*>(v_bf16);
    a.tokens = tokens;
    a.k_token = k_token;
    a.k_head = k_head;
    a.v_token = v_token;
    a.v_head = v_head;
    a.positions = positions;
    a.sequences = sequences;
    a.freqs = freqs;
    a.rot = (int32_t)rot;
    a.interleaved = layout == QUARTZ_ROTARY_INTERLEAVED;
    a.magnitude = magnitude;
    return from_hip(launch_paged_append(a, stream));
}

// sizes of an attention call; `longest`: keys of a sequence at most
static quartz_status attention_checks(int64_t sequences, int64_t heads, int64_t kv_heads, int64_t d,
                                      int64_t page_size, int64_t table_pages, int64_t window, int64_t& longest)
{
    if ((d != 64 && d != 128 && d != 256) || page_size < 8 || page_size > 4096 ||
        (page_size & (page_size - 1)) != 0)
        return QUARTZ_ERR_UNSUPPORTED;
    if (sequences < 0 || sequences > kMaxBlocks512 || kv_heads <= 0 || heads < kv_heads || heads > kMaxK ||
        heads % kv_heads != 0 || table_pages < 0 || table_pages > kMaxPositions / page_size || window < 0 ||
        !product_ok(sequences, heads, kMaxBlocks512))
        return QUARTZ_ERR_SHAPE;
    longest = table_pages * page_size;
    if (window > 0 && window < longest)
        longest = window;
    return QUARTZ_OK;
}

size_t quartz_paged_attention_workspace_bytes(int64_t sequences, int64_t heads, int64_t kv_heads, int64_t d,
                                              int64_t page_size, int64_t table_pages, int64_t window)
{
    int64_t longest = 0;
    if (attention_checks(sequences, heads, kv_heads, d, page_size, table_pages, window, longest) != QUARTZ_OK ||
        sequences == 0)
        return 0;
    // enough for either cache type
    return paged_attention_bytes(d, std::max(paged_blocks(sequences, heads, kv_heads, d, false, longest),
                                             paged_blocks(sequences, heads, kv_heads, d, true, longest)));
}

quartz_status quartz_paged_attention(const void* q_bf16, void* o_bf16, int64_t sequences, int64_t heads,
                                     int64_t kv_heads, int64_t d, int64_t q_token, int64_t q_head,
                                     int64_t o_token, int64_t o_head, const void* k_cache, const void* v_cache,
                                     int32_t cache_type, float k_scale, float v_scale, int64_t pages,
                                     int64_t page_size, int64_t page_stride, const int32_t* table,
                                     int64_t table_pages, int64_t table_stride, const int32_t* lengths,
                                     float scale, int64_t window, void* workspace, size_t workspace_bytes,
                                     hipStream_t stream)
{
    // one factor for the scores, which fp32 has to hold with all its bits
    const double factor = (double)scale * (double)k_scale * 1.4426950408889634;
    if (!std::isfinite(scale) || (factor != 0.0 && !std::isnormal((float)factor)) || v_scale < kMinValueScale)
        return QUARTZ_ERR_UNSUPPORTED;
    int64_t longest = 0;
    quartz_status st = attention_checks(sequences, heads, kv_heads, d, page_size, table_pages, window, longest);
    if (st != QUARTZ_OK)
        return st;
    if (!stride_ok(q_token) || !stride_ok(q_head) || !stride_ok(o_token) || !stride_ok(o_head))
        return QUARTZ_ERR_SHAPE;
    PagedAttention a{};
    a.cache = {const_cast<void*>(k_cache), const_cast<void*>(v_cache), pages, page_stride, (int32_t)kv_heads,
               (int32_t)d, shift_of(page_size), cache_type == QUARTZ_CACHE_E4M3, k_scale, v_scale, table,
               sequences, table_stride, (int32_t)table_pages};
    st = cache_checks(a.cache, page_size, cache_type, sequences > 0);
    if (st != QUARTZ_OK || sequences == 0)
        return st;
    if (!q_bf16 || !o_bf16 || !lengths)
        return QUARTZ_ERR_NULL;
    if (!aligned16(q_bf16) || !aligned(o_bf16, 8) || !aligned(lengths, 4) || !aligned16(workspace) ||
        ((q_token | q_head) & 7) != 0 || ((o_token | o_head) & 3) != 0)
        return QUARTZ_ERR_ALIGN;
    const int blocks = paged_blocks(sequences, heads, kv_heads, d, a.cache.fp8, longest);
    const size_t need = paged_attention_bytes(d, blocks);
    if (need > 0 && (!workspace || workspace_bytes < need))
        return QUARTZ_ERR_WORKSPACE;
    a.q = static_cast<const uint16_t*>(q_bf16);
    a.o = static_cast<uint16_t*>(o_bf16);
    a.q_token = q_token;
    a.q_head = q_head;
    a.o_token = o_token;
    a.o_head = o_head;
    a.heads = (int32_t)heads;
    a.lengths = lengths;
    a.scale = (float)factor;
    a.window = (int32_t)(window < kMaxPositions ? window : kMaxPositions);
    a.shared = blocks;
    a.waves = paged_waves(sequences, heads, kv_heads, longest);
    a.workspace = static_cast<float*>(workspace);
    return from_hip(launch_paged_attention(a, stream));
}

}  // extern "C"
