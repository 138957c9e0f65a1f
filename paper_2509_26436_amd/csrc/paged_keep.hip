// The accepted tokens of a drafted tree, moved to the places behind their sequence:
// place first + kept[i] to first + i, in keys and values.
//
// A thread moves 16 bytes of one head's rows, the same in every place, so that no
// two threads touch a byte.  kept[i] > i (an entry that is i stays, a smaller one
// is none), so a row's source is never a row that an earlier entry has written: all
// sources hold what they held before the call, however many are in flight.
// Bound by latency: entries, pages, rows one after the other.
#include <algorithm>

#include "quartz_internal.h"

namespace quartz {
namespace {

constexpr int kThreads = 256;
constexpr int kEntries = 256;                    // resolved at a time
constexpr int kFlight = 8;                       // rows on their way

__global__ __launch_bounds__(kThreads) void paged_keep_kernel(const PagedKeep a, uint32_t blocks)
{
    const PagedCacheView& c = a.cache;
    __shared__ int64_t from[kEntries], to[kEntries];          // bytes, -1: not moved
    const int bytes = c.fp8 ? 1 : 2, pieces = c.d * bytes / 16;
    const int64_t b = blockIdx.x / blocks;
    const uint32_t id = (uint32_t)(blockIdx.x % blocks) * kThreads + threadIdx.x;
    const uint32_t row = id / (uint32_t)pieces;               // head, keys or values
    const bool mine = row < 2u * (uint32_t)c.heads;
    const int64_t head = row >> 1, size = (int64_t)c.page_stride * bytes;
    uint8_t* at = static_cast<uint8_t*>(row & 1 ? c.v : c.k) + (head << c.page_shift) * c.d * bytes + 16 * (id % (uint32_t)pieces);
    const int64_t first = a.first[b];
    const int mask = (1 << c.page_shift) - 1;
    auto place = [&](int64_t position) -> int64_t {
        if (position < 0 || (position >> c.page_shift) >= c.table_pages)
            return -1;
        const int32_t page = c.table[b * c.table_stride + (position >> c.page_shift)];
        return page >= 0 && page < c.pages ? page * size + (int64_t)((int)position & mask) * c.d * bytes : -1;
    };
    for (int64_t i0 = 0; i0 < a.most; i0 += kEntries) {
        const int count = (int)min((int64_t)kEntries, a.most - i0);
        __syncthreads();
        if ((int)threadIdx.x < count) {
            const int64_t i = i0 + threadIdx.x, node = a.kept[b * a.kept_stride + i];
            int64_t source = -1, target = -1;
            if (node > i) {
                source = place(first + node);
                target = place(first + i);
            }
            from[threadIdx.x] = target < 0 ? -1 : source;
            to[threadIdx.x] = target;
        }
        __syncthreads();
        if (!mine)
            continue;
        for (int i = 0; i < count; i += kFlight) {
            uint4 w[kFlight];
#pragma unroll
            for (int j = 0; j < kFlight; ++j)
                if (i + j < count && from[i + j] >= 0)
                    w[j] = *reinterpret_cast<const uint4*>(at + from[i + j]);
#pragma unroll
            for (int j = 0; j < kFlight; ++j)
                if (i + j < count && from[i + j] >= 0)
                    *reinterpret_cast<uint4*>(at + to[i + j]) = w[j];
        }
    }
}

}  // namespace

hipError_t launch_paged_keep(const PagedKeep& a, hipStream_t stream)
{
    const int64_t pieces = a.cache.d * (a.cache.fp8 ? 1 : 2) / 16;
    const int64_t blocks = (2 * a.cache.heads * pieces + kThreads - 1) / kThreads;
    paged_keep_kernel<<<(uint32_t)(a.cache.sequences * blocks), kThreads, 0, stream>>>(a, (uint32_t)blocks);
    return hipGetLastError();
}

}  // namespace quartz
