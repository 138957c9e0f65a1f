// The accepted tokens of a drafted tree, moved to the places behind their sequence:
// place first + kept[i] to first + i, in keys and values.
//
// A column is 16 bytes of one head's rows, the same in every place.  A block takes
// kColumns of a sequence's, and kEntries entries at a time: all their rows are read,
// then all are written.  kept[i] > i where anything moves, so a source is never a row
// that an earlier entry has written, and the entries of later turns find theirs as
// they were before the call.  Bound by the memory where there are many: 256 sequences of
// up to 128 entries (8 heads of 128 e4m3 channels, 34 MB each way) take 15 us, 4.5 TB/s.
// For that the eight rows of a thread have to be on their way together, without a branch
// between their loads and in registers: one after the other through scratch memory, as
// an array of uint4 lies, they take 31 us and twice the bytes.  A few entries of 64
// sequences 4.4, a launch.
#include <algorithm>

#include "quartz_internal.h"

namespace quartz {
namespace {

typedef uint32_t v4u __attribute__((ext_vector_type(4)));     // (an array of uint4 would lie in scratch memory)

constexpr int kThreads = 256;
constexpr int kColumns = 16;
constexpr int kTeams = kThreads / kColumns, kFlight = 8;
constexpr int kEntries = kTeams * kFlight;

__global__ __launch_bounds__(kThreads) void paged_keep_kernel(const PagedKeep a, uint32_t blocks)
{
    const PagedCacheView& c = a.cache;
    __shared__ int64_t from[kEntries], to[kEntries];          // bytes, -1: not moved
    const int bytes = c.fp8 ? 1 : 2, pieces = c.d * bytes / 16;
    const int64_t b = blockIdx.x / blocks;
    const uint32_t column = (uint32_t)(blockIdx.x % blocks) * kColumns + threadIdx.x % kColumns;
    const int team = (int)threadIdx.x / kColumns;
    const uint32_t row = column / (uint32_t)pieces;           // head, keys or values
    const bool mine = row < 2u * (uint32_t)c.heads;
    const int64_t head = mine ? row >> 1 : 0, size = (int64_t)c.page_stride * bytes;
    uint8_t* at = static_cast<uint8_t*>(row & 1 ? c.v : c.k) + (head << c.page_shift) * c.d * bytes + 16 * (column % (uint32_t)pieces);
    const int64_t first = a.first[b];
    const int mask = (1 << c.page_shift) - 1;
    auto place = [&](int64_t position) -> int64_t {
        if (position < 0 || (position >> c.page_shift) >= c.table_pages)
            return -1;
        const int32_t page = c.table[b * c.table_stride + (position >> c.page_shift)];
        return page >= 0 && page < c.pages ? page * size + (int64_t)((int)position & mask) * c.d * bytes : -1;
    };
    for (int64_t i0 = 0; i0 < a.most; i0 += kEntries) {
        __syncthreads();
        int64_t source = -1, target = -1;
        if (threadIdx.x < kEntries) {
            const int64_t i = i0 + threadIdx.x, node = i < a.most ? a.kept[b * a.kept_stride + i] : -1;
            if (node > i) {
                source = place(first + node);
                target = place(first + i);
            }
            if (source < 0)
                target = -1;
            from[threadIdx.x] = target < 0 ? 0 : source;
            to[threadIdx.x] = target;
        }
        if (!__syncthreads_or(target >= 0))
            continue;
        // There is a page: entries that do not move read its first row, which nothing uses,
        // so that no branch stands between the loads.
        v4u w[kFlight];
#pragma unroll
        for (int j = 0; j < kFlight; ++j)
            w[j] = *reinterpret_cast<const v4u*>(at + from[team + j * kTeams]);
        // Every row has been read before one is written: the barrier alone would not wait
        // for loads that are on their way.
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kFlight; ++j)
            if (mine && to[team + j * kTeams] >= 0)
                *reinterpret_cast<v4u*>(at + to[team + j * kTeams]) = w[j];
    }
}

}  // namespace

int64_t paged_keep_blocks(int64_t heads, int64_t d, bool fp8)
{
    const int64_t pieces = d * (fp8 ? 1 : 2) / 16;
    return (2 * heads * pieces + kColumns - 1) / kColumns;
}

hipError_t launch_paged_keep(const PagedKeep& a, hipStream_t stream)
{
    const int64_t blocks = paged_keep_blocks(a.cache.heads, a.cache.d, a.cache.fp8);
    paged_keep_kernel<<<(uint32_t)(a.cache.sequences * blocks), kThreads, 0, stream>>>(a, (uint32_t)blocks);
    return hipGetLastError();
}

}  // namespace quartz
