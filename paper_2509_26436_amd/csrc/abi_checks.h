// Argument checks that the C entry points share.
#pragma once

#include <hip/hip_runtime_api.h>
#include <stdint.h>

#include "quartz.h"

namespace quartz {

constexpr int64_t kMaxK = int64_t(1) << 20;       // at most 16384 groups per row
// rows x groups of one call (M x K/64 or N x K/64): 2^34 elements, 32 GiB of
// bf16 input; keeps every grid below 2^32 threads
constexpr int64_t kMaxRowGroups = int64_t(1) << 28;
// leading dimension of the activations and of the output (elements): 64 bf16
// rows of it stay below 2^31 bytes (one buffer range per wave of output rows)
constexpr int64_t kMaxLd = int64_t(1) << 24;

// sizes that every entry point accepts: rows >= 0, 0 <= K <= kMaxK, K % 64 == 0
// and rows * K / 64 <= kMaxRowGroups
inline bool size_ok(int64_t rows, int64_t K)
{
    if (rows < 0 || K < 0 || K % 64 != 0 || K > kMaxK)
        return false;
    return K == 0 || rows <= kMaxRowGroups / (K / 64);
}

inline bool aligned(const void* p, uintptr_t bytes)
{
    return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0;
}

inline bool aligned16(const void* p) { return aligned(p, 16); }

inline quartz_status from_hip(hipError_t e) { return e == hipSuccess ? QUARTZ_OK : QUARTZ_ERR_HIP; }

}  // namespace quartz
