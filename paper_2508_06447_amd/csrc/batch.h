// Sizes of calls on a batch of requests (batch.hip, kv8.hip).
#pragma once
#include "slim_common.h"

namespace slim {

constexpr int kBatchRequestsMost = 4096;                 // their sums lie in LDS, twice

// n / d for 0 <= n < 2^31: (n M) >> (31 + s), 2^s >= d, M = floor(2^(31 + s) / d) + 1, so that 2^(31 + s) < M d <= 2^(31 + s) + 2^s.
struct Divide {
    uint32_t factor;
    int shift;
    explicit Divide(int d) {
        shift = 31;
        while ((1ll << (shift - 31)) < d) ++shift;
        factor = (uint32_t)((1ull << shift) / (unsigned)d + 1);
    }
    __device__ __forceinline__ int operator()(int n) const { return (int)(((unsigned long long)(unsigned)n * factor) >> shift); }
};

}  // namespace slim
