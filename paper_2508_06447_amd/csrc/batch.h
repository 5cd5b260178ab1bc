// Sizes of calls on a batch of requests (batch.hip, kv8.hip).
#pragma once
#include "slim_common.h"

namespace slim {

constexpr int kBatchRequestsMost = 4096;                 // their sums lie in LDS, twice

}  // namespace slim
