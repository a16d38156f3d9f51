// Routes in the order of their experts: a stable counting sort.
#pragma once

#include "cq_device.h"
#include "experts_internal.h"

namespace cq {

constexpr int kPlanThreads = 256, kPlanWaves = kPlanThreads / kWave;
constexpr int kPlanExperts = 1024;  // most

// Lanes of the wave that hold the same value as this one (of `bits` bits).
__device__ __forceinline__ uint64_t same_value(int v, int bits) {
    uint64_t same = __ballot(1);
    for (int b = 0; b < bits; ++b) {
        const uint64_t set = __ballot((v >> b) & 1);
        same &= (v >> b) & 1 ? set : ~set;
    }
    return same;
}

}  // namespace cq
