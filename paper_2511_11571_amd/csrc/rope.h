// Rotary positions: a call as the kernel takes it.
#pragma once
#include "common.h"

namespace moba {

constexpr int kRopeMaxPairs = 64;

struct RopeArgs {
    double freq[kRopeMaxPairs];         // turns per position of every pair
    const void* x[2];                   // Q, K
    void* y[2];
    int32_t xrows[2], yrows[2];         // rows that a slice takes in memory
    int32_t heads[2];                   // heads[1] = 0: no K
    const int32_t* pos;                 // [batch, N] or nullptr
    int64_t pos0;
    int32_t batch, N, D, rot, interleaved, dtype;
    float amp, sign;                    // sign of the angle: -1 for the gradient
};

hipError_t launch_rope(const RopeArgs& a, hipStream_t st);

}  // namespace moba
