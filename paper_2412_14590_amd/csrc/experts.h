// Which tile of which expert a block takes, found on the device: how many rows an expert has is known there only.
#pragma once

#include "internal.h"

namespace mixllm {

// inclusive sum over the lanes of a wave (all active)
static __device__ inline int wave_scan(int v)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    return v;
}
static __device__ inline int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// first place and rows of expert e, clamped to the places there are
static __device__ inline void expert_rows(const ExpertsArgs &a, int e, int &first, int &count)
{
    first = min(max(a.offsets[e], 0), a.places);
    count = max(min(a.offsets[e + 1], a.places) - first, 0);
}

}  // namespace mixllm
