// norm.hpp -- arguments of the group norm kernels (private to the library).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "cpe_head.h"

namespace cpe {

constexpr int kNormThreads = 256;
constexpr int kNormBlocks = 1024;      // workgroups of a pass over the map (or one per sample)
constexpr int kNormJoinWays = 32;      // partial results that are joined at a time
constexpr int kNormCounters = 64;      // per sample: of the join's teams and of the sample
constexpr int kNormMaxChannels = 8192;
constexpr int64_t kCacheBytes = (int64_t)128 << 20;      // read and written, half of what the last cache holds

struct NormArgs {
    const void *x, *dy;
    void *out;                          // y or dx (dx may be null)
    int64_t x_ld, x_sample, dy_ld, dy_sample, out_ld, out_sample;
    const float *gamma, *beta;          // may be null
    const int32_t *valid;               // may be null
    float *stats;                       // [samples][G][2]: written by the forward, read by the backward
    float *part;                        // scratch: [samples][blocks][G or C][2]
    float *group_part;                  // scratch (backward): [samples][blocks][G][2]
    float *group_sums;                  // scratch (backward): [samples][G][2]
    float *joined;                      // scratch: [samples][32][G][2], the first level of the join
    int32_t *counters;                  // [samples][kNormCounters], 0 between calls
    float *dgamma, *dbeta;              // may be null
    int32_t samples, pixels, channels, groups;
    int32_t blocks, chunk;              // workgroups per sample, rows that each takes at a time
    float eps;
    int act;
    bool backward;
};

hipError_t launch_norm_f32(const NormArgs &a, hipStream_t stream);
hipError_t launch_norm_f16(const NormArgs &a, hipStream_t stream);
hipError_t launch_norm_bf16(const NormArgs &a, hipStream_t stream);

}  // namespace cpe
