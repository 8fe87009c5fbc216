// rows.hpp -- arguments of the kernels that work row by row: packing, RMS
// norm and its gradient (private to the library).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "cpe_rows8.h"

namespace cpe {

constexpr int kRowsMaxWidth = 65536;
constexpr int kRmsMaxChannels = 16384;
constexpr int kRmsMaxBlocks = 1024;           // workgroups of the gradient, whose partial dgamma are joined
constexpr float kLeastScale = 1.17549435e-38f;        // 2^-126

// Workgroups that a gradient of C channels may have: their partial sums take
// 8 MiB at most, or those of one workgroup per CU.
inline int rms_most_blocks(int32_t channels)
{
    const int by_bytes = (1 << 21) / channels;
    return by_bytes > kRmsMaxBlocks ? kRmsMaxBlocks : by_bytes < 256 ? 256 : by_bytes;
}

// Workgroups of a gradient whose rows fill `want` of them: `lanes` threads take a
// row.  Up to eight turns of one workgroup of several rows at once are its alone,
// without the launch that joins dgamma: a call on 16 x 1024 in bf16 takes 6.4 us, on
// 32 x 1024 8.9, with the join 9.2; of a row in more than a wave 4 x 8192 10.0 against
// 9.2.  Without dgamma there is no join: 32 x 1024 in one workgroup 8.4, in eight 6.4.
inline int32_t rms_grad_blocks(int64_t want, int32_t channels, int lanes, bool dgamma)
{
    const int64_t most = rms_most_blocks(channels), alone = lanes <= 64 ? 8 : 1;
    return (int32_t)(dgamma && want <= alone ? 1 : want < most ? want : most);
}

// h = x (+ residual, rounded), y = h rstd gamma (norm), or y = x; any of
// h, y, y packed and rstd.
struct RowsArgs {
    const void *x, *residual;                 // residual may be null
    const float *gamma;                       // may be null
    void *sum, *y;                            // may be null
    int8_t *q;                                // may be null, with scale
    float *scale, *rstd;                      // rstd may be null
    int64_t ldx, ldr, lds, ldy, ldq;
    int32_t rows, width;
    float eps, inverse_width;
};

// x = q s; fold: q times the power of two of s alone (scale_parts).
struct UnpackArgs {
    const int8_t *q;
    const float *scale;
    void *x;
    int64_t ldq, ldx;
    int32_t rows, width;
    bool fold;
};

struct RmsGradArgs {
    const void *h;                            // of the type, or 8 bits where h_scale is given
    const float *h_scale;
    const void *dy, *dsum;                    // dsum may be null
    const float *gamma, *rstd;                // gamma may be null
    void *dx;                                 // may be null
    float *dgamma, *part;                     // may be null; scratch [blocks][width]
    int64_t ldh, ldd, lds, ldx;
    int32_t rows, width, blocks;
    float inverse_width;
};

#define CPE_ROWS_LAUNCHES(type)                                                  \
    hipError_t launch_pack_##type(const RowsArgs &a, hipStream_t stream);       \
    hipError_t launch_unpack_##type(const UnpackArgs &a, hipStream_t stream);   \
    hipError_t launch_rms_##type(const RowsArgs &a, hipStream_t stream);        \
    hipError_t launch_rms_grad_##type(RmsGradArgs a, hipStream_t stream);
CPE_ROWS_LAUNCHES(f32)
CPE_ROWS_LAUNCHES(f16)
CPE_ROWS_LAUNCHES(bf16)
#undef CPE_ROWS_LAUNCHES

}  // namespace cpe
