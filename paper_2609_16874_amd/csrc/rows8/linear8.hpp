// linear8.hpp -- arguments of the integer matrix product kernels (private to
// the library).
#pragma once

#include "cpe_rows8.h"
#include "head/linear.hpp"

namespace cpe {

constexpr int kStep8 = 128;                   // k of one LDS tile
constexpr int kLeastSteps8 = 8;               // of a split

// g.a and g.b are bytes, rows along k; a row's and a column's scale; the
// partial sums of a split product are whole numbers.
struct Gemm8Args {
    GemmArgs g;
    const float *a_scale, *b_scale;
};

hipError_t launch_gemm8_f32(const Gemm8Args &a, hipStream_t stream);
hipError_t launch_gemm8_f16(const Gemm8Args &a, hipStream_t stream);
hipError_t launch_gemm8_bf16(const Gemm8Args &a, hipStream_t stream);

}  // namespace cpe
