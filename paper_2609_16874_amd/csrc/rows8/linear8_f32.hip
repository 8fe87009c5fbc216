// linear8_f32.hip -- the integer matrix product kernels with float outputs.
#include "k_linear8.hpp"

namespace cpe {
hipError_t launch_gemm8_f32(const Gemm8Args &a, hipStream_t stream) { return launch_gemm8_type<float>(a, stream); }
}  // namespace cpe
