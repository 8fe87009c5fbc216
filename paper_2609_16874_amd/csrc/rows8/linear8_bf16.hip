// linear8_bf16.hip -- the integer matrix product kernels with bf16_t outputs.
#include "k_linear8.hpp"

namespace cpe {
hipError_t launch_gemm8_bf16(const Gemm8Args &a, hipStream_t stream) { return launch_gemm8_type<bf16_t>(a, stream); }
}  // namespace cpe
