// linear8_f16.hip -- the integer matrix product kernels with _Float16 outputs.
#include "k_linear8.hpp"

namespace cpe {
hipError_t launch_gemm8_f16(const Gemm8Args &a, hipStream_t stream) { return launch_gemm8_type<_Float16>(a, stream); }
}  // namespace cpe
