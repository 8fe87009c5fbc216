// norm_bf16.hip -- the group norm kernels for bf16_t maps.
#include "k_norm.hpp"

namespace cpe {
hipError_t launch_norm_bf16(const NormArgs &a, hipStream_t stream) { return launch_norm_type<bf16_t>(a, stream); }
}  // namespace cpe
