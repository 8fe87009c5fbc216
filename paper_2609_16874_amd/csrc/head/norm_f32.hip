// norm_f32.hip -- the group norm kernels for float maps.
#include "k_norm.hpp"

namespace cpe {
hipError_t launch_norm_f32(const NormArgs &a, hipStream_t stream) { return launch_norm_type<float>(a, stream); }
}  // namespace cpe
