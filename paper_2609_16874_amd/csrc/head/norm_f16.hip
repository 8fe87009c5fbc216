// norm_f16.hip -- the group norm kernels for _Float16 maps.
#include "k_norm.hpp"

namespace cpe {
hipError_t launch_norm_f16(const NormArgs &a, hipStream_t stream) { return launch_norm_type<_Float16>(a, stream); }
}  // namespace cpe
