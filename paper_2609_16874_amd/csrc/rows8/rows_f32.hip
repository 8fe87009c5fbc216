// rows_f32.hip -- the row kernels for float rows.
#include "k_rows.hpp"

namespace cpe {
hipError_t launch_pack_f32(const RowsArgs &a, hipStream_t stream) { return launch_pack_type<float>(a, stream); }
hipError_t launch_unpack_f32(const UnpackArgs &a, hipStream_t stream) { return launch_unpack_type<float>(a, stream); }
hipError_t launch_rms_f32(const RowsArgs &a, hipStream_t stream) { return launch_rms_type<float>(a, stream); }
hipError_t launch_rms_grad_f32(RmsGradArgs a, hipStream_t stream) { return launch_rms_grad_type<float>(a, stream); }
}  // namespace cpe
