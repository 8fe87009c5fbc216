// rows_bf16.hip -- the row kernels for bf16_t rows.
#include "k_rows.hpp"

namespace cpe {
hipError_t launch_pack_bf16(const RowsArgs &a, hipStream_t stream) { return launch_pack_type<bf16_t>(a, stream); }
hipError_t launch_unpack_bf16(const UnpackArgs &a, hipStream_t stream) { return launch_unpack_type<bf16_t>(a, stream); }
hipError_t launch_rms_bf16(const RowsArgs &a, hipStream_t stream) { return launch_rms_type<bf16_t>(a, stream); }
hipError_t launch_rms_grad_bf16(RmsGradArgs a, hipStream_t stream) { return launch_rms_grad_type<bf16_t>(a, stream); }
}  // namespace cpe
