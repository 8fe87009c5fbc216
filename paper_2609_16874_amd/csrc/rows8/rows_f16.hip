// rows_f16.hip -- the row kernels for _Float16 rows.
#include "k_rows.hpp"

namespace cpe {
hipError_t launch_pack_f16(const RowsArgs &a, hipStream_t stream) { return launch_pack_type<_Float16>(a, stream); }
hipError_t launch_unpack_f16(const UnpackArgs &a, hipStream_t stream) { return launch_unpack_type<_Float16>(a, stream); }
hipError_t launch_rms_f16(const RowsArgs &a, hipStream_t stream) { return launch_rms_type<_Float16>(a, stream); }
hipError_t launch_rms_grad_f16(RmsGradArgs a, hipStream_t stream) { return launch_rms_grad_type<_Float16>(a, stream); }
}  // namespace cpe
