// linear_f16.hip -- the matrix product kernels for _Float16 matrices.
#include "k_linear.hpp"

namespace cpe {
hipError_t launch_gemm_f16(const GemmArgs &g, hipStream_t stream)
{
    return launch_gemm_type<_Float16>(g, stream);
}
hipError_t launch_grad_f16(const GradArgs &g, hipStream_t stream)
{
    return launch_grad_type<_Float16>(g, stream);
}
hipError_t launch_narrow_grad_f16(WholeGradArgs a, hipStream_t stream)
{
    return launch_narrow_grad_type<_Float16>(a, stream);
}
hipError_t launch_rows_grad_f16(const WholeGradArgs &a, hipStream_t stream)
{
    return launch_rows_grad_type<_Float16>(a, stream);
}
}  // namespace cpe
