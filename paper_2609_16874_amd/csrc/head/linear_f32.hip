// linear_f32.hip -- the matrix product kernels for float matrices.
#include "k_linear.hpp"

namespace cpe {
hipError_t launch_gemm_f32(const GemmArgs &g, hipStream_t stream)
{
    return launch_gemm_type<float>(g, stream);
}
hipError_t launch_grad_f32(const GradArgs &g, hipStream_t stream)
{
    return launch_grad_type<float>(g, stream);
}
hipError_t launch_rows_grad_f32(const WholeGradArgs &a, hipStream_t stream)
{
    return launch_rows_grad_type<float>(a, stream);
}
}  // namespace cpe
