// linear_bf16.hip -- the matrix product kernels for bf16_t matrices.
#include "k_linear.hpp"

namespace cpe {
hipError_t launch_gemm_bf16(const GemmArgs &g, hipStream_t stream)
{
    return launch_gemm_type<bf16_t>(g, stream);
}
hipError_t launch_grad_bf16(const GradArgs &g, hipStream_t stream)
{
    return launch_grad_type<bf16_t>(g, stream);
}
hipError_t launch_narrow_grad_bf16(WholeGradArgs a, hipStream_t stream)
{
    return launch_narrow_grad_type<bf16_t>(a, stream);
}
hipError_t launch_rows_grad_bf16(const WholeGradArgs &a, hipStream_t stream)
{
    return launch_rows_grad_type<bf16_t>(a, stream);
}
}  // namespace cpe
