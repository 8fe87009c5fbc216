// linear8.hip -- C ABI of the integer matrix product (include/cpe_rows8.h):
// argument checks, the handle and its scratch.
#include "rows8/linear8.hpp"

#include <new>

#include "head/common.hpp"

using namespace cpe;

struct cpe_linear8 {
    int32_t max_rows, in, out;
    cpe_head_dtype dtype;
    cpe_activation act;
    int device;
    float *ws;
    size_t ws_bytes;
};

namespace {

bool check_matrix(const void *p, int64_t ld, int32_t width, size_t element)
{
    return p && aligned_to(p, element) && ld >= width && ld <= (int64_t)1 << 40;
}

}  // namespace

extern "C" {

cpe_status cpe_linear8_create(cpe_linear8 **out, int32_t max_rows, int32_t in_features, int32_t out_features,
                              cpe_head_dtype dtype, cpe_activation act)
{
    if (!out) return CPE_ERR_INVALID_ARG;
    *out = nullptr;
    if (max_rows < 1 || max_rows > 0x7fffffff - (1 << 23) + 1) return CPE_ERR_INVALID_ARG;
    if (in_features < 1 || in_features > 65536 || out_features < 1 || out_features > 65536)
        return CPE_ERR_INVALID_ARG;
    if (dtype != CPE_HEAD_F32 && dtype != CPE_HEAD_F16 && dtype != CPE_HEAD_BF16) return CPE_ERR_INVALID_ARG;
    if (act < CPE_ACT_NONE || act > CPE_ACT_GELU) return CPE_ERR_INVALID_ARG;
    cpe_linear8 *h = new (std::nothrow) cpe_linear8{};
    if (!h) return CPE_ERR_OUT_OF_MEMORY;
    h->max_rows = max_rows;
    h->in = in_features;
    h->out = out_features;
    h->dtype = dtype;
    h->act = act;
    if (hipGetDevice(&h->device) != hipSuccess) {
        delete h;
        return CPE_ERR_HIP;
    }
    // what the splits of some call of up to max_rows rows fill
    const int64_t splits = ceil_div(in_features, kStep8) / kLeastSteps8;
    const int64_t bytes = splits < 2 ? 0 : splits * max_rows * ceil_div(out_features, 4) * 16;
    h->ws_bytes = (size_t)(bytes < kSplitBytes ? bytes : kSplitBytes);
    void *p = nullptr;
    if (h->ws_bytes > 0 && hipMalloc(&p, h->ws_bytes) != hipSuccess) {
        (void)hipGetLastError();
        delete h;
        return CPE_ERR_OUT_OF_MEMORY;
    }
    h->ws = static_cast<float *>(p);
    *out = h;
    return CPE_OK;
}

cpe_status cpe_linear8_forward(cpe_linear8 *h, hipStream_t stream, int32_t rows, const int8_t *q, int64_t q_ld,
                               const float *scale, const int8_t *w, int64_t w_ld, const float *w_scale,
                               const float *bias, const void *residual, int64_t residual_ld, void *y, int64_t y_ld,
                               void *preact, int64_t preact_ld)
{
    if (!h || rows < 0 || rows > h->max_rows) return CPE_ERR_INVALID_ARG;
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess) return CPE_ERR_HIP;
    if (dev != h->device) return CPE_ERR_INVALID_ARG;
    if (!aligned_to(bias, 4) || !aligned_to(scale, 4) || !aligned_to(w_scale, 4)) return CPE_ERR_INVALID_ARG;
    if (rows == 0) return CPE_OK;
    const size_t element = element_size(h->dtype);
    if (!check_matrix(q, q_ld, h->in, 1) || !check_matrix(w, w_ld, h->in, 1) || !scale || !w_scale ||
        !check_matrix(y, y_ld, h->out, element))
        return CPE_ERR_INVALID_ARG;
    if (!apart(y, {q, scale, w, w_scale, bias})) return CPE_ERR_INVALID_ARG;     // (other workgroups still read them)
    if (residual && !check_matrix(residual, residual_ld, h->out, element)) return CPE_ERR_INVALID_ARG;
    if (residual == y && residual_ld != y_ld) return CPE_ERR_INVALID_ARG;
    if (preact && (!check_matrix(preact, preact_ld, h->out, element) ||
                   !apart(preact, {q, scale, w, w_scale, bias, residual, y})))
        return CPE_ERR_INVALID_ARG;
    Gemm8Args a{};
    a.a_scale = scale;
    a.b_scale = w_scale;
    a.g.a = q;
    a.g.lda = q_ld;
    a.g.b = w;
    a.g.ldb = w_ld;
    a.g.m = rows;
    a.g.n = h->out;
    a.g.k = h->in;
    a.g.out = y;
    a.g.ldo = y_ld;
    a.g.bias = bias;
    a.g.residual = residual;
    a.g.ldr = residual_ld;
    a.g.preact = preact;
    a.g.ldp = preact_ld;
    a.g.act = h->act;
    a.g.part = h->ws;
    a.g.part_bytes = (int64_t)h->ws_bytes;
    (void)hipGetLastError();
    const hipError_t e = h->dtype == CPE_HEAD_F32   ? launch_gemm8_f32(a, stream)
                         : h->dtype == CPE_HEAD_F16 ? launch_gemm8_f16(a, stream)
                                               : launch_gemm8_bf16(a, stream);
    return e == hipSuccess ? CPE_OK : CPE_ERR_HIP;
}

cpe_status cpe_linear8_destroy(cpe_linear8 *h)
{
    if (!h) return CPE_OK;
    const hipError_t e = hipFree(h->ws);
    delete h;
    return e == hipSuccess ? CPE_OK : CPE_ERR_HIP;
}

size_t cpe_linear8_workspace_bytes(const cpe_linear8 *h) { return h ? h->ws_bytes : 0; }

}  // extern "C"
