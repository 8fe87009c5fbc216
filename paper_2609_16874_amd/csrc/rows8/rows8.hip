// rows8.hip -- C ABI of packed rows and the RMS norm (include/cpe_rows8.h):
// argument checks, the handle and its scratch.
#include <cmath>
#include <new>

#include "head/common.hpp"
#include "rows8/rows.hpp"

using namespace cpe;

struct cpe_rms {
    int32_t max_rows, channels;
    cpe_head_dtype dtype;
    float eps;
    int device;
    float *ws;
    size_t ws_bytes;
};

namespace {

constexpr int32_t kMostRows = 0x7fffffff - (1 << 23) + 1;

bool is_dtype(cpe_head_dtype t) { return t == CPE_HEAD_F32 || t == CPE_HEAD_F16 || t == CPE_HEAD_BF16; }

bool check_rows(const void *p, int64_t ld, int32_t width, size_t element)
{
    return p && aligned_to(p, element) && ld >= width && ld <= (int64_t)1 << 40;
}

cpe_status check_call(const cpe_rms *h, int32_t rows, const float *gamma)
{
    if (!h || rows < 0 || rows > h->max_rows || !aligned_to(gamma, 4)) return CPE_ERR_INVALID_ARG;
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess) return CPE_ERR_HIP;
    return dev == h->device ? CPE_OK : CPE_ERR_INVALID_ARG;
}

// Whether `out` is an input that it may take the place of (the same rows), or
// none of the inputs.
bool in_place(const void *out, int64_t ld, const void *input, int64_t input_ld) { return out != input || ld == input_ld; }

template <typename Args>
cpe_status launch(cpe_head_dtype t, hipError_t (*f32)(Args, hipStream_t), hipError_t (*f16)(Args, hipStream_t),
                  hipError_t (*bf16)(Args, hipStream_t), Args a, hipStream_t stream)
{
    (void)hipGetLastError();
    const hipError_t e = t == CPE_HEAD_F32 ? f32(a, stream) : t == CPE_HEAD_F16 ? f16(a, stream) : bf16(a, stream);
    return e == hipSuccess ? CPE_OK : CPE_ERR_HIP;
}

}  // namespace

extern "C" {

cpe_status cpe_rows8_pack(hipStream_t stream, int32_t rows, int32_t width, cpe_head_dtype dtype, const void *x,
                          int64_t x_ld, int8_t *q, int64_t q_ld, float *scale)
{
    if (rows < 0 || rows > kMostRows || width < 1 || width > kRowsMaxWidth || !is_dtype(dtype))
        return CPE_ERR_INVALID_ARG;
    if (rows == 0) return CPE_OK;
    if (!check_rows(x, x_ld, width, element_size(dtype)) || !check_rows(q, q_ld, width, 1) || !scale ||
        !aligned_to(scale, 4) || !apart(q, {x}) || !apart(scale, {x, q}))
        return CPE_ERR_INVALID_ARG;
    RowsArgs a{};
    a.x = x;
    a.ldx = x_ld;
    a.q = q;
    a.ldq = q_ld;
    a.scale = scale;
    a.rows = rows;
    a.width = width;
    return launch<const RowsArgs &>(dtype, launch_pack_f32, launch_pack_f16, launch_pack_bf16, a, stream);
}

cpe_status cpe_rows8_unpack(hipStream_t stream, int32_t rows, int32_t width, const int8_t *q, int64_t q_ld,
                            const float *scale, cpe_head_dtype dtype, void *x, int64_t x_ld)
{
    if (rows < 0 || rows > kMostRows || width < 1 || width > kRowsMaxWidth || !is_dtype(dtype))
        return CPE_ERR_INVALID_ARG;
    if (rows == 0) return CPE_OK;
    if (!check_rows(x, x_ld, width, element_size(dtype)) || !check_rows(q, q_ld, width, 1) || !scale ||
        !aligned_to(scale, 4) || !apart(x, {q, scale}))
        return CPE_ERR_INVALID_ARG;
    UnpackArgs a{};
    a.q = q;
    a.ldq = q_ld;
    a.scale = scale;
    a.x = x;
    a.ldx = x_ld;
    a.rows = rows;
    a.width = width;
    return launch<const UnpackArgs &>(dtype, launch_unpack_f32, launch_unpack_f16, launch_unpack_bf16, a, stream);
}

cpe_status cpe_rms_create(cpe_rms **out, int32_t max_rows, int32_t channels, cpe_head_dtype dtype, float eps)
{
    if (!out) return CPE_ERR_INVALID_ARG;
    *out = nullptr;
    if (max_rows < 1 || max_rows > kMostRows || channels < 1 || channels > kRmsMaxChannels || !is_dtype(dtype))
        return CPE_ERR_INVALID_ARG;
    if (!std::isfinite(eps) || eps < kLeastScale) return CPE_ERR_INVALID_ARG;
    cpe_rms *h = new (std::nothrow) cpe_rms{};
    if (!h) return CPE_ERR_OUT_OF_MEMORY;
    h->max_rows = max_rows;
    h->channels = channels;
    h->dtype = dtype;
    h->eps = eps;
    if (hipGetDevice(&h->device) != hipSuccess) {
        delete h;
        return CPE_ERR_HIP;
    }
    const int64_t most = rms_most_blocks(channels);
    h->ws_bytes = (size_t)(max_rows < most ? max_rows : most) * channels * 4;
    void *p = nullptr;
    if (hipMalloc(&p, h->ws_bytes) != hipSuccess) {
        (void)hipGetLastError();
        delete h;
        return CPE_ERR_OUT_OF_MEMORY;
    }
    h->ws = static_cast<float *>(p);
    *out = h;
    return CPE_OK;
}

cpe_status cpe_rms_forward(cpe_rms *h, hipStream_t stream, int32_t rows, const void *x, int64_t x_ld,
                           const void *residual, int64_t residual_ld, const float *gamma, void *sum, int64_t sum_ld,
                           void *y, int64_t y_ld, int8_t *q, int64_t q_ld, float *scale, float *rstd)
{
    const cpe_status st = check_call(h, rows, gamma);
    if (st != CPE_OK) return st;
    if (!aligned_to(rstd, 4) || !aligned_to(scale, 4)) return CPE_ERR_INVALID_ARG;
    if (rows == 0) return CPE_OK;
    const size_t element = element_size(h->dtype);
    const int32_t C = h->channels;
    if (!check_rows(x, x_ld, C, element) || (residual && !check_rows(residual, residual_ld, C, element)))
        return CPE_ERR_INVALID_ARG;
    if (!sum && !y && !q) return CPE_ERR_INVALID_ARG;
    if (sum && (!check_rows(sum, sum_ld, C, element) || !in_place(sum, sum_ld, x, x_ld) ||
                !in_place(sum, sum_ld, residual, residual_ld)))
        return CPE_ERR_INVALID_ARG;
    if (y && (!check_rows(y, y_ld, C, element) || !in_place(y, y_ld, x, x_ld) ||
              !in_place(y, y_ld, residual, residual_ld)))
        return CPE_ERR_INVALID_ARG;
    if (!q != !scale || (q && !check_rows(q, q_ld, C, 1))) return CPE_ERR_INVALID_ARG;
    if (!apart(sum, {gamma}) || !apart(y, {gamma, sum}) || !apart(q, {x, residual, gamma, sum, y}) ||
        !apart(scale, {x, residual, gamma, sum, y, q}) || !apart(rstd, {x, residual, gamma, sum, y, q, scale}))
        return CPE_ERR_INVALID_ARG;
    RowsArgs a{};
    a.x = x;
    a.ldx = x_ld;
    a.residual = residual;
    a.ldr = residual_ld;
    a.gamma = gamma;
    a.sum = sum;
    a.lds = sum_ld;
    a.y = y;
    a.ldy = y_ld;
    a.q = q;
    a.ldq = q_ld;
    a.scale = scale;
    a.rstd = rstd;
    a.rows = rows;
    a.width = C;
    a.eps = h->eps;
    return launch<const RowsArgs &>(h->dtype, launch_rms_f32, launch_rms_f16, launch_rms_bf16, a, stream);
}

cpe_status cpe_rms_backward(cpe_rms *h, hipStream_t stream, int32_t rows, const void *h_rows, int64_t h_ld,
                            const float *h_scale, const void *dy, int64_t dy_ld, const float *gamma,
                            const float *rstd, const void *dsum, int64_t dsum_ld, void *dx, int64_t dx_ld,
                            float *dgamma)
{
    const cpe_status st = check_call(h, rows, gamma);
    if (st != CPE_OK) return st;
    if (rows > 0 && !dx && !dgamma) return CPE_ERR_INVALID_ARG;        // (a dx of no rows has no pointer)
    if (!aligned_to(dgamma, 4) || !aligned_to(rstd, 4) || !aligned_to(h_scale, 4)) return CPE_ERR_INVALID_ARG;
    const size_t element = element_size(h->dtype);
    const int32_t C = h->channels;
    if (rows > 0) {
        if (!check_rows(h_rows, h_ld, C, h_scale ? 1 : element) || !check_rows(dy, dy_ld, C, element) || !rstd)
            return CPE_ERR_INVALID_ARG;
        if (dsum && !check_rows(dsum, dsum_ld, C, element)) return CPE_ERR_INVALID_ARG;
        if (dx && (!check_rows(dx, dx_ld, C, element) || !in_place(dx, dx_ld, dy, dy_ld) ||
                   !in_place(dx, dx_ld, dsum, dsum_ld) || (dx == h_rows && (h_scale || dx_ld != h_ld))))
            return CPE_ERR_INVALID_ARG;
        if (!apart(dx, {h_scale, gamma, rstd}) || !apart(dgamma, {h_rows, h_scale, dy, gamma, rstd, dsum, dx}))
            return CPE_ERR_INVALID_ARG;
    } else if (!dgamma) {
        return CPE_OK;
    }
    RmsGradArgs a{};
    a.h = h_rows;
    a.ldh = h_ld;
    a.h_scale = rows > 0 ? h_scale : nullptr;
    a.dy = dy;
    a.ldd = dy_ld;
    a.gamma = gamma;
    a.rstd = rstd;
    a.dsum = dsum;
    a.lds = dsum_ld;
    a.dx = rows > 0 ? dx : nullptr;
    a.ldx = dx_ld;
    a.dgamma = dgamma;
    a.part = h->ws;
    a.rows = rows;
    a.width = C;
    return launch<RmsGradArgs>(h->dtype, launch_rms_grad_f32, launch_rms_grad_f16, launch_rms_grad_bf16, a, stream);
}

cpe_status cpe_rms_destroy(cpe_rms *h)
{
    if (!h) return CPE_OK;
    const hipError_t e = hipFree(h->ws);
    delete h;
    return e == hipSuccess ? CPE_OK : CPE_ERR_HIP;
}

size_t cpe_rms_workspace_bytes(const cpe_rms *h) { return h ? h->ws_bytes : 0; }

}  // extern "C"
