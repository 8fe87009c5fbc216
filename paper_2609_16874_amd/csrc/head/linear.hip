// linear.hip -- C ABI of the matrix product (include/cpe_head.h): argument
// checks, the handle and its scratch, and the products of the gradient.
#include "linear.hpp"

#include <new>

#include "common.hpp"
#include "rows8/rows.hpp"

using namespace cpe;

struct cpe_linear {
    int32_t max_rows, in, out;
    cpe_head_dtype dtype;
    cpe_activation act;
    int device;
    unsigned char *ws;
    size_t ws_bytes, split_bytes, sums_at, dz_at;
    int64_t dz_ld;
};

namespace {

bool check_matrix(const cpe_linear *h, const void *p, int64_t ld, int32_t width)
{
    return p && aligned_to(p, element_size(h->dtype)) && ld >= width && ld <= (int64_t)1 << 40;
}

cpe_status check_call(const cpe_linear *h, int32_t rows)
{
    if (!h || rows < 0 || rows > h->max_rows) return CPE_ERR_INVALID_ARG;
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess) return CPE_ERR_HIP;
    return dev == h->device ? CPE_OK : CPE_ERR_INVALID_ARG;
}

hipError_t launch_gemm(const cpe_linear *h, const GemmArgs &g, hipStream_t stream)
{
    return h->dtype == CPE_HEAD_F32   ? launch_gemm_f32(g, stream)
           : h->dtype == CPE_HEAD_F16 ? launch_gemm_f16(g, stream)
                                 : launch_gemm_bf16(g, stream);
}

hipError_t launch_grad(const cpe_linear *h, const GradArgs &g, hipStream_t stream)
{
    return h->dtype == CPE_HEAD_F32   ? launch_grad_f32(g, stream)
           : h->dtype == CPE_HEAD_F16 ? launch_grad_f16(g, stream)
                                 : launch_grad_bf16(g, stream);
}

hipError_t launch_unpack(const cpe_linear *h, const UnpackArgs &u, hipStream_t stream)
{
    return h->dtype == CPE_HEAD_F32   ? launch_unpack_f32(u, stream)
           : h->dtype == CPE_HEAD_F16 ? launch_unpack_f16(u, stream)
                                 : launch_unpack_bf16(u, stream);
}

// The gradient in one pass: whole vectors of features and a dw that eight
// waves' registers hold.  14.5 us against 24 .. 36 for the three products from
// 100 to 4000 rows (64 to 256 features), 110 against 200 at 409,600.
bool narrow_grad_fits(int32_t rows, int32_t n, int32_t k, cpe_head_dtype dtype)
{
    if (dtype == CPE_HEAD_F32 || rows < 1 || n % 8 != 0 || k % 8 != 0) return false;
    return (n <= 128 && k <= 256) || (n <= 64 && k <= 512);
}

// Few rows: two launches instead of four or five, 14 us against 20 on small
// products (calls as a program makes them).  Every workgroup forms the dz that
// it needs again and gathers w's columns, which costs more than that on larger
// ones: bf16 16 x 2048 to 4096 46 us against 33, 64 x 1024 to 1024 29 against
// 27; binary32, whose tiles waste more on rows that are not there, 23 x 3776 to
// 1152 28 against 39.
bool rows_grad_fits(int32_t rows, int32_t n, int32_t k, cpe_head_dtype dtype)
{
    const int64_t most = (int64_t)1 << (dtype == CPE_HEAD_F32 ? 27 : 25);
    return rows >= 1 && rows <= 64 && (int64_t)rows * n * k <= most;
}

// The most that the splits of a product of up to m x n outputs over up to k can
// fill: each split has least_steps or more, and all of them kSplitBytes or less.
int64_t most_split_bytes(size_t element, int64_t m, int64_t n, int64_t k)
{
    const int64_t splits = ceil_div(k, step_k(element)) / least_steps(element);
    if (splits < 2) return 0;
    const int64_t bytes = splits * m * ceil_div(n, 4) * 16;
    return bytes < kSplitBytes ? bytes : kSplitBytes;
}

// The handle's scratch: what some call of up to max_rows rows fills.
void plan_scratch(cpe_linear *h)
{
    const int64_t rows = h->max_rows, n = h->out, k = h->in;
    const size_t size = element_size(h->dtype);
    int64_t split = most_split_bytes(size, rows, n, k), sums = 0, dz = 0;
    // (a gradient that fits the few-row kernels at max_rows does at fewer, and needs none)
    if (!rows_grad_fits(h->max_rows, h->out, h->in, h->dtype)) {
        // partial sums of dbias: at most kSumBlocks workgroups, kSumUnroll rows or more
        // in each, and fewer workgroups above 2048 columns (kSumBlocks / slabs)
        const int64_t dealt = ceil_div(rows, kSumUnroll) * n, most = (int64_t)kSumBlocks * (n < 2048 ? n : 2048);
        sums = (dealt < most ? dealt : most) * 4;
        int64_t part;
        if (narrow_grad_fits(1, h->out, h->in, h->dtype)) {
            const int64_t strips = ceil_div(rows, kStripRows);
            part = (strips < kNarrowGradBlocks ? strips : kNarrowGradBlocks) * n * k * 4;
        } else {
            const int64_t dx = most_split_bytes(size, rows, k, n), dw = most_split_bytes(size, n, k, rows);
            part = dx > dw ? dx : dw;
            if (h->act != CPE_ACT_NONE) dz = rows * h->dz_ld * (int64_t)size;
        }
        if (part > split) split = part;
    }
    h->split_bytes = (size_t)split;
    h->sums_at = align256(h->split_bytes);
    h->dz_at = h->sums_at + align256((size_t)sums);
    h->ws_bytes = h->dz_at + align256((size_t)dz);
}

// x or preact of a gradient: of the dtype, or rows in 8 bits with their scales.
struct Kept {
    const void *p;
    int64_t ld;
    const float *scale;
    size_t element;
};

bool check_kept(const Kept &t, int32_t width)
{
    return t.p && aligned_to(t.p, t.element) && t.ld >= width && t.ld <= (int64_t)1 << 40;
}

cpe_status backward(cpe_linear *h, hipStream_t stream, int32_t rows, Kept x, const void *w, int64_t w_ld,
                    const void *dy, int64_t dy_ld, Kept preact, void *dx, int64_t dx_ld, void *dw, int64_t dw_ld,
                    float *dbias)
{
    const cpe_status st = check_call(h, rows);
    if (st != CPE_OK) return st;
    if (rows > 0 && !dx && !dw && !dbias) return CPE_ERR_INVALID_ARG;      // (a dx of no rows has no pointer)
    if (!aligned_to(dbias, 4)) return CPE_ERR_INVALID_ARG;
    const bool act = h->act != CPE_ACT_NONE;
    if (rows > 0) {
        if (!check_matrix(h, dy, dy_ld, h->out) || (act && !check_kept(preact, h->out))) return CPE_ERR_INVALID_ARG;
        if (dx && (!check_matrix(h, w, w_ld, h->in) || !check_matrix(h, dx, dx_ld, h->in)))
            return CPE_ERR_INVALID_ARG;
        if (dw && !check_kept(x, h->in)) return CPE_ERR_INVALID_ARG;
        if (!apart(dx, {dy, x.p, x.scale, w, preact.p, preact.scale}) ||
            !apart(dw, {dy, x.p, x.scale, w, preact.p, preact.scale, dx}) ||
            !apart(dbias, {dy, x.p, x.scale, w, preact.p, preact.scale, dx, dw}))
            return CPE_ERR_INVALID_ARG;
    }
    if (dw && !check_matrix(h, dw, dw_ld, h->in)) return CPE_ERR_INVALID_ARG;
    (void)hipGetLastError();
    {
        WholeGradArgs a{};
        a.x = x.p;
        a.ldx = x.ld;
        a.x_scale = x.scale;
        a.w = w;
        a.ldw = w_ld;
        a.dy = dy;
        a.ldd = dy_ld;
        a.preact = preact.p;
        a.ldp = preact.ld;
        a.z_scale = preact.scale;
        a.dx = dx;
        a.lddx = dx_ld;
        a.dw = dw;
        a.lddw = dw_ld;
        a.dbias = dbias;
        a.part = reinterpret_cast<float *>(h->ws);
        a.part_sums = reinterpret_cast<float *>(h->ws + h->sums_at);
        a.rows = rows;
        a.n = h->out;
        a.k = h->in;
        a.act = h->act;
        if (rows_grad_fits(rows, h->out, h->in, h->dtype)) {
            const hipError_t e = h->dtype == CPE_HEAD_F32   ? launch_rows_grad_f32(a, stream)
                                 : h->dtype == CPE_HEAD_F16 ? launch_rows_grad_f16(a, stream)
                                                       : launch_rows_grad_bf16(a, stream);
            return e == hipSuccess ? CPE_OK : CPE_ERR_HIP;
        }
        if (narrow_grad_fits(rows, h->out, h->in, h->dtype)) {
            const hipError_t e = h->dtype == CPE_HEAD_F16 ? launch_narrow_grad_f16(a, stream)
                                                     : launch_narrow_grad_bf16(a, stream);
            return e == hipSuccess ? CPE_OK : CPE_ERR_HIP;
        }
    }
    const bool fold = x.scale && folds(h->act, element_size(h->dtype));
    const void *dz = dy;
    int64_t dz_ld = dy_ld;
    if (dbias || (act && rows > 0)) {
        GradArgs a{};
        a.dy = dy;
        a.ldd = dy_ld;
        a.preact = preact.p;
        a.ldp = preact.ld;
        a.z_scale = act ? preact.scale : nullptr;
        a.x_scale = x.scale;
        if (act && (dx || dw)) {
            a.dz = h->ws + h->dz_at;
            a.ldz = h->dz_ld;
            dz = a.dz;
            dz_ld = a.ldz;
        }
        a.part = reinterpret_cast<float *>(h->ws + h->sums_at);
        a.sums = dbias;
        a.rows = rows;
        a.n = h->out;
        a.act = h->act;
        if (launch_grad(h, a, stream) != hipSuccess) return CPE_ERR_HIP;
    }
    // With many n x in 8 bits becomes x of the dtype in the place of dx, which is
    // written after dw then: dw's tiles would convert each byte once for every 128 n
    // (bf16 with GELU: 7744 x 1024 to 4096 189 us in all, 204 otherwise; to 2048 116
    // and 123; to 1024 85 and 84).  Many rows of few features pay for the unpacking
    // (50,000 x 512 to 2048 425 and 405, to 512 163 and 137), those of more gain below
    // the threshold as well (7744 x 4096 to 1536 254 and 282).
    const bool first_dw = dw && dx && rows > 0 && x.scale && h->out >= 2048;
    auto run_dx = [&]() {       // dx[r][k] = sum_n dz[r][n] w[n][k]
        GemmArgs g{};
        g.a = dz;
        g.lda = dz_ld;
        g.b = w;
        g.ldb = w_ld;
        g.b_cols = true;
        g.m = rows;
        g.n = h->in;
        g.k = h->out;
        g.out = dx;
        g.ldo = dx_ld;
        g.row_scale = fold ? x.scale : nullptr;
        g.part = reinterpret_cast<float *>(h->ws);
        g.part_bytes = (int64_t)h->split_bytes;
        return launch_gemm(h, g, stream) == hipSuccess;
    };
    if (first_dw) {
        UnpackArgs u{};
        u.q = static_cast<const int8_t *>(x.p);
        u.ldq = x.ld;
        u.scale = x.scale;
        u.x = dx;
        u.ldx = dx_ld;
        u.rows = rows;
        u.width = h->in;
        u.fold = fold;
        if (launch_unpack(h, u, stream) != hipSuccess) return CPE_ERR_HIP;
    } else if (dx && rows > 0 && !run_dx()) {
        return CPE_ERR_HIP;
    }
    if (dw) {                   // dw[n][k] = sum_r dz[r][n] x[r][k]
        GemmArgs g{};
        g.a = dz;
        g.lda = dz_ld;
        g.a_cols = true;
        g.b = first_dw ? dx : x.p;
        g.ldb = first_dw ? dx_ld : x.ld;
        g.b_cols = true;
        g.b_scale = first_dw ? nullptr : x.scale;
        g.fold = fold;
        g.m = h->out;
        g.n = h->in;
        g.k = rows;
        g.out = dw;
        g.ldo = dw_ld;
        g.part = reinterpret_cast<float *>(h->ws);
        g.part_bytes = (int64_t)h->split_bytes;
        if (launch_gemm(h, g, stream) != hipSuccess) return CPE_ERR_HIP;
    }
    if (first_dw && !run_dx()) return CPE_ERR_HIP;
    return CPE_OK;
}

}  // namespace

extern "C" {

cpe_status cpe_linear_create(cpe_linear **out, int32_t max_rows, int32_t in_features, int32_t out_features,
                             cpe_head_dtype dtype, cpe_activation act)
{
    if (!out) return CPE_ERR_INVALID_ARG;
    *out = nullptr;
    if (max_rows < 1 || max_rows > 0x7fffffff - (1 << 23) + 1) return CPE_ERR_INVALID_ARG;
    if (in_features < 1 || in_features > 65536 || out_features < 1 || out_features > 65536)
        return CPE_ERR_INVALID_ARG;
    if (dtype != CPE_HEAD_F32 && dtype != CPE_HEAD_F16 && dtype != CPE_HEAD_BF16) return CPE_ERR_INVALID_ARG;
    if (act < CPE_ACT_NONE || act > CPE_ACT_GELU) return CPE_ERR_INVALID_ARG;
    cpe_linear *h = new (std::nothrow) cpe_linear{};
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
    h->dz_ld = (out_features + 7) / 8 * 8;
    plan_scratch(h);
    void *p = nullptr;
    if (h->ws_bytes > 0 && hipMalloc(&p, h->ws_bytes) != hipSuccess) {
        (void)hipGetLastError();
        delete h;
        return CPE_ERR_OUT_OF_MEMORY;
    }
    h->ws = static_cast<unsigned char *>(p);
    *out = h;
    return CPE_OK;
}

cpe_status cpe_linear_forward(cpe_linear *h, hipStream_t stream, int32_t rows, const void *x, int64_t x_ld,
                              const void *w, int64_t w_ld, const float *bias, const void *residual,
                              int64_t residual_ld, void *y, int64_t y_ld, void *preact, int64_t preact_ld)
{
    const cpe_status st = check_call(h, rows);
    if (st != CPE_OK) return st;
    if (!aligned_to(bias, 4)) return CPE_ERR_INVALID_ARG;
    if (rows == 0) return CPE_OK;
    if (!check_matrix(h, x, x_ld, h->in) || !check_matrix(h, w, w_ld, h->in) || !check_matrix(h, y, y_ld, h->out))
        return CPE_ERR_INVALID_ARG;
    if (y == x || y == w) return CPE_ERR_INVALID_ARG;       // (other workgroups still read them)
    if (residual && !check_matrix(h, residual, residual_ld, h->out)) return CPE_ERR_INVALID_ARG;
    if (residual == y && residual_ld != y_ld) return CPE_ERR_INVALID_ARG;
    if (preact && (!check_matrix(h, preact, preact_ld, h->out) || preact == y || preact == residual || preact == x ||
                   preact == w))
        return CPE_ERR_INVALID_ARG;
    GemmArgs g{};
    g.a = x;
    g.lda = x_ld;
    g.b = w;
    g.ldb = w_ld;
    g.m = rows;
    g.n = h->out;
    g.k = h->in;
    g.out = y;
    g.ldo = y_ld;
    g.bias = bias;
    g.residual = residual;
    g.ldr = residual_ld;
    g.preact = preact;
    g.ldp = preact_ld;
    g.act = h->act;
    g.part = reinterpret_cast<float *>(h->ws);
    g.part_bytes = (int64_t)h->split_bytes;
    (void)hipGetLastError();
    return launch_gemm(h, g, stream) == hipSuccess ? CPE_OK : CPE_ERR_HIP;
}

cpe_status cpe_linear_backward(cpe_linear *h, hipStream_t stream, int32_t rows, const void *x, int64_t x_ld,
                               const void *w, int64_t w_ld, const void *dy, int64_t dy_ld, const void *preact,
                               int64_t preact_ld, void *dx, int64_t dx_ld, void *dw, int64_t dw_ld, float *dbias)
{
    const size_t element = h ? element_size(h->dtype) : 1;
    return backward(h, stream, rows, {x, x_ld, nullptr, element}, w, w_ld, dy, dy_ld,
                    {preact, preact_ld, nullptr, element}, dx, dx_ld, dw, dw_ld, dbias);
}

cpe_status cpe_linear_backward8(cpe_linear *h, hipStream_t stream, int32_t rows, const int8_t *q, int64_t q_ld,
                                const float *scale, const void *w, int64_t w_ld, const void *dy, int64_t dy_ld,
                                const int8_t *zq, int64_t zq_ld, const float *z_scale, void *dx, int64_t dx_ld,
                                void *dw, int64_t dw_ld, float *dbias)
{
    if (!h || !aligned_to(scale, 4) || !aligned_to(z_scale, 4)) return CPE_ERR_INVALID_ARG;
    if (rows > 0 && (!scale || (h->act != CPE_ACT_NONE && !z_scale))) return CPE_ERR_INVALID_ARG;
    return backward(h, stream, rows, {q, q_ld, scale, 1}, w, w_ld, dy, dy_ld, {zq, zq_ld, z_scale, 1}, dx, dx_ld, dw,
                    dw_ld, dbias);
}

cpe_status cpe_linear_destroy(cpe_linear *h)
{
    if (!h) return CPE_OK;
    const hipError_t e = hipFree(h->ws);
    delete h;
    return e == hipSuccess ? CPE_OK : CPE_ERR_HIP;
}

size_t cpe_linear_workspace_bytes(const cpe_linear *h) { return h ? h->ws_bytes : 0; }

}  // extern "C"
