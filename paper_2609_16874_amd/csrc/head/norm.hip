// norm.hip -- C ABI of the group norm (include/cpe_head.h): argument checks,
// the handle and its scratch.
#include "norm.hpp"

#include <cmath>
#include <new>

#include "common.hpp"

using namespace cpe;

struct cpe_norm {
    int32_t max_samples, max_pixels, channels, groups;
    cpe_head_dtype dtype;
    cpe_activation act;
    float eps;
    int device;
    unsigned char *ws;
    size_t ws_bytes, group_part_at, group_sums_at, joined_at, counters_at, stats_at;
};

namespace {

// A map of `samples` x `pixels` rows of C elements: its strides keep rows and
// samples apart (either order of the two, as a permuted view has them).
bool strides_ok(int64_t ld, int64_t sample, int32_t samples, int32_t pixels, int32_t C)
{
    constexpr int64_t most = (int64_t)1 << 40;
    if (ld < C || ld > most) return false;
    if (samples <= 1) return true;
    if (sample < C || sample > most) return false;
    // (by division: pixels x ld may pass 64 bits)
    return (sample - C) / ld >= pixels - 1 || ld >= (int64_t)(samples - 1) * sample + C;
}

bool check_map(const cpe_norm *h, const void *p, int64_t ld, int64_t sample, int32_t samples, int32_t pixels)
{
    return p && aligned_to(p, element_size(h->dtype)) && strides_ok(ld, sample, samples, pixels, h->channels);
}

cpe_status check_call(const cpe_norm *h, int32_t samples, int32_t pixels, const float *gamma, const float *beta,
                      const int32_t *valid)
{
    if (!h || samples < 0 || samples > h->max_samples || pixels < 0 || pixels > h->max_pixels)
        return CPE_ERR_INVALID_ARG;
    if (!aligned_to(gamma, 4) || !aligned_to(beta, 4) || !aligned_to(valid, 4)) return CPE_ERR_INVALID_ARG;
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess) return CPE_ERR_HIP;
    return dev == h->device ? CPE_OK : CPE_ERR_INVALID_ARG;
}

cpe_status launch(const cpe_norm *h, const NormArgs &a, hipStream_t stream)
{
    (void)hipGetLastError();
    const hipError_t e = h->dtype == CPE_HEAD_F32   ? launch_norm_f32(a, stream)
                         : h->dtype == CPE_HEAD_F16 ? launch_norm_f16(a, stream)
                                               : launch_norm_bf16(a, stream);
    return e == hipSuccess ? CPE_OK : CPE_ERR_HIP;
}

NormArgs common_args(const cpe_norm *h, int32_t samples, int32_t pixels, const float *gamma, const float *beta,
                     const int32_t *valid)
{
    NormArgs a{};
    a.gamma = gamma;
    a.beta = beta;
    a.valid = valid;
    a.part = reinterpret_cast<float *>(h->ws);
    a.group_part = reinterpret_cast<float *>(h->ws + h->group_part_at);
    a.group_sums = reinterpret_cast<float *>(h->ws + h->group_sums_at);
    a.joined = reinterpret_cast<float *>(h->ws + h->joined_at);
    a.counters = reinterpret_cast<int32_t *>(h->ws + h->counters_at);
    a.samples = samples;
    a.pixels = pixels;
    a.channels = h->channels;
    a.groups = h->groups;
    a.eps = h->eps;
    a.act = h->act;
    return a;
}

}  // namespace

extern "C" {

cpe_status cpe_norm_create(cpe_norm **out, int32_t max_samples, int32_t max_pixels, int32_t channels,
                           int32_t groups, cpe_head_dtype dtype, cpe_activation act, float eps)
{
    if (!out) return CPE_ERR_INVALID_ARG;
    *out = nullptr;
    if (max_samples < 1 || max_samples > 65535 || max_pixels < 1 || max_pixels > 0x7fffffff - (1 << 23) + 1)
        return CPE_ERR_INVALID_ARG;
    if (channels < 1 || channels > kNormMaxChannels || groups < 1 || channels % groups != 0)
        return CPE_ERR_INVALID_ARG;
    if (dtype != CPE_HEAD_F32 && dtype != CPE_HEAD_F16 && dtype != CPE_HEAD_BF16) return CPE_ERR_INVALID_ARG;
    if (act < CPE_ACT_NONE || act > CPE_ACT_GELU) return CPE_ERR_INVALID_ARG;
    if (!std::isfinite(eps) || eps <= 0.0f) return CPE_ERR_INVALID_ARG;
    cpe_norm *h = new (std::nothrow) cpe_norm{};
    if (!h) return CPE_ERR_OUT_OF_MEMORY;
    h->max_samples = max_samples;
    h->max_pixels = max_pixels;
    h->channels = channels;
    h->groups = groups;
    h->dtype = dtype;
    h->act = act;
    h->eps = eps;
    if (hipGetDevice(&h->device) != hipSuccess) {
        delete h;
        return CPE_ERR_HIP;
    }
    const size_t blocks = max_samples > kNormBlocks ? max_samples : kNormBlocks;
    h->group_part_at = align256(blocks * channels * 8);
    h->group_sums_at = h->group_part_at + align256(blocks * groups * 8);
    h->stats_at = h->group_sums_at + align256((size_t)max_samples * groups * 8);
    h->joined_at = h->stats_at + align256((size_t)max_samples * groups * 8);
    // (only samples of more than kJoinWays workgroups join in two levels)
    const size_t large = max_samples < kNormBlocks / kNormJoinWays ? max_samples : kNormBlocks / kNormJoinWays;
    h->counters_at = h->joined_at + align256(large * kNormJoinWays * groups * 8);
    h->ws_bytes = h->counters_at + align256((size_t)max_samples * kNormCounters * 4);
    void *p = nullptr;
    if (hipMalloc(&p, h->ws_bytes) != hipSuccess) {
        (void)hipGetLastError();
        delete h;
        return CPE_ERR_OUT_OF_MEMORY;
    }
    if (hipMemset(static_cast<unsigned char *>(p) + h->counters_at, 0, h->ws_bytes - h->counters_at) != hipSuccess ||
        hipDeviceSynchronize() != hipSuccess) {
        (void)hipGetLastError();
        (void)hipFree(p);
        delete h;
        return CPE_ERR_HIP;
    }
    h->ws = static_cast<unsigned char *>(p);
    *out = h;
    return CPE_OK;
}

cpe_status cpe_norm_forward(cpe_norm *h, hipStream_t stream, int32_t samples, int32_t pixels, const void *x,
                            int64_t x_ld, int64_t x_sample, const float *gamma, const float *beta,
                            const int32_t *valid, void *y, int64_t y_ld, int64_t y_sample, float *stats)
{
    const cpe_status st = check_call(h, samples, pixels, gamma, beta, valid);
    if (st != CPE_OK) return st;
    if (!aligned_to(stats, 8)) return CPE_ERR_INVALID_ARG;
    if (samples == 0 || pixels == 0) return CPE_OK;
    if (!check_map(h, x, x_ld, x_sample, samples, pixels) || !check_map(h, y, y_ld, y_sample, samples, pixels))
        return CPE_ERR_INVALID_ARG;
    if (x == y && (x_ld != y_ld || (samples > 1 && x_sample != y_sample))) return CPE_ERR_INVALID_ARG;
    NormArgs a = common_args(h, samples, pixels, gamma, beta, valid);
    a.x = x;
    a.x_ld = x_ld;
    a.x_sample = x_sample;
    a.out = y;
    a.out_ld = y_ld;
    a.out_sample = y_sample;
    a.stats = stats ? stats : reinterpret_cast<float *>(h->ws + h->stats_at);
    return launch(h, a, stream);
}

cpe_status cpe_norm_backward(cpe_norm *h, hipStream_t stream, int32_t samples, int32_t pixels, const void *x,
                             int64_t x_ld, int64_t x_sample, const void *dy, int64_t dy_ld, int64_t dy_sample,
                             const float *gamma, const float *beta, const int32_t *valid, const float *stats,
                             void *dx, int64_t dx_ld, int64_t dx_sample, float *dgamma, float *dbeta)
{
    const cpe_status st = check_call(h, samples, pixels, gamma, beta, valid);
    if (st != CPE_OK) return st;
    // (a dx of nothing has no pointer)
    if (samples > 0 && pixels > 0 && !dx && !dgamma && !dbeta) return CPE_ERR_INVALID_ARG;
    if (!aligned_to(dgamma, 4) || !aligned_to(dbeta, 4) || !aligned_to(stats, 8)) return CPE_ERR_INVALID_ARG;
    NormArgs a = common_args(h, samples, pixels, gamma, beta, valid);
    a.backward = true;
    a.dgamma = dgamma;
    a.dbeta = dbeta;
    if (samples == 0 || pixels == 0) {
        if (!dgamma && !dbeta) return CPE_OK;
        a.samples = 0;      // the sums over no samples
        return launch(h, a, stream);
    }
    if (!stats || !check_map(h, x, x_ld, x_sample, samples, pixels) ||
        !check_map(h, dy, dy_ld, dy_sample, samples, pixels))
        return CPE_ERR_INVALID_ARG;
    if (dx && !check_map(h, dx, dx_ld, dx_sample, samples, pixels)) return CPE_ERR_INVALID_ARG;
    if (dx == x && (x_ld != dx_ld || (samples > 1 && x_sample != dx_sample))) return CPE_ERR_INVALID_ARG;
    if (dx == dy && (dy_ld != dx_ld || (samples > 1 && dy_sample != dx_sample))) return CPE_ERR_INVALID_ARG;
    a.x = x;
    a.x_ld = x_ld;
    a.x_sample = x_sample;
    a.dy = dy;
    a.dy_ld = dy_ld;
    a.dy_sample = dy_sample;
    a.out = dx;
    a.out_ld = dx_ld;
    a.out_sample = dx_sample;
    a.stats = const_cast<float *>(stats);
    return launch(h, a, stream);
}

cpe_status cpe_norm_destroy(cpe_norm *h)
{
    if (!h) return CPE_OK;
    const hipError_t e = hipFree(h->ws);
    delete h;
    return e == hipSuccess ? CPE_OK : CPE_ERR_HIP;
}

size_t cpe_norm_workspace_bytes(const cpe_norm *h) { return h ? h->ws_bytes : 0; }

}  // extern "C"
