// k_norm.hpp -- group norm with an activation over channels-last maps, and
// its gradient (private to the library; included once per element type).
//
// Threads.  A thread owns V neighbouring channels (up to 16 bytes of a row)
// and walks down the rows, so its channel constants stay in registers: a
// workgroup of 256 covers R = 256 / (C / V) rows at a time, whole rows and so
// whole cache lines, or one row in several column steps where C / V > 256.
//
// Statistics.  Each thread sums (x - s) and (x - s)^2 with s its first value
// of the channel, so a mean far from zero cancels nothing; threads, then
// workgroups, are merged as (count, mean, sum of squares about the mean),
//   mean = sum n_i mean_i / n,  M2 = sum M2_i + n_i (mean_i - mean)^2,
// in a fixed order.
#pragma once

#include "head_common.hpp"
#include "norm.hpp"

#pragma clang fp contract(fast)

namespace cpe {
namespace {

constexpr int kNormUnroll = 4;      // rows of a thread in flight

// The rows of one workgroup: range [r0, r1) of sample b's pb pixels.
struct RowRange {
    int b, i, pb, r0, r1;
};
__device__ __forceinline__ int valid_pixels(const NormArgs &a, int b)
{
    if (!a.valid) return a.pixels;
    const int v = a.valid[b];
    return v < 0 ? 0 : v > a.pixels ? a.pixels : v;
}
__device__ __forceinline__ int rows_per_block(int rows, int blocks) { return (rows + blocks - 1) / blocks; }
__device__ __forceinline__ RowRange row_range(const NormArgs &a)
{
    RowRange r;
    r.b = blockIdx.x / a.blocks;
    r.i = blockIdx.x - r.b * a.blocks;
    r.pb = valid_pixels(a, r.b);
    const int64_t step = rows_per_block(r.pb, a.blocks), lo = step * r.i, hi = lo + step;
    r.r0 = lo < r.pb ? (int)lo : r.pb;
    r.r1 = hi < r.pb ? (int)hi : r.pb;
    return r;
}

// c / cpg for c < 8192 through the reciprocal: c + 1/2 is at least 1/2 from a
// multiple of cpg, and the product's error stays under 1e-3 / cpg.
__device__ __forceinline__ int group_of(int c, float inv_cpg) { return (int)(((float)c + 0.5f) * inv_cpg); }

// A vector's channels: their groups' statistics, and gamma and beta.
template <int V>
struct Channels {
    float mean[V], rstd[V], gamma[V], beta[V];
    __device__ __forceinline__ Channels(const NormArgs &a, int b, int col)
    {
        const int cpg = a.channels / a.groups;
        const float inv_cpg = 1.0f / (float)cpg;
        const float2 *stats = reinterpret_cast<const float2 *>(a.stats) + (int64_t)b * a.groups;
        if (cpg % V == 0) {         // all in one group
            const float2 st = stats[group_of(col * V, inv_cpg)];
#pragma unroll
            for (int v = 0; v < V; v++) {
                mean[v] = st.x;
                rstd[v] = st.y;
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; v++) {
                const float2 st = stats[group_of(col * V + v, inv_cpg)];
                mean[v] = st.x;
                rstd[v] = st.y;
            }
        }
        Vec<float, V> g, s;
#pragma unroll
        for (int v = 0; v < V; v++) {
            g.v[v] = 1.0f;
            s.v[v] = 0.0f;
        }
        if (a.gamma) g = load_vec<float, V>(a.gamma + col * V);
        if (a.beta) s = load_vec<float, V>(a.beta + col * V);
#pragma unroll
        for (int v = 0; v < V; v++) {
            gamma[v] = g.v[v];
            beta[v] = s.v[v];
        }
    }
};

// How a workgroup covers a row of C channels.
template <int V>
struct Columns {
    int per_row, rows, col, row;     // vectors in a row, rows at a time, this thread's first vector and row
    __device__ __forceinline__ explicit Columns(int channels)
    {
        per_row = channels / V;
        rows = per_row >= kNormThreads ? 1 : kNormThreads / per_row;
        if (rows == 1) {
            row = 0;
            col = threadIdx.x;
        } else {
            row = threadIdx.x / per_row;
            col = threadIdx.x - row * per_row;
            if (row >= rows) col = per_row;        // left over: no column
        }
    }
};

// Lanes that share one group's sum: a power of two, at most a wave.
__device__ __forceinline__ int lanes_per_group(int groups)
{
    int n = 64;
    while (n > 1 && n * groups > kNormThreads) n >>= 1;
    return n;
}
__device__ __forceinline__ float sum_lanes(float v, int lanes)
{
    for (int o = lanes >> 1; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
__device__ __forceinline__ double sum_lanes(double v, int lanes)
{
    for (int o = lanes >> 1; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// Partial statistics: part[b][block][g] = (mean, M2) over the block's rows.
template <typename T, int V>
__global__ __launch_bounds__(kNormThreads) void k_norm_stats(NormArgs a)
{
    extern __shared__ float lds[];      // [rows][C] means, then [rows][C] M2
    const RowRange rr = row_range(a);
    const Columns<V> cols(a.channels);
    const int C = a.channels, n_rows = rr.r1 - rr.r0;
    float *lmean = lds, *lm2 = lds + cols.rows * C;
    const T *x = static_cast<const T *>(a.x) + rr.b * a.x_sample;
    for (int col = cols.col; col < cols.per_row; col += kNormThreads) {
        const T *p = x + col * V + (rr.r0 + cols.row) * a.x_ld;
        const int64_t step = cols.rows * a.x_ld;
        int n = n_rows > cols.row ? (n_rows - cols.row + cols.rows - 1) / cols.rows : 0;
        const float inv = 1.0f / (float)(n > 0 ? n : 1);
        float shift[V], s1[V], s2[V];
#pragma unroll
        for (int v = 0; v < V; v++) shift[v] = s1[v] = s2[v] = 0.0f;
        if (n > 0) {
            const Vec<T, V> f = load_vec<T, V>(p);
#pragma unroll
            for (int v = 0; v < V; v++) shift[v] = (float)f.v[v];
        }
        auto add = [&](const Vec<T, V> &f) {
#pragma unroll
            for (int v = 0; v < V; v++) {
                const float d = (float)f.v[v] - shift[v];
                s1[v] += d;
                s2[v] = fmaf(d, d, s2[v]);
            }
        };
        for (; n >= kNormUnroll; n -= kNormUnroll) {
            Vec<T, V> f[kNormUnroll];
#pragma unroll
            for (int u = 0; u < kNormUnroll; u++) f[u] = load_vec<T, V>(p + u * step);
#pragma unroll
            for (int u = 0; u < kNormUnroll; u++) add(f[u]);
            p += kNormUnroll * step;
        }
        for (; n > 0; n--, p += step) add(load_vec<T, V>(p));
#pragma unroll
        for (int v = 0; v < V; v++) {
            const int at = cols.row * C + col * V + v;
            lmean[at] = fmaf(s1[v], inv, shift[v]);
            lm2[at] = s2[v] - s1[v] * s1[v] * inv;
        }
    }
    __syncthreads();
    const int lanes = lanes_per_group(a.groups), cpg = C / a.groups, entries = cols.rows * cpg;
    const int lane = threadIdx.x & (lanes - 1);
    const float inv_n = 1.0f / ((float)(n_rows > 0 ? n_rows : 1) * (float)cpg);
    float2 *part = reinterpret_cast<float2 *>(a.part) + (int64_t)blockIdx.x * a.groups;
    auto count = [&](int row) { return (float)(n_rows > row ? (n_rows - row + cols.rows - 1) / cols.rows : 0); };
    for (int g0 = 0; g0 < a.groups; g0 += kNormThreads / lanes) {
        const int g = g0 + threadIdx.x / lanes;
        const bool on = g < a.groups;
        float mean = 0.0f, m2 = 0.0f;
        for (int e = lane; on && e < entries; e += lanes) {
            const int row = e / cpg, at = row * C + g * cpg + (e - row * cpg);
            mean += count(row) * lmean[at];
        }
        mean = sum_lanes(mean, lanes) * inv_n;
        for (int e = lane; on && e < entries; e += lanes) {
            const int row = e / cpg, at = row * C + g * cpg + (e - row * cpg);
            const float d = lmean[at] - mean, n = count(row);
            if (n > 0.0f) m2 += fmaf(n * d, d, lm2[at]);
        }
        m2 = sum_lanes(m2, lanes);
        if (on && lane == 0) part[g] = make_float2(mean, m2);
    }
}

// stats[b][g] = (mean, rstd) from the workgroups' partials: one workgroup per
// group, its threads' at most kMergeEach partials in flight together.
constexpr int kMergeEach = 8;
template <int THREADS>
__global__ __launch_bounds__(THREADS) void k_norm_merge(NormArgs a)
{
    __shared__ double lds[2][THREADS / 64];
    const int b = blockIdx.x / a.groups, g = blockIdx.x - b * a.groups;
    const int pb = valid_pixels(a, b), cpg = a.channels / a.groups;
    const int64_t step = rows_per_block(pb, a.blocks);
    const float2 *part = reinterpret_cast<const float2 *>(a.part) + (int64_t)b * a.blocks * a.groups + g;
    float2 p[kMergeEach];
    double rows[kMergeEach];
#pragma unroll
    for (int e = 0; e < kMergeEach; e++) {
        const int i = threadIdx.x + e * THREADS;
        const int64_t left = pb - step * i;
        const bool on = i < a.blocks && left > 0;
        p[e] = on ? part[(int64_t)i * a.groups] : make_float2(0.0f, 0.0f);
        rows[e] = (double)(!on ? 0 : left < step ? left : step);
    }
    auto total = [&](double v, int slot) {
        v = sum_lanes(v, 64);
        if constexpr (THREADS == 64) return v;
        if ((threadIdx.x & 63) == 0) lds[slot][threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0;
        for (int w = 0; w < THREADS / 64; w++) v += lds[slot][w];
        return v;
    };
    const double n = pb > 0 ? pb : 1;
    double mean = 0.0, m2 = 0.0;
#pragma unroll
    for (int e = 0; e < kMergeEach; e++) mean += rows[e] * (double)p[e].x;
    mean = total(mean, 0) / n;
#pragma unroll
    for (int e = 0; e < kMergeEach; e++) {
        const double d = (double)p[e].x - mean;
        if (rows[e] > 0.0) m2 += (double)p[e].y + rows[e] * cpg * d * d;
    }
    m2 = total(m2, 1);
    if (threadIdx.x == 0) {
        const double var = m2 > 0.0 || m2 != m2 ? m2 / (n * cpg) : 0.0;
        reinterpret_cast<float2 *>(a.stats)[blockIdx.x] = make_float2((float)mean, (float)(1.0 / sqrt(var + a.eps)));
    }
}
static_assert(kNormBlocks <= 256 * kMergeEach, "every partial of a group has a place");

// y = act((x - mean) (rstd gamma) + beta); pixels from the sample's count on
// are set to 0.
template <typename T, int V, int ACT>
__global__ __launch_bounds__(kNormThreads) void k_norm_apply(NormArgs a)
{
    const int b = blockIdx.x / a.blocks, i = blockIdx.x - b * a.blocks;
    const Columns<V> cols(a.channels);
    const int pb = valid_pixels(a, b);
    const int64_t span = rows_per_block(a.pixels, a.blocks), lo = span * i;
    const int64_t hi = lo + span < a.pixels ? lo + span : a.pixels;
    const T *x = static_cast<const T *>(a.x) + b * a.x_sample;
    T *y = static_cast<T *>(a.out) + b * a.out_sample;
    for (int col = cols.col; col < cols.per_row; col += kNormThreads) {
        const Channels<V> ch(a, b, col);
        float scale[V];
#pragma unroll
        for (int v = 0; v < V; v++) scale[v] = ch.rstd[v] * ch.gamma[v];
        auto one = [&](const Vec<T, V> &f) {
            Vec<T, V> o;
#pragma unroll
            for (int v = 0; v < V; v++)
                o.v[v] = (T)activate<ACT>(fmaf((float)f.v[v] - ch.mean[v], scale[v], ch.beta[v]));
            return o;
        };
        const int64_t xs = cols.rows * a.x_ld, ys = cols.rows * a.out_ld;
        int64_t r = lo + cols.row;
        const T *px = x + col * V + r * a.x_ld;
        T *py = y + col * V + r * a.out_ld;
        const int64_t end = hi < pb ? hi : pb;
        for (; r + (kNormUnroll - 1) * cols.rows < end; r += kNormUnroll * cols.rows) {
            Vec<T, V> f[kNormUnroll];
#pragma unroll
            for (int u = 0; u < kNormUnroll; u++) f[u] = load_vec<T, V>(px + u * xs);
#pragma unroll
            for (int u = 0; u < kNormUnroll; u++) store_vec<T, V>(py + u * ys, one(f[u]));
            px += kNormUnroll * xs;
            py += kNormUnroll * ys;
        }
        for (; r < end; r += cols.rows, px += xs, py += ys) store_vec<T, V>(py, one(load_vec<T, V>(px)));
        Vec<T, V> zero;
#pragma unroll
        for (int v = 0; v < V; v++) zero.v[v] = (T)0.0f;
        for (; r < hi; r += cols.rows, py += ys) store_vec<T, V>(py, zero);
    }
}

// part[b][block][c] = (sum du, sum du xh) over the block's rows.
template <typename T, int V, int ACT>
__global__ __launch_bounds__(kNormThreads) void k_norm_grad_sums(NormArgs a)
{
    extern __shared__ float lds[];      // [rows][C] sums of du, then of du xh
    const RowRange rr = row_range(a);
    const Columns<V> cols(a.channels);
    const int C = a.channels, n_rows = rr.r1 - rr.r0;
    float *l1 = lds, *l2 = lds + cols.rows * C;
    for (int col = cols.col; col < cols.per_row; col += kNormThreads) {
        const Channels<V> ch(a, rr.b, col);
        float scale[V];
#pragma unroll
        for (int v = 0; v < V; v++) scale[v] = ch.rstd[v] * ch.gamma[v];
        const int64_t first = rr.r0 + cols.row;
        const T *px = static_cast<const T *>(a.x) + rr.b * a.x_sample + col * V + first * a.x_ld;
        const T *pd = static_cast<const T *>(a.dy) + rr.b * a.dy_sample + col * V + first * a.dy_ld;
        const int64_t xs = cols.rows * a.x_ld, ds = cols.rows * a.dy_ld;
        int n = n_rows > cols.row ? (n_rows - cols.row + cols.rows - 1) / cols.rows : 0;
        float s1[V], s2[V];
#pragma unroll
        for (int v = 0; v < V; v++) s1[v] = s2[v] = 0.0f;
        auto add = [&](const Vec<T, V> &fx, const Vec<T, V> &fd) {
#pragma unroll
            for (int v = 0; v < V; v++) {
                const float d = (float)fx.v[v] - ch.mean[v];
                const float du = (float)fd.v[v] * activate_grad<ACT>(fmaf(d, scale[v], ch.beta[v]));
                s1[v] += du;
                s2[v] = fmaf(du, d, s2[v]);
            }
        };
        for (; n >= kNormUnroll; n -= kNormUnroll) {
            Vec<T, V> fx[kNormUnroll], fd[kNormUnroll];
#pragma unroll
            for (int u = 0; u < kNormUnroll; u++) {
                fx[u] = load_vec<T, V>(px + u * xs);
                fd[u] = load_vec<T, V>(pd + u * ds);
            }
#pragma unroll
            for (int u = 0; u < kNormUnroll; u++) add(fx[u], fd[u]);
            px += kNormUnroll * xs;
            pd += kNormUnroll * ds;
        }
        for (; n > 0; n--, px += xs, pd += ds) add(load_vec<T, V>(px), load_vec<T, V>(pd));
#pragma unroll
        for (int v = 0; v < V; v++) {
            const int at = cols.row * C + col * V + v;
            l1[at] = s1[v];
            l2[at] = s2[v] * ch.rstd[v];
        }
    }
    __syncthreads();
    float2 *part = reinterpret_cast<float2 *>(a.part) + (int64_t)blockIdx.x * C;
    for (int c = threadIdx.x; c < C; c += kNormThreads) {
        float s1 = 0.0f, s2 = 0.0f;
        for (int r = 0; r < cols.rows; r++) {
            s1 += l1[r * C + c];
            s2 += l2[r * C + c];
        }
        part[c] = make_float2(s1, s2);
    }
}

// chan[b][c] = the workgroups' partials summed: kMergeChannels channels of a
// sample (a cache line of partials) per workgroup, 64 lanes of partials each.
constexpr int kMergeChannels = 16, kMergeLanes = 64;
__global__ __launch_bounds__(kMergeChannels *kMergeLanes) void k_norm_grad_merge(NormArgs a)
{
    __shared__ double l1[kMergeLanes / 4][kMergeChannels], l2[kMergeLanes / 4][kMergeChannels];
    const int slabs = (a.channels + kMergeChannels - 1) / kMergeChannels;
    const int b = blockIdx.x / slabs, at = threadIdx.x % kMergeChannels, lane = threadIdx.x / kMergeChannels;
    const int c = (blockIdx.x - b * slabs) * kMergeChannels + at;
    const float2 *part = reinterpret_cast<const float2 *>(a.part) + (int64_t)b * a.blocks * a.channels;
    double s1 = 0.0, s2 = 0.0;
    if (c < a.channels) {
#pragma unroll 8
        for (int i = lane; i < a.blocks; i += kMergeLanes) {
            const float2 p = part[(int64_t)i * a.channels + c];
            s1 += (double)p.x;
            s2 += (double)p.y;
        }
    }
    // a wave holds four lanes of partials, sixteen threads apart
    s1 += __shfl_xor(s1, 16);
    s2 += __shfl_xor(s2, 16);
    s1 += __shfl_xor(s1, 32);
    s2 += __shfl_xor(s2, 32);
    if ((threadIdx.x & 63) < kMergeChannels) {
        l1[threadIdx.x >> 6][at] = s1;
        l2[threadIdx.x >> 6][at] = s2;
    }
    __syncthreads();
    if (threadIdx.x < kMergeChannels && c < a.channels) {
        for (int w = 1; w < kMergeLanes / 4; w++) {
            s1 += l1[w][at];
            s2 += l2[w][at];
        }
        reinterpret_cast<float2 *>(a.chan)[(int64_t)b * a.channels + c] = make_float2((float)s1, (float)s2);
    }
}

// dx, and (the first workgroups) dgamma and dbeta as sums over the samples.
template <typename T, int V, int ACT>
__global__ __launch_bounds__(kNormThreads) void k_norm_grad_apply(NormArgs a)
{
    extern __shared__ float lds[];      // [G][2]: the group's a / n and q / n
    const int C = a.channels, cpg = C / a.groups;
    const float2 *chan = reinterpret_cast<const float2 *>(a.chan);
    const int64_t me = (int64_t)blockIdx.x * kNormThreads + threadIdx.x;
    if ((a.dgamma || a.dbeta) && me < C) {
        double s1 = 0.0, s2 = 0.0;
        for (int b = 0; b < a.samples; b++) {
            const float2 p = chan[(int64_t)b * C + me];
            s1 += (double)p.x;
            s2 += (double)p.y;
        }
        if (a.dbeta) a.dbeta[me] = (float)s1;
        if (a.dgamma) a.dgamma[me] = (float)s2;
    }
    const int b = blockIdx.x / a.blocks, i = blockIdx.x - b * a.blocks;
    if (!a.out || b >= a.samples) return;
    const int pb = valid_pixels(a, b);
    const float inv_n = pb > 0 ? 1.0f / ((float)pb * (float)cpg) : 0.0f;
    const int lanes = lanes_per_group(a.groups), lane = threadIdx.x & (lanes - 1);
    for (int g0 = 0; g0 < a.groups; g0 += kNormThreads / lanes) {
        const int g = g0 + threadIdx.x / lanes;
        float s1 = 0.0f, s2 = 0.0f;
        for (int e = lane; g < a.groups && e < cpg; e += lanes) {
            const int c = g * cpg + e;
            const float2 p = chan[(int64_t)b * C + c];
            const float gamma = a.gamma ? a.gamma[c] : 1.0f;
            s1 = fmaf(gamma, p.x, s1);
            s2 = fmaf(gamma, p.y, s2);
        }
        s1 = sum_lanes(s1, lanes);
        s2 = sum_lanes(s2, lanes);
        if (g < a.groups && lane == 0) {
            lds[2 * g] = s1 * inv_n;
            lds[2 * g + 1] = s2 * inv_n;
        }
    }
    __syncthreads();
    const Columns<V> cols(C);
    const int64_t span = rows_per_block(a.pixels, a.blocks), lo = span * i;
    const int64_t hi = lo + span < a.pixels ? lo + span : a.pixels;
    const int64_t end = hi < pb ? hi : pb;
    const float inv_cpg = 1.0f / (float)cpg;
    for (int col = cols.col; col < cols.per_row; col += kNormThreads) {
        // dx = du (rstd gamma) - rstd a/n - (x - mean) rstd^2 q/n
        const Channels<V> ch(a, b, col);
        float scale[V], flat[V], slope[V];
#pragma unroll
        for (int v = 0; v < V; v++) {
            const int g = group_of(col * V + v, inv_cpg);
            scale[v] = ch.rstd[v] * ch.gamma[v];
            flat[v] = -ch.rstd[v] * lds[2 * g];
            slope[v] = -ch.rstd[v] * ch.rstd[v] * lds[2 * g + 1];
        }
        auto one = [&](const Vec<T, V> &fx, const Vec<T, V> &fd) {
            Vec<T, V> o;
#pragma unroll
            for (int v = 0; v < V; v++) {
                const float d = (float)fx.v[v] - ch.mean[v];
                const float du = (float)fd.v[v] * activate_grad<ACT>(fmaf(d, scale[v], ch.beta[v]));
                o.v[v] = (T)fmaf(du, scale[v], fmaf(d, slope[v], flat[v]));
            }
            return o;
        };
        const int64_t xs = cols.rows * a.x_ld, ds = cols.rows * a.dy_ld, os = cols.rows * a.out_ld;
        int64_t r = lo + cols.row;
        const T *px = static_cast<const T *>(a.x) + b * a.x_sample + col * V + r * a.x_ld;
        const T *pd = static_cast<const T *>(a.dy) + b * a.dy_sample + col * V + r * a.dy_ld;
        T *po = static_cast<T *>(a.out) + b * a.out_sample + col * V + r * a.out_ld;
        for (; r + (kNormUnroll - 1) * cols.rows < end; r += kNormUnroll * cols.rows) {
            Vec<T, V> fx[kNormUnroll], fd[kNormUnroll];
#pragma unroll
            for (int u = 0; u < kNormUnroll; u++) {
                fx[u] = load_vec<T, V>(px + u * xs);
                fd[u] = load_vec<T, V>(pd + u * ds);
            }
#pragma unroll
            for (int u = 0; u < kNormUnroll; u++) store_vec<T, V>(po + u * os, one(fx[u], fd[u]));
            px += kNormUnroll * xs;
            pd += kNormUnroll * ds;
            po += kNormUnroll * os;
        }
        for (; r < end; r += cols.rows, px += xs, pd += ds, po += os)
            store_vec<T, V>(po, one(load_vec<T, V>(px), load_vec<T, V>(pd)));
        Vec<T, V> zero;
#pragma unroll
        for (int v = 0; v < V; v++) zero.v[v] = (T)0.0f;
        for (; r < hi; r += cols.rows, po += os) store_vec<T, V>(po, zero);
    }
}

// Workgroups per sample: enough to fill the chip, no fewer rows each than
// `rows`, no more in all than kNormBlocks (the scratch) or one per sample.
int blocks_per_sample(const NormArgs &a, int rows)
{
    const int64_t want = ceil_div(a.pixels, rows), cap = kNormBlocks / a.samples;
    return (int)(want < 1 ? 1 : want < cap ? want : cap < 1 ? 1 : cap);
}

// Vectors of V channels: LDS floats per sum and rows at a time (Columns).
inline int rows_at_a_time(int C, int V) { return C / V >= kNormThreads ? 1 : kNormThreads / (C / V); }

template <typename T, int V, int ACT>
hipError_t launch_norm(NormArgs a, hipStream_t stream)
{
    const int rows = rows_at_a_time(a.channels, V);
    const size_t lds = 2 * sizeof(float) * (size_t)rows * a.channels;
    if (!a.backward) {
        a.blocks = blocks_per_sample(a, rows * kNormUnroll);
        hipLaunchKernelGGL((k_norm_stats<T, V>), dim3(a.samples * a.blocks), dim3(kNormThreads), lds, stream, a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        if (a.blocks <= 64 * kMergeEach)
            hipLaunchKernelGGL(k_norm_merge<64>, dim3(a.samples * a.groups), dim3(64), 0, stream, a);
        else
            hipLaunchKernelGGL(k_norm_merge<256>, dim3(a.samples * a.groups), dim3(256), 0, stream, a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        hipLaunchKernelGGL((k_norm_apply<T, V, ACT>), dim3(a.samples * a.blocks), dim3(kNormThreads), 0, stream, a);
        return hipGetLastError();
    }
    if (a.samples > 0) {
        a.blocks = blocks_per_sample(a, rows * kNormUnroll);
        hipLaunchKernelGGL((k_norm_grad_sums<T, V, ACT>), dim3(a.samples * a.blocks), dim3(kNormThreads), lds, stream,
                           a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        hipLaunchKernelGGL(k_norm_grad_merge, dim3(a.samples * (int)ceil_div(a.channels, kMergeChannels)),
                           dim3(kMergeChannels * kMergeLanes), 0, stream, a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    } else {
        a.blocks = 1;
    }
    const int vectors = (int)ceil_div(a.channels, kNormThreads), grid = a.samples * a.blocks;
    hipLaunchKernelGGL((k_norm_grad_apply<T, V, ACT>), dim3(grid > vectors ? grid : vectors), dim3(kNormThreads),
                       2 * sizeof(float) * a.groups, stream, a);
    return hipGetLastError();
}

template <typename T, int V>
hipError_t launch_norm_act(const NormArgs &a, hipStream_t stream)
{
    switch (a.act) {
    case CPE_ACT_RELU: return launch_norm<T, V, CPE_ACT_RELU>(a, stream);
    case CPE_ACT_SILU: return launch_norm<T, V, CPE_ACT_SILU>(a, stream);
    case CPE_ACT_GELU: return launch_norm<T, V, CPE_ACT_GELU>(a, stream);
    default: return launch_norm<T, V, CPE_ACT_NONE>(a, stream);
    }
}

// The widest vectors that divide a row.
template <typename T>
hipError_t launch_norm_type(const NormArgs &a, hipStream_t stream)
{
    if constexpr (sizeof(T) == 2)
        if (a.channels % 8 == 0) return launch_norm_act<T, 8>(a, stream);
    if (a.channels % 4 == 0) return launch_norm_act<T, 4>(a, stream);
    if (a.channels % 2 == 0) return launch_norm_act<T, 2>(a, stream);
    return launch_norm_act<T, 1>(a, stream);
}

}  // namespace
}  // namespace cpe
