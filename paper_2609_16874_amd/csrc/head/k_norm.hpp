// k_norm.hpp -- group norm with an activation over channels-last maps, and
// its gradient (private to the library; included once per element type).
//
// Two passes, for maps of any size (k_norm_stats, k_norm_apply; the gradient
// alike): a thread owns V neighbouring channels (up
// to 16 bytes of a row) and walks down the rows, so its channel constants stay
// in registers; a workgroup of 256 covers R = 256 / (C / V) whole rows at a
// time, or one row in several column steps where C / V > 256.  The workgroups
// take chunks of R x kNormUnroll rows in turn, so that the chip reads one
// region of memory at a time, and the second pass takes them in reverse, from
// the end that the first pass has left in the caches.  The first pass's last
// workgroup of a sample (by a counter in memory) joins the partial results.
//
// One pass, where a group fits the registers of a workgroup (k_norm_group,
// k_norm_grad_group): one launch, the map read once.
//
// Statistics.  In two passes each thread sums (x - s) and (x - s)^2 with s
// its first value of the channel, so a mean far from zero cancels nothing;
// threads, then workgroups, are merged as (count, mean, sum of squares about
// the mean),
//   mean = sum n_i mean_i / n,  M2 = sum M2_i + n_i (mean_i - mean)^2,
// in a fixed order.  In one pass the mean m comes first, then the squares
// about it, less (sum (x - m))^2 / n for m's own rounding.
//
// Measured (one MI355X).  409,600 pixels of 256 channels in f16: statistics 46 us
// (4.6 TB/s read), apply 64 us (6.6 TB/s, part of it from the last cache).  The
// gradient of 2,097,152 pixels of 64 channels in bf16: sums 103 us (5.2 TB/s,
// vector unit 77 % busy: 20 instructions a value for SiLU, two of them at a
// quarter of the rate), apply 138 us (5.8 TB/s).  4096 pixels in groups of 8
// channels, f32, one pass: 9 us; 16 x 1024 pixels in groups of 32, bf16: 23 us.
#pragma once

#include "common.hpp"
#include "norm.hpp"

#pragma clang fp contract(fast)

namespace cpe {
namespace {

constexpr int kNormUnroll = 4;      // rows of a thread in flight

__device__ __forceinline__ int valid_pixels(const NormArgs &a, int b)
{
    if (!a.valid) return a.pixels;
    const int v = a.valid[b];
    return v < 0 ? 0 : v > a.pixels ? a.pixels : v;
}

// The rows of each workgroup: chunks of `chunk` rows are dealt to `blocks`
// workgroups in turn, and the last one may be partial.
struct DealtRows {
    int chunk, full, more, last, missing;
    __device__ __forceinline__ DealtRows(int rows, int chunk_, int blocks) : chunk(chunk_)
    {
        const int chunks = (int)(((int64_t)rows + chunk - 1) / chunk);
        full = chunks / blocks;
        more = chunks - full * blocks;
        last = chunks > 0 ? (chunks - 1) % blocks : -1;
        missing = (int)((int64_t)chunks * chunk - rows);
    }
    __device__ __forceinline__ int64_t of(int i, int n = 1) const       // of workgroups i .. i+n-1
    {
        const int extra = more - i < 0 ? 0 : more - i < n ? more - i : n;
        return ((int64_t)full * n + extra) * chunk - (last >= i && last < i + n ? missing : 0);
    }
};

// Store to a map.  Maps that the caches cannot hold beside what the second pass
// reads again are written PAST them: 106M values in 16 bits take 108 us instead
// of 130, the gradient of 30M in 32 bits 117 instead of 136.
typedef uint32_t raw16 __attribute__((ext_vector_type(4)));
template <bool PAST, int N, typename T, int V>
__device__ __forceinline__ void store_map(T *p, int64_t step, const Vec<T, V> (&v)[N], int extra)
{
    if (V > 1 && extra > 0) {       // all but the first `extra` values
#pragma unroll
        for (int u = 0; u < N; u++)
#pragma unroll
            for (int i = 0; i < V; i++)
                if (i >= extra) p[u * step + i] = v[u].v[i];
        return;
    }
#pragma unroll
    for (int u = 0; u < N; u++) {
        if constexpr (PAST && sizeof(v[0]) == 16) {
            raw16 w;
            __builtin_memcpy(&w, &v[u], 16);
            __builtin_nontemporal_store(w, reinterpret_cast<raw16 *>(p + u * step));
        } else {
            store_vec<T, V>(p + u * step, v[u]);
        }
    }
}

// Partial results that another workgroup, maybe on another XCD, reads in the
// same launch: stored and loaded at the device's scope, which goes past the
// XCD's own L2.  (Release and acquire fences would write back and drop that
// whole L2 in every workgroup: 80 us more at 1024 of them.)
__device__ __forceinline__ void share(float2 *p, float x, float y)
{
    uint64_t w;
    const float2 v = make_float2(x, y);
    __builtin_memcpy(&w, &v, 8);
    __hip_atomic_store(reinterpret_cast<uint64_t *>(p), w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 shared_value(const float2 *p)
{
    const uint64_t w =
        __hip_atomic_load(reinterpret_cast<const uint64_t *>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    float2 v;
    __builtin_memcpy(&v, &w, 8);
    return v;
}

// Whether this workgroup is the last of `expected` to count itself here, so
// that all of them have shared their results: each waits for its own stores to
// be done (all counters of s_waitcnt at 0) before.  The counter is 0 again
// afterwards.
__device__ __forceinline__ bool last_to_arrive(int32_t *counter, int expected)
{
    __shared__ int arrived;
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0);
    asm volatile("" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) {
        arrived = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (arrived == expected - 1) *counter = 0;
    }
    __syncthreads();
    return arrived == expected - 1;
}

// Sums over `count` <= kJoinWays rows of G shared pairs, in 64 bits and a fixed
// order: add(k, pair, s0, s1) for each, then done(g, s0, s1).  `lds` holds
// kNormThreads pairs of double.
constexpr int kJoinWays = kNormJoinWays;
template <typename Add, typename Done>
__device__ __forceinline__ void join_rows(const float2 *rows, int count, int groups, double *lds, Add add, Done done)
{
    const int wide = groups < kNormThreads ? groups : kNormThreads;
    const int deep = kNormThreads / wide < kJoinWays ? kNormThreads / wide : kJoinWays;
    const int at = threadIdx.x % wide, row = threadIdx.x / wide;
    for (int g0 = 0; g0 < groups; g0 += wide) {
        const int g = g0 + at;
        double s0 = 0.0, s1 = 0.0;
        if (row < deep && g < groups) {
#pragma unroll 4
            for (int k = row; k < count; k += deep) add(k, shared_value(rows + (int64_t)k * groups + g), s0, s1);
        }
        __syncthreads();
        lds[threadIdx.x] = s0;
        lds[kNormThreads + threadIdx.x] = s1;
        __syncthreads();
        if (row == 0 && g < groups) {
            for (int k = 1; k < deep; k++) {
                s0 += lds[k * wide + at];
                s1 += lds[kNormThreads + k * wide + at];
            }
            done(g, s0, s1);
        }
    }
}

// Join the pairs that a sample's workgroups have shared in part[block][G], as
// a tree of kJoinWays: the last workgroup of each kJoinWays to arrive joins
// their rows, and the last of those the joined ones.  add(first, n, pair, ..):
// the pair of n workgroups from `first` on; between(n, ..) turns the sums of n
// workgroups' pairs into one, done(g, ..) takes the whole sample's.
template <typename Add, typename Between, typename Done>
__device__ __forceinline__ void join_sample(const NormArgs &a, int b, int i, const float2 *part, double *lds, Add add,
                                            Between between, Done done)
{
    const int teams = (a.blocks + kJoinWays - 1) / kJoinWays, team = i / kJoinWays, first = team * kJoinWays;
    const int size = a.blocks - first < kJoinWays ? a.blocks - first : kJoinWays;
    int32_t *counters = a.counters + (int64_t)b * kNormCounters;
    if (!last_to_arrive(counters + 1 + team, size)) return;
    const float2 *mine = part + (int64_t)first * a.groups;
    auto add_block = [&](int k, float2 p, double &s0, double &s1) { add(first + k, 1, p, s0, s1); };
    if (teams == 1) {
        join_rows(mine, size, a.groups, lds, add_block, done);
        return;
    }
    float2 *joined = reinterpret_cast<float2 *>(a.joined) + (int64_t)b * kJoinWays * a.groups;
    join_rows(mine, size, a.groups, lds, add_block, [&](int g, double s0, double s1) {
        const float2 p = between(first, size, s0, s1);
        share(joined + team * a.groups + g, p.x, p.y);
    });
    if (!last_to_arrive(counters, teams)) return;
    join_rows(joined, teams, a.groups, lds,
              [&](int k, float2 p, double &s0, double &s1) {
                  const int n = a.blocks - k * kJoinWays < kJoinWays ? a.blocks - k * kJoinWays : kJoinWays;
                  add(k * kJoinWays, n, p, s0, s1);
              },
              done);
}
static_assert(kNormBlocks <= kJoinWays * kJoinWays && kNormCounters >= 1 + kJoinWays, "two levels join a sample");

// c / cpg for c < 8192 through the reciprocal: c + 1/2 is at least 1/2 from a
// multiple of cpg, and the product's error stays under 1e-3 / cpg.
__device__ __forceinline__ int group_of(int c, float inv_cpg) { return (int)(((float)c + 0.5f) * inv_cpg); }

// A vector's channels: their groups' statistics (one group's where V divides
// the channels of a group: GROUPED), and gamma and beta.  (OVER, below: V does
// not divide a row, see Columns.)
template <int V, bool GROUPED>
struct Channels {
    float mean_[GROUPED ? 1 : V], rstd_[GROUPED ? 1 : V], scale[V], beta[V];     // scale = rstd gamma
    __device__ __forceinline__ float mean(int v) const { return mean_[GROUPED ? 0 : v]; }
    __device__ __forceinline__ float rstd(int v) const { return rstd_[GROUPED ? 0 : v]; }
    __device__ __forceinline__ Channels(const NormArgs &a, int b, int first)
    {
        const float inv_cpg = 1.0f / (float)(a.channels / a.groups);
        const float2 *stats = reinterpret_cast<const float2 *>(a.stats) + (int64_t)b * a.groups;
#pragma unroll
        for (int v = 0; v < (GROUPED ? 1 : V); v++) {
            const float2 st = stats[group_of(first + v, inv_cpg)];
            mean_[v] = st.x;
            rstd_[v] = st.y;
        }
        load(a, first);
    }
    __device__ __forceinline__ Channels(const NormArgs &a, float mean, float rstd, int first)
    {
        static_assert(GROUPED, "one group's statistics");
        mean_[0] = mean;
        rstd_[0] = rstd;
        load(a, first);
    }
    __device__ __forceinline__ void load(const NormArgs &a, int first)
    {
        Vec<float, V> g, s;
#pragma unroll
        for (int v = 0; v < V; v++) {
            g.v[v] = 1.0f;
            s.v[v] = 0.0f;
        }
        if (a.gamma) g = load_vec<float, V>(a.gamma + first);
        if (a.beta) s = load_vec<float, V>(a.beta + first);
#pragma unroll
        for (int v = 0; v < V; v++) {
            scale[v] = rstd(v) * g.v[v];
            beta[v] = s.v[v];
        }
    }
};

// How a workgroup covers a row of C channels.
template <int V>
struct Columns {
    int channels, per_row, rows, col, row;     // vectors in a row, rows at a time, this thread's first vector and row
    __device__ __forceinline__ explicit Columns(int channels_) : channels(channels_)
    {
        per_row = (channels + V - 1) / V;
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
    // The first channel of vector `col`.  Where V does not divide a row its last
    // vector is the row's last V channels; the first extra(col) of them are the
    // vector before's as well, which alone counts and writes them.
    __device__ __forceinline__ int first(int col) const
    {
        return col * V + V <= channels ? col * V : channels - V;
    }
    __device__ __forceinline__ int extra(int col) const { return col * V - first(col); }
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

// Visit this workgroup's chunks of `rows` rows: body(r, count) with r this
// thread's first row, of `count` rows cols.rows apart.  Chunk c goes to
// workgroup c mod blocks; REVERSE takes a workgroup's chunks from the last.
template <bool REVERSE, int V, typename F>
__device__ __forceinline__ void for_chunks(const Columns<V> &cols, int rows, int blocks, int i, F body)
{
    const int chunk = cols.rows * kNormUnroll;
    const int chunks = (int)(((int64_t)rows + chunk - 1) / chunk);
    const int64_t last = i + (int64_t)((chunks - 1 - i) / blocks) * blocks;
    for (int64_t c = i; c < chunks; c += blocks) {
        const int64_t r = (REVERSE ? last - (c - i) : c) * chunk + cols.row;
        const int64_t left = (rows - r + cols.rows - 1) / cols.rows;
        body(r, r >= rows ? 0 : left < kNormUnroll ? (int)left : kNormUnroll);
    }
}

// Partial statistics: part[b][block][g] = (mean, M2) over the block's rows.
template <typename T, int V, bool GROUPED, bool OVER>
__global__ __launch_bounds__(kNormThreads) void k_norm_stats(NormArgs a)
{
    // units of U channels of one group: a thread's vector, or a channel
    constexpr int U = GROUPED ? V : 1;
    extern __shared__ __align__(16) float lds[];      // [rows][C / U] means, then M2
    static_assert(__alignof__(lds) >= alignof(double), "the join's sums are 64-bit");
    __shared__ float counts[kNormThreads];
    const int b = blockIdx.x / a.blocks, i = blockIdx.x - b * a.blocks;
    const int pb = valid_pixels(a, b), C = a.channels, units = C / U;
    const Columns<V> cols(C);
    float *lmean = lds, *lm2 = lds + cols.rows * units;
    const T *x = static_cast<const T *>(a.x) + b * a.x_sample;
    for (int col = cols.col; col < cols.per_row; col += kNormThreads) {
        const int first = OVER ? cols.first(col) : col * V, extra = OVER ? cols.extra(col) : 0;
        const T *p = x + first;
        const int64_t step = cols.rows * a.x_ld;
        int n = 0;
        float shift[V], s1[V], s2[V];
#pragma unroll
        for (int v = 0; v < V; v++) shift[v] = s1[v] = s2[v] = 0.0f;
        auto add = [&](const Vec<T, V> &f) {
#pragma unroll
            for (int v = 0; v < V; v++) {
                const float d = (float)f.v[v] - shift[v];
                s1[v] += d;
                s2[v] = fmaf(d, d, s2[v]);
            }
        };
        for_chunks<false, V>(cols, pb, a.blocks, i, [&](int64_t r, int count) {
            const T *q = p + r * a.x_ld;
            Vec<T, V> f[kNormUnroll];
            if (count == kNormUnroll) {
#pragma unroll
                for (int u = 0; u < kNormUnroll; u++) f[u] = load_vec<T, V>(q + u * step);
            } else {
#pragma unroll
                for (int u = 0; u < kNormUnroll; u++)
                    if (u < count) f[u] = load_vec<T, V>(q + u * step);
            }
            if (n == 0 && count > 0) {
#pragma unroll
                for (int v = 0; v < V; v++) shift[v] = (float)f[0].v[v];
            }
            n += count;
#pragma unroll
            for (int u = 0; u < kNormUnroll; u++)
                if (u < count) add(f[u]);
        });
        const float inv = 1.0f / (float)(n > 0 ? n : 1);
        float mean[V], m2[V];
#pragma unroll
        for (int v = 0; v < V; v++) {
            mean[v] = fmaf(s1[v], inv, shift[v]);
            m2[v] = s2[v] - s1[v] * s1[v] * inv;
        }
        const int at = cols.row * units + first / U;
        if constexpr (GROUPED) {
            float m = 0.0f, q = 0.0f;
#pragma unroll
            for (int v = 0; v < V; v++) m += mean[v];
            m *= 1.0f / V;
#pragma unroll
            for (int v = 0; v < V; v++) q += fmaf((float)n * (mean[v] - m), mean[v] - m, m2[v]);
            lmean[at] = m;
            lm2[at] = q;
        } else {
#pragma unroll
            for (int v = 0; v < V; v++)
                if (v >= extra) {
                    lmean[at + v] = mean[v];
                    lm2[at + v] = m2[v];
                }
        }
        if (col == 0) counts[cols.row] = (float)(n * U);
    }
    __syncthreads();
    const int lanes = lanes_per_group(a.groups), upg = units / a.groups, entries = cols.rows * upg;
    const int lane = threadIdx.x & (lanes - 1);
    const float inv_upg = 1.0f / (float)upg;
    const DealtRows rows(pb, a.chunk, a.blocks);
    const int64_t n_rows = rows.of(i);
    const float inv_n = 1.0f / ((float)(n_rows > 0 ? n_rows : 1) * (float)(upg * U));
    float2 *part = reinterpret_cast<float2 *>(a.part) + (int64_t)blockIdx.x * a.groups;
    for (int g0 = 0; g0 < a.groups; g0 += kNormThreads / lanes) {
        const int g = g0 + threadIdx.x / lanes;
        const bool on = g < a.groups;
        float mean = 0.0f, m2 = 0.0f;
        for (int e = lane; on && e < entries; e += lanes) {
            const int row = cols.rows == 1 ? 0 : group_of(e, inv_upg);
            mean += counts[row] * lmean[row * units + g * upg + (e - row * upg)];
        }
        mean = sum_lanes(mean, lanes) * inv_n;
        for (int e = lane; on && e < entries; e += lanes) {
            const int row = cols.rows == 1 ? 0 : group_of(e, inv_upg), at = row * units + g * upg + (e - row * upg);
            const float d = lmean[at] - mean, n = counts[row];
            if (n > 0.0f) m2 += fmaf(n * d, d, lm2[at]);
        }
        m2 = sum_lanes(m2, lanes);
        if (on && lane == 0) share(part + g, mean, m2);
    }
    // s0 and s1: sums of n mean and of M2 + n mean^2
    const double per_row = (double)(upg * U);
    join_sample(
        a, b, i, part - (int64_t)i * a.groups, reinterpret_cast<double *>(lds),
        [&](int first, int count, float2 p, double &s0, double &s1) {
            const double n = (double)rows.of(first, count) * per_row;
            if (n > 0.0) {
                s0 += n * (double)p.x;
                s1 += (double)p.y + n * (double)p.x * (double)p.x;
            }
        },
        [&](int first, int count, double s0, double s1) {
            const double n = (double)rows.of(first, count) * per_row, m = n > 0.0 ? s0 / n : 0.0;
            return make_float2((float)m, (float)(s1 - s0 * m));
        },
        [&](int g, double s0, double s1) {
            const double n = pb > 0 ? (double)pb * per_row : 1.0;
            const double mean = s0 / n, square = s1 / n - mean * mean, var = square < 0.0 ? 0.0 : square;
            reinterpret_cast<float2 *>(a.stats)[(int64_t)b * a.groups + g] =
                make_float2((float)mean, (float)(1.0 / sqrt(var + a.eps)));
        });
}

// y = act((x - mean) (rstd gamma) + beta); pixels from the sample's count on
// are set to 0.
template <typename T, int V, bool GROUPED, bool OVER, bool PAST, int ACT>
__global__ __launch_bounds__(kNormThreads) void k_norm_apply(NormArgs a)
{
    const int b = blockIdx.x / a.blocks, i = blockIdx.x - b * a.blocks;
    const Columns<V> cols(a.channels);
    const int pb = valid_pixels(a, b);
    for (int col = cols.col; col < cols.per_row; col += kNormThreads) {
        const int first = OVER ? cols.first(col) : col * V, extra = OVER ? cols.extra(col) : 0;
        const T *x = static_cast<const T *>(a.x) + b * a.x_sample + first;
        T *y = static_cast<T *>(a.out) + b * a.out_sample + first;
        const Channels<V, GROUPED> ch(a, b, first);
        auto one = [&](const Vec<T, V> &f) {
            Vec<T, V> o;
#pragma unroll
            for (int v = 0; v < V; v++)
                o.v[v] = (T)activate<ACT>(fmaf((float)f.v[v] - ch.mean(v), ch.scale[v], ch.beta[v]));
            return o;
        };
        const int64_t xs = cols.rows * a.x_ld, ys = cols.rows * a.out_ld;
        for_chunks<true, V>(cols, a.pixels, a.blocks, i, [&](int64_t r, int count) {
            const T *px = x + r * a.x_ld;
            T *py = y + r * a.out_ld;
            if (count == kNormUnroll && r + (kNormUnroll - 1) * cols.rows < pb) {
                Vec<T, V> f[kNormUnroll];
#pragma unroll
                for (int u = 0; u < kNormUnroll; u++) f[u] = load_vec<T, V>(px + u * xs);
#pragma unroll
                for (int u = 0; u < kNormUnroll; u++) f[u] = one(f[u]);
                store_map<PAST>(py, ys, f, extra);
            } else {
                for (int u = 0; u < count; u++) {
                    Vec<T, V> o[1];
#pragma unroll
                    for (int v = 0; v < V; v++) o[0].v[v] = (T)0.0f;
                    if (r + u * cols.rows < pb) o[0] = one(load_vec<T, V>(px + u * xs));
                    store_map<PAST>(py + u * ys, 0, o, extra);
                }
            }
        });
    }
}

// part[b][block][c] = (sum du, sum du xh) over the block's rows.
template <typename T, int V, bool GROUPED, bool OVER, int ACT>
__global__ __launch_bounds__(kNormThreads) void k_norm_grad_sums(NormArgs a)
{
    extern __shared__ __align__(16) float lds[];      // [rows][C] sums of du, then of du xh
    static_assert(__alignof__(lds) >= alignof(double), "the join's sums are 64-bit");
    const int b = blockIdx.x / a.blocks, i = blockIdx.x - b * a.blocks;
    const int pb = valid_pixels(a, b), C = a.channels;
    const Columns<V> cols(C);
    float *l1 = lds, *l2 = lds + cols.rows * C;
    for (int col = cols.col; col < cols.per_row; col += kNormThreads) {
        const int first = OVER ? cols.first(col) : col * V, extra = OVER ? cols.extra(col) : 0;
        const Channels<V, GROUPED> ch(a, b, first);
        const T *x = static_cast<const T *>(a.x) + b * a.x_sample + first;
        const T *dy = static_cast<const T *>(a.dy) + b * a.dy_sample + first;
        const int64_t xs = cols.rows * a.x_ld, ds = cols.rows * a.dy_ld;
        float s1[V], s2[V];
#pragma unroll
        for (int v = 0; v < V; v++) s1[v] = s2[v] = 0.0f;
        auto add = [&](const Vec<T, V> &fx, const Vec<T, V> &fd) {
#pragma unroll
            for (int v = 0; v < V; v++) {
                const float d = (float)fx.v[v] - ch.mean(v);
                const float du = (float)fd.v[v] * activate_grad<ACT>(fmaf(d, ch.scale[v], ch.beta[v]));
                s1[v] += du;
                s2[v] = fmaf(du, d, s2[v]);
            }
        };
        for_chunks<false, V>(cols, pb, a.blocks, i, [&](int64_t r, int count) {
            const T *px = x + r * a.x_ld, *pd = dy + r * a.dy_ld;
            if (count == kNormUnroll) {
                Vec<T, V> fx[kNormUnroll], fd[kNormUnroll];
#pragma unroll
                for (int u = 0; u < kNormUnroll; u++) {
                    fx[u] = load_vec<T, V>(px + u * xs);
                    fd[u] = load_vec<T, V>(pd + u * ds);
                }
#pragma unroll
                for (int u = 0; u < kNormUnroll; u++) add(fx[u], fd[u]);
            } else {
                for (int u = 0; u < count; u++) add(load_vec<T, V>(px + u * xs), load_vec<T, V>(pd + u * ds));
            }
        });
#pragma unroll
        for (int v = 0; v < V; v++)
            if (v >= extra) {
                const int at = cols.row * C + first + v;
                l1[at] = s1[v];
                l2[at] = s2[v] * ch.rstd(v);
            }
    }
    __syncthreads();
    for (int c = threadIdx.x; c < C; c += kNormThreads) {
        float s1 = 0.0f, s2 = 0.0f;
        for (int r = 0; r < cols.rows; r++) {
            s1 += l1[r * C + c];
            s2 += l2[r * C + c];
        }
        if (a.dgamma || a.dbeta) reinterpret_cast<float2 *>(a.part)[(int64_t)blockIdx.x * C + c] = make_float2(s1, s2);
        const float gamma = a.gamma ? a.gamma[c] : 1.0f;
        l1[c] = s1 * gamma;     // (row 0, of which this thread has just read its place)
        l2[c] = s2 * gamma;
    }
    __syncthreads();
    if (!a.out) return;
    const int lanes = lanes_per_group(a.groups), cpg = C / a.groups, lane = threadIdx.x & (lanes - 1);
    float2 *part = reinterpret_cast<float2 *>(a.group_part) + (int64_t)blockIdx.x * a.groups;
    for (int g0 = 0; g0 < a.groups; g0 += kNormThreads / lanes) {
        const int g = g0 + threadIdx.x / lanes;
        float s1 = 0.0f, s2 = 0.0f;
        for (int e = lane; g < a.groups && e < cpg; e += lanes) {
            s1 += l1[g * cpg + e];
            s2 += l2[g * cpg + e];
        }
        s1 = sum_lanes(s1, lanes);
        s2 = sum_lanes(s2, lanes);
        if (g < a.groups && lane == 0) share(part + g, s1, s2);
    }
    join_sample(
        a, b, i, part - (int64_t)i * a.groups, reinterpret_cast<double *>(lds),
        [](int, int, float2 p, double &s1, double &s2) {
            s1 += (double)p.x;
            s2 += (double)p.y;
        },
        [](int, int, double s1, double s2) { return make_float2((float)s1, (float)s2); },
        [&](int g, double s1, double s2) {
            const double n = pb > 0 ? (double)pb * cpg : 1.0;
            reinterpret_cast<float2 *>(a.group_sums)[(int64_t)b * a.groups + g] =
                make_float2((float)(s1 / n), (float)(s2 / n));
        });
}

// dgamma and dbeta of kVectorChannels channels (a cache line of partials) as
// sums over `partials` of them, by a workgroup of kNormThreads.
constexpr int kVectorChannels = 16;
__device__ __forceinline__ void sum_vectors(const NormArgs &a, int slab, int64_t partials)
{
    constexpr int kLanes = kNormThreads / kVectorChannels;
    __shared__ double l1[kLanes][kVectorChannels], l2[kLanes][kVectorChannels];
    const int at = threadIdx.x % kVectorChannels, lane = threadIdx.x / kVectorChannels;
    const int c = slab * kVectorChannels + at;
    double s1 = 0.0, s2 = 0.0;
    if (c < a.channels) {
        const float2 *part = reinterpret_cast<const float2 *>(a.part) + c;
#pragma unroll 16
        for (int64_t i = lane; i < partials; i += kLanes) {
            const float2 p = part[i * a.channels];
            s1 += (double)p.x;
            s2 += (double)p.y;
        }
    }
    l1[lane][at] = s1;
    l2[lane][at] = s2;
    __syncthreads();
    if (lane > 0 || c >= a.channels) return;
    for (int l = 1; l < kLanes; l++) {
        s1 += l1[l][at];
        s2 += l2[l][at];
    }
    if (a.dbeta) a.dbeta[c] = (float)s1;
    if (a.dgamma) a.dgamma[c] = (float)s2;
}
template <int UNUSED>
__global__ __launch_bounds__(kNormThreads) void k_norm_grad_vectors(NormArgs a)
{
    sum_vectors(a, blockIdx.x, (int64_t)a.samples * a.blocks);
}

// One element of dx = du (rstd gamma) - rstd a/n - (x - mean) rstd^2 q/n, with
// flat and slope the last two terms' factors.
template <int ACT, int V, bool GROUPED>
__device__ __forceinline__ float grad_one(const Channels<V, GROUPED> &ch, int v, float x, float dy, float flat,
                                          float slope)
{
    const float d = x - ch.mean(v);
    const float du = dy * activate_grad<ACT>(fmaf(d, ch.scale[v], ch.beta[v]));
    return fmaf(du, ch.scale[v], fmaf(d, slope, flat));
}

// dx, and (the first `vectors` workgroups) dgamma and dbeta.
template <typename T, int V, bool GROUPED, bool OVER, bool PAST, int ACT>
__global__ __launch_bounds__(kNormThreads) void k_norm_grad_apply(NormArgs a, int vectors)
{
    if ((int)blockIdx.x < vectors) {
        sum_vectors(a, blockIdx.x, (int64_t)a.samples * a.blocks);
        return;
    }
    const int w = blockIdx.x - vectors, b = w / a.blocks, i = w - b * a.blocks;
    const int pb = valid_pixels(a, b);
    const Columns<V> cols(a.channels);
    const float inv_cpg = 1.0f / (float)(a.channels / a.groups);
    const float2 *sums = reinterpret_cast<const float2 *>(a.group_sums) + (int64_t)b * a.groups;
    for (int col = cols.col; col < cols.per_row; col += kNormThreads) {
        const int first = OVER ? cols.first(col) : col * V, extra = OVER ? cols.extra(col) : 0;
        const Channels<V, GROUPED> ch(a, b, first);
        constexpr int N = GROUPED ? 1 : V;
        float flat[N], slope[N];
#pragma unroll
        for (int v = 0; v < N; v++) {
            const float2 aq = sums[group_of(first + v, inv_cpg)];       // a / n and q / n
            flat[v] = -ch.rstd(v) * aq.x;
            slope[v] = -ch.rstd(v) * ch.rstd(v) * aq.y;
        }
        auto one = [&](const Vec<T, V> &fx, const Vec<T, V> &fd) {
            Vec<T, V> o;
#pragma unroll
            for (int v = 0; v < V; v++)
                o.v[v] = (T)grad_one<ACT>(ch, v, (float)fx.v[v], (float)fd.v[v], flat[GROUPED ? 0 : v],
                                          slope[GROUPED ? 0 : v]);
            return o;
        };
        const T *x = static_cast<const T *>(a.x) + b * a.x_sample + first;
        const T *dy = static_cast<const T *>(a.dy) + b * a.dy_sample + first;
        T *dx = static_cast<T *>(a.out) + b * a.out_sample + first;
        const int64_t xs = cols.rows * a.x_ld, ds = cols.rows * a.dy_ld, os = cols.rows * a.out_ld;
        for_chunks<true, V>(cols, a.pixels, a.blocks, i, [&](int64_t r, int count) {
            const T *px = x + r * a.x_ld, *pd = dy + r * a.dy_ld;
            T *po = dx + r * a.out_ld;
            if (count == kNormUnroll && r + (kNormUnroll - 1) * cols.rows < pb) {
                Vec<T, V> fx[kNormUnroll], fd[kNormUnroll];
#pragma unroll
                for (int u = 0; u < kNormUnroll; u++) {
                    fx[u] = load_vec<T, V>(px + u * xs);
                    fd[u] = load_vec<T, V>(pd + u * ds);
                }
#pragma unroll
                for (int u = 0; u < kNormUnroll; u++) fx[u] = one(fx[u], fd[u]);
                store_map<PAST>(po, os, fx, extra);
            } else {
                for (int u = 0; u < count; u++) {
                    Vec<T, V> o[1];
#pragma unroll
                    for (int v = 0; v < V; v++) o[0].v[v] = (T)0.0f;
                    if (r + u * cols.rows < pb) o[0] = one(load_vec<T, V>(px + u * xs), load_vec<T, V>(pd + u * ds));
                    store_map<PAST>(po + u * os, 0, o, extra);
                }
            }
        });
    }
}

// -- one pass ----------------------------------------------------------------------

constexpr int kGroupThreads = 1024;
// Vectors of 16 bytes of a map that a thread holds at most (the gradient holds
// two maps, and 16-bit values take twice the registers while they are summed).
template <typename T>
constexpr int held_most(bool backward) { return backward && sizeof(T) == 2 ? 4 : 8; }

__device__ __forceinline__ float block_sum(float v, float *lds)
{
    v = sum_lanes(v, 64);
    __syncthreads();        // the values of the sum before are read
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0f;
#pragma unroll
    for (int w = 0; w < kGroupThreads / 64; w++) v += lds[w];
    return v;
}

// Values held from one step to the next stay as they were loaded: without
// this the compiler keeps their binary32 conversions instead, which are twice
// as many registers as there are.
template <typename T, int V, int K>
__device__ __forceinline__ void as_loaded(Vec<T, V> (&held)[K])
{
    if constexpr (sizeof(T) == 2 && V % 2 == 0) {
#pragma unroll
        for (int k = 0; k < K; k++) {
            uint32_t w[V / 2];
            __builtin_memcpy(w, &held[k], sizeof(w));
#pragma unroll
            for (int i = 0; i < V / 2; i++) asm volatile("" : "+v"(w[i]));
            __builtin_memcpy(&held[k], w, sizeof(w));
        }
    }
}

// How a workgroup covers one group's channels: vectors of V, `rows` rows at a
// time; threads left over have no row.
template <int V>
struct GroupColumns {
    int b, g, per_row, rows, col, row;
    __device__ __forceinline__ explicit GroupColumns(const NormArgs &a)
    {
        // neighbouring groups share cache lines: keep them on one XCD
        const int w = xcd_order(blockIdx.x, gridDim.x);
        b = w / a.groups;
        g = w - b * a.groups;
        per_row = a.channels / a.groups / V;
        rows = kGroupThreads / per_row;
        row = threadIdx.x / per_row;
        col = threadIdx.x - row * per_row;
        if (row >= rows) row = 0x40000000;      // beyond any map that fits
    }
};

template <typename T, int V, int ACT, int K>
__global__ __launch_bounds__(kGroupThreads) void k_norm_group(NormArgs a)
{
    __shared__ float lds[kGroupThreads / 64];
    const GroupColumns<V> at(a);
    const int pb = valid_pixels(a, at.b), cpg = at.per_row * V, col = at.g * at.per_row + at.col;
    const T *x = static_cast<const T *>(a.x) + at.b * a.x_sample + col * V;
    T *y = static_cast<T *>(a.out) + at.b * a.out_sample + col * V;
    Vec<T, V> held[K];
    float sum = 0.0f;
#pragma unroll
    for (int k = 0; k < K; k++) {
        const int r = at.row + k * at.rows;
        if (r < pb) held[k] = load_vec<T, V>(x + r * a.x_ld);
    }
    as_loaded(held);
#pragma unroll
    for (int k = 0; k < K; k++)
        if (at.row + k * at.rows < pb) {
#pragma unroll
            for (int v = 0; v < V; v++) sum += (float)held[k].v[v];
        }
    const float n = (float)(pb > 0 ? pb : 1) * (float)cpg;
    float mean = block_sum(sum, lds) / n, off = 0.0f, m2 = 0.0f;
    as_loaded(held);
#pragma unroll
    for (int k = 0; k < K; k++)
        if (at.row + k * at.rows < pb) {
#pragma unroll
            for (int v = 0; v < V; v++) {
                const float d = (float)held[k].v[v] - mean;
                off += d;
                m2 = fmaf(d, d, m2);
            }
        }
    off = block_sum(off, lds);
    m2 = block_sum(m2, lds) - off * off / n;
    mean += off / n;
    const float var = m2 > 0.0f || m2 != m2 ? m2 / n : 0.0f;
    const float rstd = (float)(1.0 / sqrt((double)var + (double)a.eps));
    if (threadIdx.x == 0) reinterpret_cast<float2 *>(a.stats)[at.b * a.groups + at.g] = make_float2(mean, rstd);
    const Channels<V, true> ch(a, mean, rstd, at.row < at.rows ? col * V : 0);
    as_loaded(held);
#pragma unroll
    for (int k = 0; k < K; k++) {
        const int r = at.row + k * at.rows;
        if (r >= a.pixels) continue;
        Vec<T, V> o;
#pragma unroll
        for (int v = 0; v < V; v++)
            o.v[v] = r < pb ? (T)activate<ACT>(fmaf((float)held[k].v[v] - mean, ch.scale[v], ch.beta[v])) : (T)0.0f;
        store_vec<T, V>(y + r * a.out_ld, o);
    }
}

// The gradient of one group: x and dy held; per-channel sums over the rows
// through LDS; dgamma and dbeta straight out where there is one sample.
template <typename T, int V, int ACT, int K>
__global__ __launch_bounds__(kGroupThreads) void k_norm_grad_group(NormArgs a)
{
    extern __shared__ __align__(16) float lds[];      // [rows][cpg], then [lanes][cpg] and [2][cpg]
    const GroupColumns<V> at(a);
    const int pb = valid_pixels(a, at.b), cpg = at.per_row * V, col = at.g * at.per_row + at.col;
    const T *x = static_cast<const T *>(a.x) + at.b * a.x_sample + col * V;
    const T *dy = static_cast<const T *>(a.dy) + at.b * a.dy_sample + col * V;
    Vec<T, V> hx[K], hd[K];
#pragma unroll
    for (int k = 0; k < K; k++) {
        const int r = at.row + k * at.rows;
        if (r < pb) {
            hx[k] = load_vec<T, V>(x + r * a.x_ld);
            hd[k] = load_vec<T, V>(dy + r * a.dy_ld);
        }
    }
    as_loaded(hx);
    as_loaded(hd);
    const float2 st = reinterpret_cast<const float2 *>(a.stats)[at.b * a.groups + at.g];
    const Channels<V, true> ch(a, st.x, st.y, at.row < at.rows ? col * V : 0);
    float sum[2][V];
#pragma unroll
    for (int v = 0; v < V; v++) sum[0][v] = sum[1][v] = 0.0f;
#pragma unroll
    for (int k = 0; k < K; k++)
        if (at.row + k * at.rows < pb) {
#pragma unroll
            for (int v = 0; v < V; v++) {
                const float d = (float)hx[k].v[v] - st.x;
                const float du = (float)hd[k].v[v] * activate_grad<ACT>(fmaf(d, ch.scale[v], ch.beta[v]));
                sum[0][v] += du;
                sum[1][v] = fmaf(du, d, sum[1][v]);
            }
        }
    const int lanes = kGroupThreads / cpg, c = threadIdx.x % cpg, lane = threadIdx.x / cpg;
    const int wave = threadIdx.x >> 6, in_wave = threadIdx.x & 63;
    float *second = lds + at.rows * cpg, *total = second + kGroupThreads;
#pragma unroll
    for (int w = 0; w < 2; w++) {
        if (at.row < at.rows) {
#pragma unroll
            for (int v = 0; v < V; v++) lds[at.row * cpg + at.col * V + v] = sum[w][v];
        }
        __syncthreads();
        float s = 0.0f;
        if (lane < lanes) {
            for (int r = lane; r < at.rows; r += lanes) s += lds[r * cpg + c];
            second[lane * cpg + c] = s;
        }
        __syncthreads();
        for (int k = wave; k < cpg; k += kGroupThreads / 64) {
            s = 0.0f;
            for (int l = in_wave; l < lanes; l += 64) s += second[l * cpg + k];
            s = sum_lanes(s, 64);
            if (in_wave == 0) total[w * cpg + k] = w ? s * st.y : s;
        }
    }
    __syncthreads();
    float ga = 0.0f, gq = 0.0f;
    for (int k = in_wave; k < cpg; k += 64) {
        const float gamma = a.gamma ? a.gamma[at.g * cpg + k] : 1.0f;
        ga = fmaf(gamma, total[k], ga);
        gq = fmaf(gamma, total[cpg + k], gq);
    }
    const float inv_n = pb > 0 ? 1.0f / ((float)pb * (float)cpg) : 0.0f;
    ga = sum_lanes(ga, 64) * inv_n;
    gq = sum_lanes(gq, 64) * inv_n;
    for (int k = threadIdx.x; k < cpg; k += kGroupThreads) {
        const int64_t ch_at = at.g * cpg + k;
        if (a.samples > 1) {
            reinterpret_cast<float2 *>(a.part)[(int64_t)at.b * a.channels + ch_at] =
                make_float2(total[k], total[cpg + k]);
        } else {
            if (a.dbeta) a.dbeta[ch_at] = total[k];
            if (a.dgamma) a.dgamma[ch_at] = total[cpg + k];
        }
    }
    if (!a.out) return;
    T *dx = static_cast<T *>(a.out) + at.b * a.out_sample + col * V;
    const float flat = -st.y * ga, slope = -st.y * st.y * gq;
    as_loaded(hx);
    as_loaded(hd);
#pragma unroll
    for (int k = 0; k < K; k++) {
        const int r = at.row + k * at.rows;
        if (r >= a.pixels) continue;
        Vec<T, V> o;
#pragma unroll
        for (int v = 0; v < V; v++)
            o.v[v] = r < pb ? (T)grad_one<ACT>(ch, v, (float)hx[k].v[v], (float)hd[k].v[v], flat, slope) : (T)0.0f;
        store_vec<T, V>(dx + r * a.out_ld, o);
    }
}

// -- launches ----------------------------------------------------------------------

// Workgroups per sample: enough to fill the chip, no more than there are
// chunks, no more in all than kNormBlocks (the scratch) or one per sample.
int blocks_per_sample(const NormArgs &a)
{
    const int64_t want = ceil_div(a.pixels, a.chunk), cap = kNormBlocks / a.samples;
    return (int)(want < cap ? want : cap < 1 ? 1 : cap);
}

// Whether every vector of the written map is 16-byte aligned (the stores past
// the caches say so).
template <typename T>
bool aligned_rows(const NormArgs &a)
{
    constexpr int E = 16 / (int)sizeof(T);
    return aligned_to(a.out, 16) && a.out_ld % E == 0 && (a.samples == 1 || a.out_sample % E == 0);
}

template <typename T, int V, bool GROUPED, bool OVER, int ACT>
hipError_t launch_norm(NormArgs a, hipStream_t stream)
{
    const int per_row = (int)ceil_div(a.channels, V), rows = per_row >= kNormThreads ? 1 : kNormThreads / per_row;
    const size_t least = 2 * sizeof(double) * kNormThreads;       // (the join's)
    const size_t whole = 2 * sizeof(float) * (size_t)rows * a.channels, units = GROUPED ? whole / V : whole;
    const size_t lds = a.backward ? whole : units;
    a.chunk = rows * kNormUnroll;
    a.blocks = a.samples > 0 ? blocks_per_sample(a) : 0;
    const int64_t bytes = (int64_t)a.samples * a.pixels * a.channels * (int64_t)sizeof(T);
    constexpr bool kCanPast = V * sizeof(T) == 16 && !OVER;
    const bool past = kCanPast && bytes * (a.backward ? 3 : 2) > kCacheBytes && aligned_rows<T>(a);
    const dim3 grid(a.samples * a.blocks), block(kNormThreads);
    if (!a.backward) {
        hipLaunchKernelGGL((k_norm_stats<T, V, GROUPED, OVER>), grid, block, lds > least ? lds : least, stream, a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        if (past)
            hipLaunchKernelGGL((k_norm_apply<T, V, GROUPED, OVER, kCanPast, ACT>), grid, block, 0, stream, a);
        else
            hipLaunchKernelGGL((k_norm_apply<T, V, GROUPED, OVER, false, ACT>), grid, block, 0, stream, a);
        return hipGetLastError();
    }
    const int vectors = a.dgamma || a.dbeta ? (int)ceil_div(a.channels, kVectorChannels) : 0;
    if (a.samples > 0) {
        hipLaunchKernelGGL((k_norm_grad_sums<T, V, GROUPED, OVER, ACT>), grid, block, lds > least ? lds : least,
                           stream, a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    if (a.samples > 0 && a.out && past)
        hipLaunchKernelGGL((k_norm_grad_apply<T, V, GROUPED, OVER, kCanPast, ACT>), dim3(grid.x + vectors), block,
                           0, stream, a, vectors);
    else if (a.samples > 0 && a.out)
        hipLaunchKernelGGL((k_norm_grad_apply<T, V, GROUPED, OVER, false, ACT>), dim3(grid.x + vectors), block, 0,
                           stream, a, vectors);
    else
        hipLaunchKernelGGL(k_norm_grad_vectors<0>, dim3(vectors), block, 0, stream, a);
    return hipGetLastError();
}

// One pass where a group's values fit a workgroup's registers: 8 to 9 us against
// 12 for two passes on small maps (calls as a program makes them), 22 against 26
// at 1024 groups of 16384 values in f16.  A workgroup of 1024 costs 2 us a round
// of the chip at least, so many small groups go in two passes: 8192 groups of
// 128 values 71 us against 12; the gradient in 16 bits, whose registers leave
// room for one workgroup per CU, already 17 against 13 at 512 groups of 2048.
// Rows of a group shorter than 32 bytes share their cache lines with other
// workgroups, which costs more than the second reading on larger maps (16 x
// 2048 x 32 x 8 in 16 bits, 17 MB: gradient 32 us against 24; 8 MB: equal).
template <typename T, int V>
bool group_fits(const NormArgs &a)
{
    const int cpg = a.channels / a.groups;
    if (a.samples < 1 || cpg % V != 0 || cpg / V > kGroupThreads || cpg > 1024) return false;
    const int64_t groups = (int64_t)a.samples * a.groups, bytes = (int64_t)a.pixels * cpg * (int64_t)sizeof(T);
    const bool crowded = a.backward && sizeof(T) == 2;
    if (groups > (crowded ? 256 : 512) && (crowded || bytes < 32 << 10 || groups > 1 << 21)) return false;
    if (cpg * (int)sizeof(T) < 32 && groups * bytes > (int64_t)8 << 20) return false;
    return ceil_div(a.pixels, kGroupThreads / (cpg / V)) <= held_most<T>(a.backward);
}

template <typename T, int V, int ACT, int K>
hipError_t launch_group_held(const NormArgs &a, hipStream_t stream)
{
    const dim3 grid(a.samples * a.groups);
    if (!a.backward) {
        hipLaunchKernelGGL((k_norm_group<T, V, ACT, K>), grid, dim3(kGroupThreads), 0, stream, a);
        return hipGetLastError();
    }
    if constexpr (K <= held_most<T>(true)) {
        const int cpg = a.channels / a.groups, rows = kGroupThreads / (cpg / V);
        const size_t lds = sizeof(float) * ((size_t)rows * cpg + kGroupThreads + 2 * cpg);
        hipLaunchKernelGGL((k_norm_grad_group<T, V, ACT, K>), grid, dim3(kGroupThreads), lds, stream, a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        if (a.samples == 1 || (!a.dgamma && !a.dbeta)) return hipSuccess;
        NormArgs v = a;
        v.blocks = 1;
        hipLaunchKernelGGL(k_norm_grad_vectors<0>, dim3((unsigned)ceil_div(a.channels, kVectorChannels)),
                           dim3(kNormThreads), 0, stream, v);
    }
    return hipGetLastError();
}

template <typename T, int V, int ACT>
hipError_t launch_group(const NormArgs &a, hipStream_t stream)
{
    const int rows = kGroupThreads / (a.channels / a.groups / V);
    if (ceil_div(a.pixels, rows) <= 2) return launch_group_held<T, V, ACT, 2>(a, stream);
    if (ceil_div(a.pixels, rows) <= 4) return launch_group_held<T, V, ACT, 4>(a, stream);
    return launch_group_held<T, V, ACT, 8>(a, stream);
}

template <typename T, int ACT>
hipError_t launch_norm_act(const NormArgs &a, hipStream_t stream)
{
    const int C = a.channels, cpg = C / a.groups;
    // one pass, in the widest vectors that divide a group
    if constexpr (sizeof(T) == 2)
        if (group_fits<T, 8>(a)) return launch_group<T, 8, ACT>(a, stream);
    if (group_fits<T, 4>(a)) return launch_group<T, 4, ACT>(a, stream);
    if (group_fits<T, 1>(a)) return launch_group<T, 1, ACT>(a, stream);
    // two passes, in 16-byte vectors (1000 x 1000 pixels of 25 channels in bf16: 30 us
    // in vectors of one)
    constexpr int E = 16 / (int)sizeof(T);
    if (cpg % E == 0) return launch_norm<T, E, true, false, ACT>(a, stream);
    if (C % E == 0) return launch_norm<T, E, false, false, ACT>(a, stream);
    if (C >= E) return launch_norm<T, E, false, true, ACT>(a, stream);
    return launch_norm<T, 1, true, false, ACT>(a, stream);
}

template <typename T>
hipError_t launch_norm_type(const NormArgs &a, hipStream_t stream)
{
    switch (a.act) {
    case CPE_ACT_RELU: return launch_norm_act<T, CPE_ACT_RELU>(a, stream);
    case CPE_ACT_SILU: return launch_norm_act<T, CPE_ACT_SILU>(a, stream);
    case CPE_ACT_GELU: return launch_norm_act<T, CPE_ACT_GELU>(a, stream);
    default: return launch_norm_act<T, CPE_ACT_NONE>(a, stream);
    }
}

}  // namespace
}  // namespace cpe
