// k_rows.hpp -- kernels that work row by row: packing rows into 8 bits, RMS
// norm with the residual's addition, its gradient (private to the library;
// included once per element type).
//
// A row belongs to LANES neighbouring threads, N vectors of V elements each,
// and stays in their registers between its reduction and what is written: each
// input is read once.  (The widest forms spill some: packing more than 32,768 elements
// 80 bytes a lane in f16, 20 in bf16, 12 in f32; the gradient of more than 8192
// channels 28 to 36 in f32, 12 in 16 bits from packed rows.)  Up to 64 lanes a row's sums pass between the lanes of
// its wave, beyond that through LDS.  Workgroups take rows in turn, with the
// next row's loads in flight while the present one is worked on; gamma stays
// in registers.
//
// A row whose length is no multiple of V ends with its last V elements; those
// that the vector before has too are left out of the sums and of the stores.
//
// A thread has sixteen elements of 16 bits (eight of 32) where the row is long
// enough: what a row costs whatever its length (the steps of its reductions, its
// root and quotients, about 80 instructions a wave) is shared by twice the elements
// of one vector.  A root and two divisions of the compiler's would double it; the
// hardware's approximations take their place, the quotients' corrected once, the
// reciprocal root's (off by 2^-23 of it at most) as it is.
//
// Bound by memory.  Measured (one MI355X, other data from call to call): 409,600 x 256
// in f16 packed 59 us (5.4 TB/s), unpacked right after 52 (6.0; 60 where the last cache
// does not have the bytes; in f32 138, 3.8 TB/s), norm to y, bytes and rstd 97 (5.4;
// 137 with eight elements a thread and the compiler's divisions); 7744 x 1024 in bf16
// with the residual, its sum and bytes 11 us (5.0); the gradient of 307,039 x 100 in f32
// 75 us (4.9) and 4 for the join of dgamma; 4096 x 16384 in f16, a workgroup of 1024
// threads to a row and no load ahead, 90 (4.5).
#pragma once

#include "head/common.hpp"
#include "rows8/rows.hpp"

#pragma clang fp contract(fast)

namespace cpe {
namespace {

constexpr int kRowThreads = 256;

template <int LANES>
constexpr int row_threads() { return LANES <= 64 ? kRowThreads : LANES; }
template <int LANES>
constexpr int rows_at_once() { return LANES <= 64 ? kRowThreads / LANES : 1; }

// Waves of a SIMD, by the elements that a thread holds: the kernels are compiled
// for them, and the grids fill the chip with them.
constexpr int row_waves(int lanes, int elements) { return lanes > 256 ? 4 : elements <= 8 ? 6 : elements <= 16 ? 5 : 3; }
constexpr int grad_waves(int lanes, int elements) { return lanes > 256 ? 4 : elements <= 8 ? 5 : elements <= 16 ? 3 : 2; }
// Whether the next row's loads are in flight with the present one's work, and the
// gradient's gamma stays: not where the registers do not hold them, nor in the norm
// of longer rows, which writes as much as it reads (16,384 x 3000 in f32 packed 43 us
// with them, 54 without; normed and added to a residual 121 and 114).
constexpr bool row_ahead(int lanes, int elements, bool norm) { return lanes <= 256 || (elements <= 8 && !norm); }

// op over the LANES threads of a row, in a fixed order, for all of them.
// Steps 1, 2, 4 and 8 within rows of sixteen lanes by DPP (quads permuted, then
// mirrored halves, whose lanes are alike by then), 16 and 32 by the swaps of
// half waves.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 0xf, 0xf, false);
}
template <int LANES, typename V, typename Op>
__device__ __forceinline__ V wave_reduce(V v, Op op)
{
    static_assert(sizeof(V) == 4, "");
    auto bits = [](V x) { return __builtin_bit_cast(uint32_t, x); };
    auto value = [](uint32_t x) { return __builtin_bit_cast(V, x); };
    if constexpr (LANES >= 2) v = op(v, value(dpp<0xb1>(bits(v))));
    if constexpr (LANES >= 4) v = op(v, value(dpp<0x4e>(bits(v))));
    if constexpr (LANES >= 8) v = op(v, value(dpp<0x141>(bits(v))));
    if constexpr (LANES >= 16) v = op(v, value(dpp<0x140>(bits(v))));
    if constexpr (LANES >= 32) {
        const auto p = __builtin_amdgcn_permlane16_swap(bits(v), bits(v), false, false);
        v = op(value(p[0]), value(p[1]));
    }
    if constexpr (LANES >= 64) {
        const auto p = __builtin_amdgcn_permlane32_swap(bits(v), bits(v), false, false);
        v = op(value(p[0]), value(p[1]));
    }
    return v;
}
// turn: alternates from one call to the next, so that one barrier a call is enough.
template <int LANES, typename V, typename Op>
__device__ __forceinline__ V row_reduce(V v, Op op, int &turn)
{
    v = wave_reduce<(LANES < 64 ? LANES : 64)>(v, op);
    if constexpr (LANES > 64) {
        constexpr int kWaves = LANES / 64;
        __shared__ V lds[2][kWaves];
        if ((threadIdx.x & 63) == 0) lds[turn][threadIdx.x >> 6] = v;
        __syncthreads();
        v = lds[turn][0];
#pragma unroll
        for (int w = 1; w < kWaves; w++) v = op(v, lds[turn][w]);
        turn ^= 1;
    }
    return v;
}

// The vectors of a thread's share of a row: their first elements, how many of
// each one's elements another vector has (all where there is none), and masks
// of those that it has.
template <typename T, int V, int LANES, int N>
struct RowShare {
    static constexpr int kWords = (V * (int)sizeof(T) + 3) / 4;
    static constexpr bool kMasks = sizeof(T) < 4 && N <= 4;       // held in registers
    int at[N], extra[N];
    bool full;                                // no element is left out, in any thread
    uint32_t mask[kMasks ? N : 1][kWords];
    __device__ __forceinline__ RowShare(int width)
    {
        const int lane = threadIdx.x % LANES;
        full = width == LANES * N * V;
#pragma unroll
        for (int i = 0; i < N; i++) {
            const int c = (lane + i * LANES) * V;
            at[i] = c + V <= width ? c : c < width ? width - V : 0;
            extra[i] = c < width ? c - at[i] : V;
            if constexpr (kMasks)
#pragma unroll
                for (int w = 0; w < kWords; w++) mask[i][w] = word_mask(extra[i], w);
        }
    }
    __device__ __forceinline__ static uint32_t word_mask(int left_out, int w)
    {
        const int gone = left_out * (int)sizeof(T) - 4 * w;       // bytes of this word
        return gone <= 0 ? 0xffffffffu : gone >= 4 ? 0u : 0xffffffffu << (8 * gone);
    }
    // 0 in the place of what is left out, whatever was loaded there
    __device__ __forceinline__ Vec<T, V> own(int i, Vec<T, V> v) const
    {
        if (full) return v;
        uint32_t w[kWords] = {};
        __builtin_memcpy(w, &v, sizeof v);
#pragma unroll
        for (int j = 0; j < kWords; j++)
            if constexpr (sizeof(T) == 4)
                w[j] = j >= extra[i] ? w[j] : 0u;
            else
                w[j] &= kMasks ? mask[kMasks ? i : 0][j] : word_mask(extra[i], j);
        __builtin_memcpy(&v, w, sizeof v);
        return v;
    }
};

// The elements of a vector that are this thread's; PAST: past the caches.
template <bool PAST = false, typename T, int V>
__device__ __forceinline__ void store_own(T *p, const Vec<T, V> &v, int extra)
{
    if (extra == 0) {
        if constexpr (PAST)
            store_words<true>(p, v);
        else
            store_vec<T, V>(p, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < V; i++)
        if (i >= extra) p[i] = v.v[i];
}

// gamma of a thread's share, in registers: loaded after the first row's loads
template <int V, int N>
__device__ __forceinline__ void load_gamma(const float *gamma, const int (&at)[N], float (&g)[N][V])
{
#pragma unroll
    for (int i = 0; i < N; i++) {
        Vec<float, V> v;
        if (gamma) v = load_vec<float, V>(gamma + at[i]);
#pragma unroll
        for (int e = 0; e < V; e++) g[i][e] = gamma ? v.v[e] : 1.0f;
    }
}

// The scale s of a row whose largest |x| has these bits, and 1 / s.  Both
// divisions are products with a reciprocal, corrected once by the remainder
// (fma has it exactly): the division's own rounding for the scale, whose divisor
// is a constant, and for the reciprocal to 2^-24 and a trifle.
struct RowScale {
    float scale, inverse, divisor;            // of the quotients: the scale, or times 2^64
    bool bad;
    __device__ __forceinline__ explicit RowScale(uint32_t most)
    {
        bad = most >= 0x7f800000u;
        const float m = __builtin_bit_cast(float, most), t = m * (1.0f / 127.0f);
        scale = fmaxf(fmaf(fmaf(-127.0f, t, m), 1.0f / 127.0f, t), kLeastScale);
        const float r = __builtin_amdgcn_rcpf(scale);
        inverse = fmaf(fmaf(-scale, r, 1.0f), r, r);
        divisor = scale;
    }
    // Rows with a scale below 2^-100 are divided with both sides times 2^64: the last
    // bits of their remainders, down to 2^-48 of the scale's power of two, would lie
    // below 2^-149.  (Ordinary rows pay for the comparison: at most 1.5 % of the rows
    // that memory bounds, 0.6 us of 400,000 x 24 in f32, which the caches hold.)
    template <int N, int V>
    __device__ __forceinline__ void raise(float (&x)[N][V])
    {
        if (scale >= 0x1p-100f) return;
        divisor *= 0x1p64f;
        inverse *= 0x1p-64f;
#pragma unroll
        for (int i = 0; i < N; i++)
#pragma unroll
            for (int v = 0; v < V; v++) x[i][v] *= 0x1p64f;
    }
    __device__ __forceinline__ float stored() const { return bad ? __builtin_bit_cast(float, 0x7fc00000u) : scale; }
};

// rint(x / s) as signed bytes.  The quotient x / s is x times the rounded
// reciprocal, corrected once by its remainder: the division's own rounding, so
// that a value in the middle of two bytes (which 16-bit rows hold now and then:
// 254 x is an odd multiple of m) goes to the even one.  Adding 1.5 x 2^23 then
// leaves the whole number, rounded to nearest even, in the low bits.
template <int V>
__device__ __forceinline__ Vec<int8_t, V> to_bytes(const float (&x)[V], const RowScale &s)
{
    Vec<int8_t, V> o;
    uint32_t b[V];
#pragma unroll
    for (int i = 0; i < V; i++) {
        const float t = x[i] * s.inverse, quotient = fmaf(fmaf(-t, s.divisor, x[i]), s.inverse, t);
        b[i] = __builtin_bit_cast(uint32_t, quotient + 12582912.0f);
    }
    if constexpr (V % 4 == 0) {
        uint32_t w[V / 4];
#pragma unroll
        for (int i = 0; i < V / 4; i++) {
            w[i] = __builtin_amdgcn_perm(b[4 * i + 1], b[4 * i], 0x0c0c0400u) |
                   __builtin_amdgcn_perm(b[4 * i + 3], b[4 * i + 2], 0x04000c0cu);
            w[i] = s.bad ? 0u : w[i];
        }
        __builtin_memcpy(&o, w, V);
    } else {
#pragma unroll
        for (int i = 0; i < V; i++) o.v[i] = s.bad ? (int8_t)0 : (int8_t)(b[i] & 0xffu);
    }
    return o;
}

// NORM: RMS norm; otherwise y = x, packed only.
template <typename T, int V, int LANES, int N, bool NORM, bool PAST>
__global__ __launch_bounds__(row_threads<LANES>(), row_waves(LANES, N *V)) void k_rows(RowsArgs a)
{
    constexpr int R = rows_at_once<LANES>();
    const RowShare<T, V, LANES, N> share(a.width);
    const int group = LANES <= 64 ? (int)threadIdx.x / LANES : 0;
    const bool first_lane = threadIdx.x % LANES == 0;
    struct Raw {
        Vec<T, V> x[N], r[NORM ? N : 1];
    };
    auto fetch = [&](int64_t base) {
        Raw raw;
        const int64_t row = base + group < a.rows ? base + group : a.rows - 1;
#pragma unroll
        for (int i = 0; i < N; i++) {
            raw.x[i] = load_vec<T, V>(static_cast<const T *>(a.x) + row * a.ldx + share.at[i]);
            if constexpr (NORM)
                if (a.residual) raw.r[i] = load_vec<T, V>(static_cast<const T *>(a.residual) + row * a.ldr + share.at[i]);
        }
        return raw;
    };
    int turn = 0;
    constexpr bool AHEAD = row_ahead(LANES, N * V, NORM);
    const int64_t step = (int64_t)gridDim.x * R;
    int64_t base = (int64_t)blockIdx.x * R;
    [[maybe_unused]] Raw next;
    if constexpr (AHEAD) next = fetch(base);
    [[maybe_unused]] float gamma[N][V];
    if constexpr (NORM) load_gamma<V, N>(a.gamma, share.at, gamma);
    for (; base < a.rows; base += step) {
        const Raw raw = AHEAD ? next : fetch(base);
        if (AHEAD && base + step < a.rows) next = fetch(base + step);
        const int64_t row = base + group;
        const bool on = row < a.rows;
        float h[N][V];
        [[maybe_unused]] float squares = 0.0f;
#pragma unroll
        for (int i = 0; i < N; i++) {
            const Vec<T, V> x = share.own(i, raw.x[i]);
#pragma unroll
            for (int v = 0; v < V; v++) h[i][v] = (float)x.v[v];
            if constexpr (NORM) {
                if (a.residual) {
                    const Vec<T, V> r = share.own(i, raw.r[i]);
#pragma unroll
                    for (int v = 0; v < V; v++) h[i][v] = (float)rounded<T>(h[i][v] + (float)r.v[v]);
                }
#pragma unroll
                for (int v = 0; v < V; v++) squares = fmaf(h[i][v], h[i][v], squares);
                if (a.sum && on && share.extra[i] < V) {
                    Vec<T, V> o;
#pragma unroll
                    for (int v = 0; v < V; v++) o.v[v] = (T)h[i][v];
                    store_own<PAST, T, V>(static_cast<T *>(a.sum) + row * a.lds + share.at[i], o, share.extra[i]);
                }
            }
        }
        if constexpr (NORM) {
            squares = row_reduce<LANES>(squares, [](float p, float q) { return p + q; }, turn);
            const float rstd = __builtin_amdgcn_rsqf(fmaf(squares, a.inverse_width, a.eps));
            if (a.rstd && on && first_lane) a.rstd[row] = rstd;
#pragma unroll
            for (int i = 0; i < N; i++) {
#pragma unroll
                for (int v = 0; v < V; v++) h[i][v] = h[i][v] * rstd * gamma[i][v];
                if (a.y && on && share.extra[i] < V) {
                    Vec<T, V> o;
#pragma unroll
                    for (int v = 0; v < V; v++) o.v[v] = (T)h[i][v];
                    store_own<PAST, T, V>(static_cast<T *>(a.y) + row * a.ldy + share.at[i], o, share.extra[i]);
                }
            }
        }
        if (!a.q) continue;
        // the bits of |y|: infinities and NaNs are above every finite value
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < N; i++)
#pragma unroll
            for (int v = 0; v < V; v++) most = max(most, __builtin_bit_cast(uint32_t, h[i][v]) & 0x7fffffffu);
        most = row_reduce<LANES>(most, [](uint32_t p, uint32_t q) { return max(p, q); }, turn);
        RowScale s(most);
        if (!on) continue;
        if (first_lane) a.scale[row] = s.stored();
        if constexpr (NORM || !std::is_same<T, _Float16>::value) s.raise(h);      // (f16's scales are 2^-31 or more, or of zeros)
#pragma unroll
        for (int i = 0; i < N; i++)
            if (share.extra[i] < V)
                store_own<false, int8_t, V>(a.q + row * a.ldq + share.at[i], to_bytes<V>(h[i], s), share.extra[i]);
    }
}

// x = q s.  LANES neighbouring threads take a row, eight elements each at a time
// (or one, of narrow rows).
template <typename T, int V, int LANES, bool PAST>
__global__ __launch_bounds__(kRowThreads) void k_unpack(UnpackArgs a)
{
    constexpr int R = kRowThreads / LANES, U = 4;
    const int group = threadIdx.x / LANES, lane = threadIdx.x % LANES;
    const int chunk = blockIdx.y * (LANES * V) + lane * V;        // of columns
    if (chunk >= a.width) return;
    const int at = chunk + V <= a.width ? chunk : a.width - V, extra = chunk - at;
    const int64_t step = (int64_t)gridDim.x * R;
    for (int64_t r0 = (int64_t)blockIdx.x * R + group; r0 < a.rows; r0 += U * step) {
        Vec<int8_t, V> q[U];
        float s[U];
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int64_t row = r0 + u * step < a.rows ? r0 + u * step : r0;
            q[u] = load_vec<int8_t, V>(a.q + row * a.ldq + at);
            s[u] = a.fold ? scale_parts<true>(a.scale[row]).p : a.scale[row];
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int64_t row = r0 + u * step;
            if (row >= a.rows) break;
            Vec<T, V> o;
#pragma unroll
            for (int v = 0; v < V; v++) o.v[v] = scaled_byte<T>(q[u].v[v], s[u]);
            store_own<PAST, T, V>(static_cast<T *>(a.x) + row * a.ldx + at, o, extra);
        }
    }
}

// The gradient: dx row by row, as the forward; each thread sums its columns'
// part of dgamma over the rows that it sees, the workgroup over its threads, and
// k_rms_join over the workgroups.
template <typename T, int V, int LANES, int N, bool PACKED, bool PAST>
__global__ __launch_bounds__(row_threads<LANES>(), grad_waves(LANES, N *V)) void k_rms_grad(RmsGradArgs a)
{
    using H = std::conditional_t<PACKED, int8_t, T>;
    constexpr int R = rows_at_once<LANES>();
    const RowShare<T, V, LANES, N> share(a.width);
    const RowShare<H, V, LANES, N> h_share(a.width);
    const int group = LANES <= 64 ? (int)threadIdx.x / LANES : 0;
    struct Raw {
        Vec<H, V> h[N];
        Vec<T, V> d[N], s[N];
        float rstd, scale;
    };
    auto fetch = [&](int64_t base) {
        Raw raw;
        const int64_t row = base + group < a.rows ? base + group : a.rows - 1;
#pragma unroll
        for (int i = 0; i < N; i++) {
            raw.h[i] = load_vec<H, V>(static_cast<const H *>(a.h) + row * a.ldh + share.at[i]);
            raw.d[i] = load_vec<T, V>(static_cast<const T *>(a.dy) + row * a.ldd + share.at[i]);
            if (a.dsum) raw.s[i] = load_vec<T, V>(static_cast<const T *>(a.dsum) + row * a.lds + share.at[i]);
        }
        raw.rstd = a.rstd[row];
        raw.scale = PACKED ? a.h_scale[row] : 1.0f;
        return raw;
    };
    int turn = 0;
    constexpr bool AHEAD = row_ahead(LANES, N * V, false);
    const int64_t step = (int64_t)gridDim.x * R;
    int64_t base = (int64_t)blockIdx.x * R;
    [[maybe_unused]] Raw next;
    if (AHEAD && base < a.rows) next = fetch(base);
    float gamma[N][V], acc[N][V];
    if constexpr (AHEAD) load_gamma<V, N>(a.gamma, share.at, gamma);
#pragma unroll
    for (int i = 0; i < N; i++)
#pragma unroll
        for (int v = 0; v < V; v++) acc[i][v] = 0.0f;
    for (; base < a.rows; base += step) {
        Raw raw = AHEAD ? next : fetch(base);
        if (AHEAD && base + step < a.rows) next = fetch(base + step);
        const int64_t row = base + group;
        const bool on = row < a.rows;
        if (base + R > a.rows && !on) {         // (a row that is not there adds nothing)
            raw = Raw{};
        }
        if constexpr (!AHEAD) load_gamma<V, N>(a.gamma, share.at, gamma);
        const float to_xh = PACKED ? raw.scale * raw.rstd : raw.rstd;
        float xh[N][V], t[N][V], sum = 0.0f;
#pragma unroll
        for (int i = 0; i < N; i++) {
            const Vec<T, V> d = share.own(i, raw.d[i]);
            const Vec<H, V> h = h_share.own(i, raw.h[i]);
#pragma unroll
            for (int v = 0; v < V; v++) {
                xh[i][v] = (float)h.v[v] * to_xh;
                t[i][v] = (float)d.v[v] * gamma[i][v];
                sum = fmaf(t[i][v], xh[i][v], sum);
                acc[i][v] = fmaf((float)d.v[v], xh[i][v], acc[i][v]);
            }
        }
        if (!a.dx) continue;
        sum = row_reduce<LANES>(sum, [](float p, float q) { return p + q; }, turn) * a.inverse_width;
        if (!on) continue;
#pragma unroll
        for (int i = 0; i < N; i++) {
            Vec<T, V> o;
#pragma unroll
            for (int v = 0; v < V; v++) {
                float dx = raw.rstd * fmaf(-xh[i][v], sum, t[i][v]);
                if (a.dsum) dx += (float)raw.s[i].v[v];
                o.v[v] = (T)dx;
            }
            if (share.extra[i] < V)
                store_own<PAST, T, V>(static_cast<T *>(a.dx) + row * a.ldx + share.at[i], o, share.extra[i]);
        }
    }
    if (!a.dgamma) return;
    // (one workgroup has all the sums: there is nothing to join)
    float *part = a.blocks == 1 ? a.dgamma : a.part + (int64_t)blockIdx.x * a.width;
    if constexpr (R > 1) {
        // a wave's rows' sums first, by the lanes that have the same columns
        constexpr int kWaves = kRowThreads / 64;
        __shared__ float lds[kWaves][LANES * N * V];
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < N; i++)
#pragma unroll
            for (int v = 0; v < V; v++) {
                float s = acc[i][v];
#pragma unroll
                for (int d = LANES; d < 64; d *= 2) s += __shfl_xor(s, d);
                if (lane < LANES) lds[wave][(lane + i * LANES) * V + v] = s;
            }
        __syncthreads();
        for (int c = threadIdx.x; c < a.width; c += kRowThreads) {
            // (the last vector's elements are the last V of the row)
            const int first = a.width / V * V, at = c < first || a.width % V == 0 ? c : c + (V - a.width % V);
            float s = lds[0][at];
#pragma unroll
            for (int w = 1; w < kWaves; w++) s += lds[w][at];
            part[c] = s;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; i++)
#pragma unroll
            for (int v = 0; v < V; v++)
                if (v >= share.extra[i]) part[share.at[i] + v] = acc[i][v];
    }
}

// dgamma over the workgroups' partial sums: 32 columns (a cache line) per
// workgroup, 32 lanes of partials each.
__global__ __launch_bounds__(1024) void k_rms_join(RmsGradArgs a)
{
    __shared__ double lds[16][32];
    const int at = threadIdx.x & 31, c = blockIdx.x * 32 + at;
    double s = 0.0;
    if (c < a.width) {
#pragma unroll 8
        for (int i = threadIdx.x >> 5; i < a.blocks; i += 32) s += (double)a.part[(int64_t)i * a.width + c];
    }
    s += __shfl_xor(s, 32);
    if ((threadIdx.x & 63) < 32) lds[threadIdx.x >> 6][at] = s;
    __syncthreads();
    if (threadIdx.x < 32 && c < a.width) {
        s = 0.0;
        for (int w = 0; w < 16; w++) s += lds[w][at];
        a.dgamma[c] = (float)s;
    }
}

// -- launches -----------------------------------------------------------------------

template <typename T>
constexpr int kRowVec = 16 / (int)sizeof(T);

template <int V_, int LANES_, int N_>
struct RowForm {
    static constexpr int V = V_, LANES = LANES_, N = N_;
};

// call(form) for the first of these whose lanes hold the row; WIDEST: the
// vectors that a row may have.  GRAD: one vector a thread where a row takes several
// waves, so that the registers hold the next row's loads as well (4628 x 7488 in
// bf16 46 us, 73 with two and no load ahead; 8192 x 5000 in f16 51 and 68; 20,000 x
// 2048 in f32 95 and 98).  From packed rows it goes either way: 4628 x 7488 in bf16 55
// and 70, 20,000 x 2048 in f32 with the gradient past the norm 98 and 108, but 8192 x
// 5000 in f16 69 and 62, 16,384 x 2500 in bf16 72 and 61.  The forward is slower so
// (8192 x 5000 in f16 to bytes 60 us, 37 with two).
template <typename T, int WIDEST, bool GRAD, typename Call>
hipError_t with_row_form(int width, Call call)
{
    constexpr int V = kRowVec<T>;
    if (width < V) return call(RowForm<1, 8, 1>{});
    const int vectors = (width + V - 1) / V;
    if (vectors <= 8) return call(RowForm<V, 8, 1>{});
    if (vectors <= 16) return call(RowForm<V, 8, 2>{});
    if (vectors <= 32) return call(RowForm<V, 16, 2>{});
    if (vectors <= 64) return call(RowForm<V, 32, 2>{});
    if (vectors <= 128) return call(RowForm<V, 64, 2>{});
    if (vectors <= 256) return call(RowForm<V, 256, 1>{});
    if constexpr (GRAD) {
        if (vectors <= 512) return call(RowForm<V, 512, 1>{});
        if (vectors <= 1024) return call(RowForm<V, 1024, 1>{});
    } else {
        if (vectors <= 512) return call(RowForm<V, 256, 2>{});
        if (vectors <= 1024) return call(RowForm<V, 512, 2>{});
    }
    if (vectors <= 2048) return call(RowForm<V, 1024, 2>{});
    if constexpr (WIDEST > 2048)
        if (vectors <= 4096) return call(RowForm<V, 1024, 4>{});
    if constexpr (WIDEST > 4096)
        if (vectors <= 8192) return call(RowForm<V, 1024, 8>{});
    if constexpr (WIDEST > 8192)
        if (vectors <= 16384) return call(RowForm<V, 1024, 16>{});
    return hipErrorInvalidValue;
}

// Whether what a call writes goes past the caches: where its rows, `bytes` for
// each element, are more than the last cache holds, and the written ones are
// whole lines of 16-bit values (409,600 x 256 in f16: unpacking right after packing
// 50 us against 64, norm with y, q and rstd 97 against 100; 30,000 x 2048, which fits,
// norm 44 against 45 where nothing reads y, which would then find it in memory; f32
// unpacked in two stores a thread, half a line each, 55 against 28).  Bytes stay in
// the caches, for the product that reads them next.
constexpr int64_t kCacheBytes = (int64_t)256 << 20;
template <typename T>
bool goes_past(int64_t rows, int64_t width, int64_t bytes)
{
    return sizeof(T) == 2 && rows * width * bytes > kCacheBytes && width % 64 == 0;
}
template <typename T>
bool whole_lines(const void *p, int64_t ld) { return !p || (aligned_to(p, 128) && ld % 64 == 0); }

// As many workgroups as run at once, or fewer.
template <int LANES>
int64_t row_blocks(int64_t rows, int waves)
{
    const int64_t want = ceil_div(rows, rows_at_once<LANES>()), places = 256 * (waves * 4 * 64 / row_threads<LANES>());
    return want < places ? want : places;
}

template <typename T, bool NORM>
hipError_t launch_rows_type(RowsArgs a, hipStream_t stream)
{
    a.inverse_width = 1.0f / (float)a.width;
    const bool past = (a.sum || a.y) &&
                      goes_past<T>(a.rows, a.width, (1 + !!a.residual + !!a.sum + !!a.y) * (int)sizeof(T) + !!a.q) &&
                      whole_lines<T>(a.sum, a.lds) && whole_lines<T>(a.y, a.ldy);
    constexpr int kWidest = NORM ? kRmsMaxChannels : kRowsMaxWidth;
    return with_row_form<T, kWidest / kRowVec<T>, false>(a.width, [&](auto form) {
        using F = decltype(form);
        const dim3 grid((unsigned)row_blocks<F::LANES>(a.rows, row_waves(F::LANES, F::N * F::V)));
        constexpr bool kPast = NORM && F::V * sizeof(T) == 16 && sizeof(T) == 2;
        if (past)
            hipLaunchKernelGGL((k_rows<T, F::V, F::LANES, F::N, NORM, kPast>), grid, dim3(row_threads<F::LANES>()), 0,
                               stream, a);
        else
            hipLaunchKernelGGL((k_rows<T, F::V, F::LANES, F::N, NORM, false>), grid, dim3(row_threads<F::LANES>()), 0,
                               stream, a);
        return hipGetLastError();
    });
}
template <typename T>
hipError_t launch_pack_type(const RowsArgs &a, hipStream_t stream) { return launch_rows_type<T, false>(a, stream); }
template <typename T>
hipError_t launch_rms_type(const RowsArgs &a, hipStream_t stream) { return launch_rows_type<T, true>(a, stream); }

template <typename T>
hipError_t launch_rms_grad_type(RmsGradArgs a, hipStream_t stream)
{
    a.inverse_width = 1.0f / (float)a.width;
    const bool past = a.dx && whole_lines<T>(a.dx, a.ldx) &&
                      goes_past<T>(a.rows, a.width, (2 + !!a.dsum) * (int)sizeof(T) + (a.h_scale ? 1 : (int)sizeof(T)));
    const hipError_t e = with_row_form<T, kRmsMaxChannels / kRowVec<T>, true>(a.width, [&](auto form) {
        using F = decltype(form);
        // (of no rows: one workgroup, whose partial sums are 0)
        const int64_t want = row_blocks<F::LANES>(a.rows > 0 ? a.rows : 1, grad_waves(F::LANES, F::N * F::V));
        a.blocks = rms_grad_blocks(want, a.width, F::LANES, a.dgamma != nullptr);
        const dim3 grid(a.blocks), block(row_threads<F::LANES>());
        constexpr bool kPast = F::V * sizeof(T) == 16 && sizeof(T) == 2;
        auto launch = [&](auto packed, auto beyond) {
            hipLaunchKernelGGL((k_rms_grad<T, F::V, F::LANES, F::N, decltype(packed)::value, decltype(beyond)::value>),
                               grid, block, 0, stream, a);
        };
        if (a.h_scale && past)
            launch(std::true_type{}, std::integral_constant<bool, kPast>{});
        else if (a.h_scale)
            launch(std::true_type{}, std::false_type{});
        else if (past)
            launch(std::false_type{}, std::integral_constant<bool, kPast>{});
        else
            launch(std::false_type{}, std::false_type{});
        return hipGetLastError();
    });
    if (e != hipSuccess || !a.dgamma || a.blocks == 1) return e;
    hipLaunchKernelGGL(k_rms_join, dim3((unsigned)ceil_div(a.width, 32)), dim3(1024), 0, stream, a);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_unpack_type(const UnpackArgs &a, hipStream_t stream)
{
    const bool past = goes_past<T>(a.rows, a.width, sizeof(T) + 1) && whole_lines<T>(a.x, a.ldx);
    auto launch = [&](auto vec, auto lanes) {
        constexpr int V = decltype(vec)::value, LANES = decltype(lanes)::value;
        const int64_t columns = ceil_div(a.width, LANES * V), places = ceil_div(2048, columns);
        const int64_t want = ceil_div(a.rows, kRowThreads / LANES * 4);       // (4 rows of a thread in flight)
        const dim3 grid((unsigned)(want < places ? want : places), (unsigned)columns);
        if (past)
            hipLaunchKernelGGL((k_unpack<T, V, LANES, V * sizeof(T) == 16>), grid, dim3(kRowThreads), 0, stream, a);
        else
            hipLaunchKernelGGL((k_unpack<T, V, LANES, false>), grid, dim3(kRowThreads), 0, stream, a);
        return hipGetLastError();
    };
    using std::integral_constant;
    if (a.width < 8) return launch(integral_constant<int, 1>{}, integral_constant<int, 8>{});
    if (a.width <= 64) return launch(integral_constant<int, 8>{}, integral_constant<int, 8>{});
    if (a.width <= 128) return launch(integral_constant<int, 8>{}, integral_constant<int, 16>{});
    if (a.width <= 256) return launch(integral_constant<int, 8>{}, integral_constant<int, 32>{});
    return launch(integral_constant<int, 8>{}, integral_constant<int, 64>{});
}

}  // namespace
}  // namespace cpe
