// k_rows.hpp -- kernels that work row by row: packing rows into 8 bits, RMS
// norm with the residual's addition, its gradient (private to the library;
// included once per element type).
//
// A row belongs to LANES neighbouring threads, N vectors of V elements each,
// and stays in their registers between its reduction and what is written: each
// input is read once.  Up to 64 lanes a row's sums pass between the lanes of
// its wave, beyond that through LDS.  Workgroups take rows in turn, with the
// next row's loads in flight while the present one is worked on; gamma stays
// in registers.
//
// A row whose length is no multiple of V ends with its last V elements; those
// that the vector before has too are left out of the sums and of the stores.
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

// The vectors of a thread's share of a row: their first elements, and how many
// of each one's elements another vector has (all where there is none).
template <int V, int LANES, int N>
struct RowShare {
    int at[N], extra[N];
    __device__ __forceinline__ RowShare(int width)
    {
        const int lane = threadIdx.x % LANES;
#pragma unroll
        for (int i = 0; i < N; i++) {
            const int c = (lane + i * LANES) * V;
            at[i] = c + V <= width ? c : c < width ? width - V : 0;
            extra[i] = c < width ? c - at[i] : V;
        }
    }
};

template <typename T, int V>
__device__ __forceinline__ void store_own(T *p, const Vec<T, V> &v, int extra)
{
    if (extra == 0) {
        store_vec<T, V>(p, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < V; i++)
        if (i >= extra) p[i] = v.v[i];
}

// The scale s of a row whose largest |x| has these bits, and 1 / s.
struct RowScale {
    float scale, inverse;
    bool bad;
    __device__ __forceinline__ explicit RowScale(uint32_t most)
    {
        bad = most >= 0x7f800000u;
        scale = fmaxf(__builtin_bit_cast(float, most) / 127.0f, kLeastScale);
        inverse = 1.0f / scale;
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
        const float t = x[i] * s.inverse, quotient = fmaf(fmaf(-t, s.scale, x[i]), s.inverse, t);
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
template <typename T, int V, int LANES, int N, bool NORM>
__global__ __launch_bounds__(row_threads<LANES>()) void k_rows(RowsArgs a)
{
    constexpr int R = rows_at_once<LANES>();
    const RowShare<V, LANES, N> share(a.width);
    const int group = LANES <= 64 ? (int)threadIdx.x / LANES : 0;
    const bool first_lane = threadIdx.x % LANES == 0;
    float gamma[N][V];
    if constexpr (NORM) {
#pragma unroll
        for (int i = 0; i < N; i++)
#pragma unroll
            for (int v = 0; v < V; v++) gamma[i][v] = a.gamma ? a.gamma[share.at[i] + v] : 1.0f;
    }
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
    const int64_t step = (int64_t)gridDim.x * R;
    int64_t base = (int64_t)blockIdx.x * R;
    Raw next = fetch(base);
    for (; base < a.rows; base += step) {
        const Raw raw = next;
        if (base + step < a.rows) next = fetch(base + step);
        const int64_t row = base + group;
        const bool on = row < a.rows;
        float h[N][V];
        [[maybe_unused]] float squares = 0.0f;
#pragma unroll
        for (int i = 0; i < N; i++) {
            Vec<T, V> o;
#pragma unroll
            for (int v = 0; v < V; v++) {
                float x = (float)raw.x[i].v[v];
                if constexpr (NORM) {
                    if (a.residual) x = (float)rounded<T>(x + (float)raw.r[i].v[v]);
                }
                h[i][v] = v >= share.extra[i] ? x : 0.0f;
                if constexpr (NORM) {
                    squares = fmaf(h[i][v], h[i][v], squares);
                    o.v[v] = (T)x;
                }
            }
            if constexpr (NORM)
                if (a.sum && on && share.extra[i] < V)
                    store_own<T, V>(static_cast<T *>(a.sum) + row * a.lds + share.at[i], o, share.extra[i]);
        }
        if constexpr (NORM) {
            squares = row_reduce<LANES>(squares, [](float p, float q) { return p + q; }, turn);
            const float rstd = 1.0f / sqrtf(squares / (float)a.width + a.eps);
            if (a.rstd && on && first_lane) a.rstd[row] = rstd;
#pragma unroll
            for (int i = 0; i < N; i++) {
                Vec<T, V> o;
#pragma unroll
                for (int v = 0; v < V; v++) {
                    h[i][v] = h[i][v] * rstd * gamma[i][v];
                    o.v[v] = (T)h[i][v];
                }
                if (a.y && on && share.extra[i] < V)
                    store_own<T, V>(static_cast<T *>(a.y) + row * a.ldy + share.at[i], o, share.extra[i]);
            }
        }
        if (!a.q) continue;
        // the bits of |y|: infinities and NaNs are above every finite value
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < N; i++)
#pragma unroll
            for (int v = 0; v < V; v++) {
                const uint32_t b = __builtin_bit_cast(uint32_t, h[i][v]) & 0x7fffffffu;
                // (left-out elements are 0 times what a row may hold)
                most = v >= share.extra[i] && b > most ? b : most;
            }
        most = row_reduce<LANES>(most, [](uint32_t p, uint32_t q) { return p > q ? p : q; }, turn);
        const RowScale s(most);
        if (!on) continue;
        if (first_lane) a.scale[row] = s.stored();
#pragma unroll
        for (int i = 0; i < N; i++)
            if (share.extra[i] < V)
                store_own<int8_t, V>(a.q + row * a.ldq + share.at[i], to_bytes<V>(h[i], s), share.extra[i]);
    }
}

// x = q s.  A thread takes 16 neighbouring elements of a row (or one, of narrow
// rows) at a time.
template <typename T, int V>
__global__ __launch_bounds__(kRowThreads) void k_unpack(UnpackArgs a)
{
    const int per_row = (a.width + V - 1) / V;
    const int64_t all = (int64_t)a.rows * per_row, step = (int64_t)gridDim.x * kRowThreads;
    for (int64_t i = (int64_t)blockIdx.x * kRowThreads + threadIdx.x; i < all; i += step) {
        const int64_t row = i / per_row;
        const int c = (int)(i - row * per_row) * V, at = c + V <= a.width ? c : a.width - V;
        const float s = a.scale[row];
        const Vec<int8_t, V> q = load_vec<int8_t, V>(a.q + row * a.ldq + at);
        Vec<T, V> o;
#pragma unroll
        for (int v = 0; v < V; v++) o.v[v] = scaled_byte<T>(q.v[v], s);
        store_own<T, V>(static_cast<T *>(a.x) + row * a.ldx + at, o, c - at);
    }
}

// The gradient: dx row by row, as the forward; each thread sums its columns'
// part of dgamma over the rows that it sees, the workgroup over its threads, and
// k_rms_join over the workgroups.
template <typename T, int V, int LANES, int N, bool PACKED>
__global__ __launch_bounds__(row_threads<LANES>()) void k_rms_grad(RmsGradArgs a)
{
    using H = std::conditional_t<PACKED, int8_t, T>;
    constexpr int R = rows_at_once<LANES>();
    const RowShare<V, LANES, N> share(a.width);
    const int group = LANES <= 64 ? (int)threadIdx.x / LANES : 0;
    float gamma[N][V], acc[N][V];
#pragma unroll
    for (int i = 0; i < N; i++)
#pragma unroll
        for (int v = 0; v < V; v++) {
            gamma[i][v] = a.gamma ? a.gamma[share.at[i] + v] : 1.0f;
            acc[i][v] = 0.0f;
        }
    struct Raw {
        Vec<H, V> h[N];
        Vec<T, V> d[N], s[N];
        float rstd, scale;
    };
    auto fetch = [&](int64_t base) {
        Raw raw;
        const int64_t row = base + group < a.rows ? base + group : a.rows - 1;
        raw.rstd = a.rstd[row];
        raw.scale = PACKED ? a.h_scale[row] : 1.0f;
#pragma unroll
        for (int i = 0; i < N; i++) {
            raw.h[i] = load_vec<H, V>(static_cast<const H *>(a.h) + row * a.ldh + share.at[i]);
            raw.d[i] = load_vec<T, V>(static_cast<const T *>(a.dy) + row * a.ldd + share.at[i]);
            if (a.dsum) raw.s[i] = load_vec<T, V>(static_cast<const T *>(a.dsum) + row * a.lds + share.at[i]);
        }
        return raw;
    };
    int turn = 0;
    const int64_t step = (int64_t)gridDim.x * R;
    int64_t base = (int64_t)blockIdx.x * R;
    Raw next{};
    if (base < a.rows) next = fetch(base);
    for (; base < a.rows; base += step) {
        const Raw raw = next;
        if (base + step < a.rows) next = fetch(base + step);
        const int64_t row = base + group;
        const bool on = row < a.rows;
        float xh[N][V], t[N][V], sum = 0.0f;
#pragma unroll
        for (int i = 0; i < N; i++)
#pragma unroll
            for (int v = 0; v < V; v++) {
                const bool own = on && v >= share.extra[i];
                const float d = (float)raw.d[i].v[v], x = (float)raw.h[i].v[v];
                xh[i][v] = (PACKED ? x * raw.scale : x) * raw.rstd;
                t[i][v] = d * gamma[i][v];
                sum += own ? t[i][v] * xh[i][v] : 0.0f;
                acc[i][v] += own ? d * xh[i][v] : 0.0f;
            }
        if (!a.dx) continue;
        sum = row_reduce<LANES>(sum, [](float p, float q) { return p + q; }, turn) / (float)a.width;
        if (!on) continue;
#pragma unroll
        for (int i = 0; i < N; i++) {
            Vec<T, V> o;
#pragma unroll
            for (int v = 0; v < V; v++) {
                float dx = raw.rstd * (t[i][v] - xh[i][v] * sum);
                if (a.dsum) dx += (float)raw.s[i].v[v];
                o.v[v] = (T)dx;
            }
            if (share.extra[i] < V)
                store_own<T, V>(static_cast<T *>(a.dx) + row * a.ldx + share.at[i], o, share.extra[i]);
        }
    }
    if (!a.dgamma) return;
    float *part = a.part + (int64_t)blockIdx.x * a.width;
    if constexpr (R > 1) {
        __shared__ float lds[R][LANES * N * V];
#pragma unroll
        for (int i = 0; i < N; i++)
#pragma unroll
            for (int v = 0; v < V; v++) lds[group][(threadIdx.x % LANES + i * LANES) * V + v] = acc[i][v];
        __syncthreads();
        for (int c = threadIdx.x; c < a.width; c += kRowThreads) {
            // (the last vector's elements are the last V of the row)
            const int first = a.width / V * V, at = c < first || a.width % V == 0 ? c : c + (V - a.width % V);
            float s = lds[0][at];
#pragma unroll
            for (int r = 1; r < R; r++) s += lds[r][at];
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
// vectors that a row may have.
template <typename T, int WIDEST, typename Call>
hipError_t with_row_form(int width, Call call)
{
    constexpr int V = kRowVec<T>;
    if (width < V) return call(RowForm<1, 8, 1>{});
    const int vectors = (width + V - 1) / V;
    if (vectors <= 8) return call(RowForm<V, 8, 1>{});
    if (vectors <= 16) return call(RowForm<V, 16, 1>{});
    if (vectors <= 32) return call(RowForm<V, 32, 1>{});
    if (vectors <= 64) return call(RowForm<V, 64, 1>{});
    if (vectors <= 128) return call(RowForm<V, 64, 2>{});
    if (vectors <= 256) return call(RowForm<V, 256, 1>{});
    if (vectors <= 512) return call(RowForm<V, 256, 2>{});
    if (vectors <= 1024) return call(RowForm<V, 1024, 1>{});
    if (vectors <= 2048) return call(RowForm<V, 1024, 2>{});
    if constexpr (WIDEST > 2048)
        if (vectors <= 4096) return call(RowForm<V, 1024, 4>{});
    if constexpr (WIDEST > 4096)
        if (vectors <= 8192) return call(RowForm<V, 1024, 8>{});
    if constexpr (WIDEST > 8192)
        if (vectors <= 16384) return call(RowForm<V, 1024, 16>{});
    return hipErrorInvalidValue;
}

// As many workgroups as run at once, or fewer.
template <int LANES>
unsigned row_blocks(int64_t rows, int64_t most)
{
    const int64_t want = ceil_div(rows, rows_at_once<LANES>());
    return (unsigned)(want < most ? want : most);
}
constexpr int row_places(int threads) { return 256 * (2048 / threads); }

template <typename T>
hipError_t launch_pack_type(const RowsArgs &a, hipStream_t stream)
{
    return with_row_form<T, kRowsMaxWidth / kRowVec<T>>(a.width, [&](auto form) {
        using F = decltype(form);
        constexpr int kThreads = row_threads<F::LANES>();
        const dim3 grid(row_blocks<F::LANES>(a.rows, row_places(kThreads)));
        hipLaunchKernelGGL((k_rows<T, F::V, F::LANES, F::N, false>), grid, dim3(kThreads), 0, stream, a);
        return hipGetLastError();
    });
}

template <typename T>
hipError_t launch_rms_type(const RowsArgs &a, hipStream_t stream)
{
    return with_row_form<T, kRmsMaxChannels / kRowVec<T>>(a.width, [&](auto form) {
        using F = decltype(form);
        constexpr int kThreads = row_threads<F::LANES>();
        const dim3 grid(row_blocks<F::LANES>(a.rows, row_places(kThreads)));
        hipLaunchKernelGGL((k_rows<T, F::V, F::LANES, F::N, true>), grid, dim3(kThreads), 0, stream, a);
        return hipGetLastError();
    });
}

template <typename T>
hipError_t launch_rms_grad_type(RmsGradArgs a, hipStream_t stream)
{
    const hipError_t e = with_row_form<T, kRmsMaxChannels / kRowVec<T>>(a.width, [&](auto form) {
        using F = decltype(form);
        constexpr int kThreads = row_threads<F::LANES>();
        const int64_t places = row_places(kThreads), most = rms_most_blocks(a.width);
        // (of no rows: one workgroup, whose partial sums are 0)
        a.blocks = (int32_t)row_blocks<F::LANES>(a.rows > 0 ? a.rows : 1, places < most ? places : most);
        if (a.h_scale)
            hipLaunchKernelGGL((k_rms_grad<T, F::V, F::LANES, F::N, true>), dim3(a.blocks), dim3(kThreads), 0, stream, a);
        else
            hipLaunchKernelGGL((k_rms_grad<T, F::V, F::LANES, F::N, false>), dim3(a.blocks), dim3(kThreads), 0, stream,
                               a);
        return hipGetLastError();
    });
    if (e != hipSuccess || !a.dgamma) return e;
    hipLaunchKernelGGL(k_rms_join, dim3((unsigned)ceil_div(a.width, 32)), dim3(1024), 0, stream, a);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_unpack_type(const UnpackArgs &a, hipStream_t stream)
{
    auto launch = [&](auto vec) {
        constexpr int V = decltype(vec)::value;
        const int64_t blocks = ceil_div((int64_t)a.rows * ceil_div(a.width, V), kRowThreads);
        const int64_t most = row_places(kRowThreads);
        hipLaunchKernelGGL((k_unpack<T, V>), dim3((unsigned)(blocks < most ? blocks : most)), dim3(kRowThreads), 0,
                           stream, a);
        return hipGetLastError();
    };
    if (a.width < 8) return launch(std::integral_constant<int, 1>{});
    return launch(std::integral_constant<int, 8>{});
}

}  // namespace
}  // namespace cpe
