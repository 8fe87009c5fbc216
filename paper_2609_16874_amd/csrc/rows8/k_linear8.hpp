// k_linear8.hpp -- integer matrix products on the matrix cores, with scales
// for rows and columns in the epilogue (private to the library; included once
// per output type).
//
// z = (sum_k A(m, k) B(n, k)) s_m t_n + bias_n, y = act(z) + residual, A and B
// signed bytes, both stored along k.  A fragment is 16 bytes of k per lane and
// operand, and one pair feeds a 16x16x64 instruction.  As in the products of
// 16 bits (whose LDS layout this shares: rows of 128 bytes of k, chunk c of row
// r at place c ^ (r & 7)) the B fragment goes first, so that a lane's four sums
// are neighbouring n of one row m.
//
// The sums are whole numbers below 2^31 (65536 x 2^14), so their order does not
// matter and splits of k join exactly.  They are rounded to binary32 once,
// then scaled: three roundings of 2^-24 in all.
#pragma once

#include "head/k_linear.hpp"
#include "rows8/linear8.hpp"

namespace cpe {
namespace {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

union Bytes16 {
    u32x4 u;
    i32x4 i;
};

__device__ __forceinline__ i32x4 mma8(const Bytes16 &n, const Bytes16 &m, i32x4 acc)
{
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(n.i, m.i, acc, 0, 0, 0);
}

// R rows by kStep8 of k of one operand, loaded by THREADS threads; DIRECT:
// straight into LDS through a buffer descriptor, as the products of 16 bits.
template <int R, int THREADS, bool DIRECT>
struct ByteOperand {
    static constexpr int kLoads = R * 8 / THREADS, kBytes = R * kStep8;
    const int8_t *base;
    uint32_t off[DIRECT ? kLoads : 1];
    const int8_t *src[DIRECT ? 1 : kLoads];
    bool there[DIRECT ? 1 : kLoads];
    u32x4 held[DIRECT ? 1 : kLoads];

    __device__ __forceinline__ static int row_of(int i) { return (i * THREADS + threadIdx.x) / 8; }
    __device__ __forceinline__ static int chunk_of(int i) { return (threadIdx.x & 7) ^ (row_of(i) & 7); }

    __device__ __forceinline__ void init(const void *p, int64_t ld, int r0, int r_end, int k0)
    {
        base = static_cast<const int8_t *>(p) + r0 * ld + k0;
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const int row = row_of(i), c = chunk_of(i);
            if constexpr (DIRECT) {
                off[i] = r0 + row < r_end ? (uint32_t)(row * ld + c * 16) : kBufferBytes;
            } else {
                there[i] = r0 + row < r_end;
                src[i] = base + row * ld + c * 16;
            }
        }
    }
    // the next step into LDS, or into registers; TAIL: only `left` k of it exist
    template <bool TAIL>
    __device__ __forceinline__ void fetch(lds_byte *lds, int left)
    {
        if constexpr (DIRECT) {
#ifdef __HIP_DEVICE_COMPILE__       // (the host's pass does not know the descriptor's type)
            const auto buffer =
                __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(base), 0, (int)kBufferBytes, 0x00027000);
#pragma unroll
            for (int i = 0; i < kLoads; i++) {
                uint32_t at = off[i];
                if constexpr (TAIL) at = chunk_of(i) * 16 < left ? at : kBufferBytes;
                lds_byte *to = lds + (i * THREADS + wave_base()) * 16;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer, (__attribute__((address_space(3))) void *)to, 16, at,
                                                         0, 0, 0);
            }
#endif
            base += kStep8;
        } else {
#pragma unroll
            for (int i = 0; i < kLoads; i++) {
                held[i] = load_chunk<int8_t>(src[i], there[i] ? left - chunk_of(i) * 16 : 0);
                src[i] += kStep8;
            }
        }
    }
    __device__ __forceinline__ void commit(lds_byte *lds) const
    {
        if constexpr (!DIRECT)
#pragma unroll
            for (int i = 0; i < kLoads; i++)
                *(__attribute__((address_space(3))) u32x4 *)(lds + (i * THREADS + threadIdx.x) * 16) = held[i];
    }
    // the fragment of rows r .. r+15 for the s-th half of the step
    __device__ __forceinline__ static Bytes16 read(const lds_byte *lds, int r, int s)
    {
        const int lane = threadIdx.x & 63, row = r + (lane & 15), c = (4 * s + (lane >> 4)) ^ (row & 7);
        Bytes16 f;
        f.u = *(const __attribute__((address_space(3))) u32x4 *)(lds + (row * 8 + c) * 16);
        return f;
    }
};

// W neighbouring sums of row m, scaled, then the epilogue of the other products.
template <int ACT, typename T, int W>
__device__ __forceinline__ void finish8(const Gemm8Args &a, int m, int n, const int32_t (&sum)[W])
{
    const float s = a.a_scale[m];
    float v[W];
    if (a.g.n - n >= W) {
        const Vec<float, W> t = load_vec<float, W>(a.b_scale + n);
#pragma unroll
        for (int i = 0; i < W; i++) v[i] = (float)sum[i] * s * t.v[i];
    } else {
#pragma unroll
        for (int i = 0; i < W; i++) v[i] = n + i < a.g.n ? (float)sum[i] * s * a.b_scale[n + i] : 0.0f;
    }
    finish<ACT, T, W>(a.g, m, n, v);
}

// Tiles of TM x TN outputs, two LDS tiles of kStep8 k, WM x WN waves.  The
// steps go as in the products of 16 bits: a step's two halves of fragments
// alternate in registers, the waves meet once a step, and at the meeting the
// next step's LDS tile has arrived.
template <int TM, int TN, int WM, int WN, bool DIRECT, typename T, int ACT>
__global__ __launch_bounds__(WM *WN * 64, 2) void k_gemm8(Gemm8Args args)
{
    constexpr int kThreads = WM * WN * 64;
    using A = ByteOperand<TM, kThreads, DIRECT>;
    using B = ByteOperand<TN, kThreads, DIRECT>;
    constexpr int kStage = A::kBytes + B::kBytes, FM = TM / WM / 16, FN = TN / WN / 16;
    extern __shared__ __align__(1024) unsigned char gemm8_lds[];
    const GemmArgs &g = args.g;
    const int tiles = g.tiles_m * g.tiles_n;
    const int split = blockIdx.x / tiles, tile = xcd_order(blockIdx.x - split * tiles, tiles);
    // bands of rows of tiles, down then across: tiles at work together share
    // both operands in the XCD's L2
    constexpr int kRowsOfBand = kBand * kTile / TM;
    const int band = tile / (kRowsOfBand * g.tiles_n), in_band = tile - band * kRowsOfBand * g.tiles_n;
    const int high = g.tiles_m - band * kRowsOfBand < kRowsOfBand ? g.tiles_m - band * kRowsOfBand : kRowsOfBand;
    const int m0 = (band * kRowsOfBand + in_band % high) * TM, n0 = in_band / high * TN;
    const int k0 = split * g.k_split;
    const int len = g.k - k0 < g.k_split ? g.k - k0 : g.k_split;
    const int steps = (len + kStep8 - 1) / kStep8, whole = len / kStep8;
    const int wave = wave_base() >> 6, lane = threadIdx.x & 63;
    const int wm = (wave / WN) * (TM / WM), wn = (wave % WN) * (TN / WN);
    lds_byte *lds = (lds_byte *)gemm8_lds;
    A a;
    B b;
    a.init(g.a, g.lda, m0, g.m, k0);
    b.init(g.b, g.ldb, n0, g.n, k0);
    i32x4 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; i++)
#pragma unroll
        for (int j = 0; j < FN; j++) acc[i][j] = i32x4{0, 0, 0, 0};
    auto fetch = [&](auto tail, int step) __attribute__((always_inline)) {
        constexpr bool TAIL = decltype(tail)::value;
        lds_byte *to = lds + (step & 1) * kStage;
        a.template fetch<TAIL>(to, len - step * kStep8);
        b.template fetch<TAIL>(to + A::kBytes, len - step * kStep8);
    };
    auto fetch_any = [&](int step) __attribute__((always_inline)) {
        if (step < whole)
            fetch(std::false_type{}, step);
        else
            fetch(std::true_type{}, step);
    };
    auto commit = [&](int step) {
        a.commit(lds + (step & 1) * kStage);
        b.commit(lds + (step & 1) * kStage + A::kBytes);
    };
    Bytes16 fa[2][FM], fb[2][FN];
    auto read = [&](int step, int half) {
        const lds_byte *la = lds + (step & 1) * kStage, *lb = la + A::kBytes;
#pragma unroll
        for (int i = 0; i < FM; i++) fa[half][i] = A::read(la, wm + 16 * i, half);
#pragma unroll
        for (int j = 0; j < FN; j++) fb[half][j] = B::read(lb, wn + 16 * j, half);
    };
    auto multiply = [&](int half) {
#pragma unroll
        for (int i = 0; i < FM; i++)
#pragma unroll
            for (int j = 0; j < FN; j++) acc[i][j] = mma8(fb[half][j], fa[half][i], acc[i][j]);
    };
    // (a split has one step at least)
    fetch_any(0);
    commit(0);
    wait_for_lds<true>();
    meet();
    if (steps > 1) fetch_any(1);
    read(0, 0);
    int t = 0;
    for (; t + 2 < whole; t++) {        // the steps whose loads are whole: no branch
        wait_for_lds<false>();          // the fragments of the first half
        __builtin_amdgcn_sched_barrier(0);
        read(t, 1);
        multiply(0);
        __builtin_amdgcn_sched_barrier(0);
        commit(t + 1);
        wait_for_lds<true>();
        meet();
        __builtin_amdgcn_sched_barrier(0);
        fetch(std::false_type{}, t + 2);
        read(t + 1, 0);
        multiply(1);
        __builtin_amdgcn_sched_barrier(0);
    }
    for (; t < steps; t++) {
        const bool more = t + 1 < steps;
        read(t, 1);
        multiply(0);
        if (more) commit(t + 1);
        wait_for_lds<true>();
        meet();
        if (t + 2 < steps) fetch_any(t + 2);
        if (more) read(t + 1, 0);
        multiply(1);
    }
    // no load is in flight, and every wave has read its last fragments: the sums
    // pass through LDS, 128 x 128 of them at a time, so that rows leave as whole lines
    typedef __attribute__((address_space(3))) i32x4 lds_quad;
    auto place = [&](int m, int n) { return (lds_quad *)(lds + (m * (TN / 4) + ((n >> 2) ^ (m & 15))) * 16); };
    constexpr int kPassRows = 2 * kStage / (TN * 4) < TM ? 2 * kStage / (TN * 4) : TM;      // that LDS holds
    static_assert(TM % kPassRows == 0 && kPassRows % (TM / WM) == 0, "");
    const int64_t ldpart = (g.n + 3) / 4 * 4;
#pragma unroll 1
    for (int p = 0; p < TM; p += kPassRows) {
        if (p > 0) __syncthreads();
        if (wm >= p && wm < p + kPassRows)
#pragma unroll
            for (int i = 0; i < FM; i++)
#pragma unroll
                for (int j = 0; j < FN; j++)
                    *place(wm - p + 16 * i + (lane & 15), wn + 16 * j + 4 * (lane >> 4)) = acc[i][j];
        __syncthreads();
        for (int q = threadIdx.x; q < kPassRows * TN / 8; q += kThreads) {
            const int r = q / (TN / 8), c = q % (TN / 8) * 8, m = m0 + p + r, n = n0 + c;
            if (m >= g.m || n >= g.n) continue;
            const i32x4 v0 = *place(r, c), v1 = *place(r, c + 4);
            if (g.splits > 1) {
                int32_t *to = reinterpret_cast<int32_t *>(g.part) + ((int64_t)split * g.m + m) * ldpart + n;
                *reinterpret_cast<i32x4 *>(to) = v0;
                if (n + 4 < g.n) *reinterpret_cast<i32x4 *>(to + 4) = v1;
            } else {
                const int32_t v[8] = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
                finish8<ACT, T, 8>(args, m, n, v);
            }
        }
    }
}

// The splits' partial sums added, then the epilogue.
template <typename T, int ACT>
__global__ __launch_bounds__(256) void k_gemm8_join(Gemm8Args a)
{
    const int quads = (a.g.n + 3) / 4;
    const int64_t all = (int64_t)a.g.m * quads, q = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (q >= all) return;
    const int32_t *p = reinterpret_cast<const int32_t *>(a.g.part) + q * 4;
    i32x4 v = {0, 0, 0, 0};
#pragma unroll 4
    for (int s = 0; s < a.g.splits; s++) v += *reinterpret_cast<const i32x4 *>(p + s * all * 4);
    const int m = (int)(q / quads);
    const int32_t w[4] = {v[0], v[1], v[2], v[3]};
    finish8<ACT, T, 4>(a, m, (int)(q - (int64_t)m * quads) * 4, w);
}

// Few rows: 16 n per workgroup, its waves dividing k; fragments come straight
// from memory, since no other workgroup shares the weights and the rows stay in
// the caches.
template <int MT, typename T, int ACT>
__global__ __launch_bounds__(1024) void k_gemm8_rows(Gemm8Args a)
{
    __shared__ i32x4 joined[16][MT][64];
    constexpr int kStep = 64;
    const GemmArgs &g = a.g;
    const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6, lane = threadIdx.x & 63;
    const int j = lane & 15, c = lane >> 4, n = blockIdx.x * 16 + j;
    const int steps = (g.k + kStep - 1) / kStep, each = (steps + waves - 1) / waves;
    const int lo = wave * each, hi = lo + each < steps ? lo + each : steps;
    const int8_t *pb = static_cast<const int8_t *>(g.b) + (int64_t)n * g.ldb;
    i32x4 acc[MT];
#pragma unroll
    for (int i = 0; i < MT; i++) acc[i] = i32x4{0, 0, 0, 0};
    constexpr int U = 4;
    for (int s = lo; s < hi; s += U) {
        Bytes16 fb[U], fa[U][MT];
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int k = (s + u) * kStep + c * 16, left = s + u < hi ? g.k - k : 0;
            fb[u].u = load_chunk<int8_t>(pb + k, n < g.n ? left : 0);
#pragma unroll
            for (int i = 0; i < MT; i++) {
                const int m = 16 * i + j;
                fa[u][i].u = load_chunk<int8_t>(static_cast<const int8_t *>(g.a) + m * g.lda + k, m < g.m ? left : 0);
            }
        }
#pragma unroll
        for (int u = 0; u < U; u++)
#pragma unroll
            for (int i = 0; i < MT; i++) acc[i] = mma8(fb[u], fa[u][i], acc[i]);
    }
#pragma unroll
    for (int i = 0; i < MT; i++) joined[wave][i][lane] = acc[i];
    __syncthreads();
    if (wave < MT) {
        i32x4 v = joined[0][wave][lane];
        for (int w = 1; w < waves; w++) v += joined[w][wave][lane];
        const int m = 16 * wave + j, n4 = blockIdx.x * 16 + 4 * c;
        const int32_t sum[4] = {v[0], v[1], v[2], v[3]};
        if (m < g.m && n4 < g.n) finish8<ACT, T, 4>(a, m, n4, sum);
    }
}

// -- launches -----------------------------------------------------------------------

inline bool direct8_ok(const GemmArgs &g)
{
    auto ok = [](const void *p, int64_t ld) {       // (a tile's offsets stay in the buffer)
        return aligned_to(p, 16) && ld % 16 == 0 && ld < (int64_t)kBufferBytes / 2048;
    };
    return ok(g.a, g.lda) && ok(g.b, g.ldb) && g.k % 16 == 0;
}

// Splits of k, as the products of 16 bits choose them: where the tiles alone
// leave half or more of the chip empty, with kLeastSteps8 steps or more in each.
inline void choose_splits8(GemmArgs &g)
{
    const int64_t tiles = (int64_t)g.tiles_m * g.tiles_n, steps = ceil_div(g.k, kStep8);
    int64_t splits = kSplitTiles / tiles;
    if (splits > 1 && steps / splits < 2 * kLeastSteps8) {
        splits = kSplitTiles / 2 / tiles;
        if (splits > steps / kLeastSteps8) splits = steps / kLeastSteps8;
    }
    const int64_t one = (int64_t)g.m * ceil_div(g.n, 4) * 16;      // a split's partial sums, in the scratch
    if (splits > g.part_bytes / one) splits = g.part_bytes / one;
    if (splits < 1) splits = 1;
    const int64_t each = ceil_div(steps, splits);
    g.k_split = (int32_t)(each * kStep8);
    g.splits = (int32_t)ceil_div(steps, each);
}

template <int TM, int TN, int WM, int WN, typename T, int ACT>
hipError_t launch_tiles8(Gemm8Args a, hipStream_t stream)
{
    a.g.tiles_m = (int32_t)ceil_div(a.g.m, TM);
    a.g.tiles_n = (int32_t)ceil_div(a.g.n, TN);
    choose_splits8(a.g);
    const dim3 grid(a.g.tiles_m * a.g.tiles_n * a.g.splits), block(WM * WN * 64);
    constexpr int kLds = 2 * (TM + TN) * kStep8;
    if (direct8_ok(a.g))
        hipLaunchKernelGGL((k_gemm8<TM, TN, WM, WN, true, T, ACT>), grid, block, kLds, stream, a);
    else
        hipLaunchKernelGGL((k_gemm8<TM, TN, WM, WN, false, T, ACT>), grid, block, kLds, stream, a);
    if (hipError_t e = hipGetLastError(); e != hipSuccess || a.g.splits == 1) return e;
    const int64_t quads = (int64_t)a.g.m * ((a.g.n + 3) / 4);
    hipLaunchKernelGGL((k_gemm8_join<T, ACT>), dim3((unsigned)ceil_div(quads, 256)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

template <typename T, int ACT>
hipError_t launch_rows8(const Gemm8Args &a, hipStream_t stream)
{
    const int steps = (int)ceil_div(a.g.k, 64);
    const int waves = steps >= 64 ? 16 : steps >= 16 ? 8 : 4;
    const dim3 grid((unsigned)ceil_div(a.g.n, 16)), block(64 * waves);
    if (a.g.m <= 16)
        hipLaunchKernelGGL((k_gemm8_rows<1, T, ACT>), grid, block, 0, stream, a);
    else if (a.g.m <= 32)
        hipLaunchKernelGGL((k_gemm8_rows<2, T, ACT>), grid, block, 0, stream, a);
    else
        hipLaunchKernelGGL((k_gemm8_rows<4, T, ACT>), grid, block, 0, stream, a);
    return hipGetLastError();
}

template <typename T, int ACT>
hipError_t launch_gemm8_act(const Gemm8Args &a, hipStream_t stream)
{
    if (a.g.m <= 16 || (a.g.m <= 64 && (int64_t)a.g.n * a.g.k <= (int64_t)1 << 23)) return launch_rows8<T, ACT>(a, stream);
    return launch_tiles8<128, 128, 2, 2, T, ACT>(a, stream);
}

// Rows in one launch: the grid stays under kMaxTiles.
template <typename T>
hipError_t launch_gemm8_type(const Gemm8Args &all, hipStream_t stream)
{
    const int64_t tiles_n = ceil_div(all.g.n, kTile), most = kMaxTiles / tiles_n * kTile;
    for (int64_t m = 0; m < all.g.m; m += most) {
        Gemm8Args a = all;
        a.g.a = static_cast<const int8_t *>(all.g.a) + m * all.g.lda;
        a.a_scale = all.a_scale + m;
        a.g.out = static_cast<T *>(all.g.out) + m * all.g.ldo;
        if (all.g.residual) a.g.residual = static_cast<const T *>(all.g.residual) + m * all.g.ldr;
        if (all.g.preact) a.g.preact = static_cast<T *>(all.g.preact) + m * all.g.ldp;
        a.g.m = (int32_t)(all.g.m - m < most ? all.g.m - m : most);
        hipError_t e;
        switch (a.g.act) {
        case CPE_ACT_RELU: e = launch_gemm8_act<T, CPE_ACT_RELU>(a, stream); break;
        case CPE_ACT_SILU: e = launch_gemm8_act<T, CPE_ACT_SILU>(a, stream); break;
        case CPE_ACT_GELU: e = launch_gemm8_act<T, CPE_ACT_GELU>(a, stream); break;
        default: e = launch_gemm8_act<T, CPE_ACT_NONE>(a, stream); break;
        }
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace
}  // namespace cpe
