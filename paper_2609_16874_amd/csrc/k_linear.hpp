// k_linear.hpp -- matrix products with an epilogue on the matrix cores, and
// the elementwise parts of their gradient (private to the library; included
// once per element type).
//
// out[m][n] = act(sum_k A(m, k) B(n, k) + bias[n]) + residual[m][n], each
// operand stored along k (an activation row, a weight row) or across it (the
// same matrices in the gradient's products).
//
// Fragments are 16 bytes of k per lane and operand: E = 8 elements of 16 bits
// or 4 of 32.  One 16-bit fragment pair feeds a 16x16x32 instruction, a
// 32-bit pair four 16x16x4 ones, the i-th taking element i of every lane: the
// order of k within a step is free as long as both operands share it.  The
// B fragment goes first, so that a lane's four accumulators are neighbouring
// n of one row m and are stored as one vector.
//
// LDS tiles hold 128 bytes of k.  Along k: a row per m (or n) of eight
// 16-byte chunks, chunk c of row r at place c ^ (r & 7).  Across k: a row per
// k, read back through the transposing LDS read (16 bits), its 32-byte units
// permuted by the bits of k that one read's lanes span.
#pragma once

#include "head_common.hpp"
#include "linear.hpp"

#pragma clang fp contract(fast)

namespace cpe {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) unsigned char lds_byte;

template <typename T>
constexpr int kChunk = 16 / (int)sizeof(T);           // elements in 16 bytes
template <typename T>
constexpr int kStepK = 8 * kChunk<T>;                 // k of one LDS tile

__device__ __align__(16) const uint32_t zero_chunk[4] = {0, 0, 0, 0};

union Fragment {
    u32x4 u;
    f16x8 h;
    bf16x8 b;
    f32x4 f;
    s16x4 s[2];
};

template <typename T>
__device__ __forceinline__ f32x4 mma(const Fragment &n, const Fragment &m, f32x4 acc)
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; i++) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(n.f[i], m.f[i], acc, 0, 0, 0);
        return acc;
    } else if constexpr (std::is_same<T, _Float16>::value) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(n.h, m.h, acc, 0, 0, 0);
    } else {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(n.b, m.b, acc, 0, 0, 0);
    }
}

// 16 bytes of a row of which `left` elements (any number) exist; the rest 0.
template <typename T>
__device__ __forceinline__ u32x4 load_chunk(const T *p, int64_t left)
{
    Fragment f;
    f.u = u32x4{0, 0, 0, 0};
    if (left >= kChunk<T>) {
        const Vec<T, kChunk<T>> v = load_vec<T, kChunk<T>>(p);
        __builtin_memcpy(&f, &v, 16);
    } else if (left > 0) {
        T e[kChunk<T>];
#pragma unroll
        for (int i = 0; i < kChunk<T>; i++) e[i] = i < left ? p[i] : (T)0.0f;
        __builtin_memcpy(&f, e, 16);
    }
    return f.u;
}

// One operand of a workgroup: R rows (m or n) by kStepK of k.
template <typename T, bool ACROSS, int R, bool DIRECT>
struct Operand {
    static constexpr int E = kChunk<T>, kLoads = R * 8 / kGemmThreads;
    static constexpr int kPerRow = ACROSS ? R / E : 8;    // chunks in an LDS row
    static constexpr int kBytes = R * 128;
    const T *src[kLoads];
    int room[kLoads];       // along k: k left from this chunk on; across: valid elements of the chunk
    int krow[kLoads];       // across: k of the chunk
    int64_t step;
    u32x4 held[DIRECT ? 1 : kLoads];

    __device__ __forceinline__ static int permute(int krow)      // of the 32-byte units of a row across k
    {
        if constexpr (sizeof(T) == 4) return 0;
        return R >= 128 ? (krow & 3) | ((krow >> 3) & 1) << 2 : ((krow >> 1) & 1) | ((krow >> 3) & 1) << 1;
    }

    __device__ __forceinline__ void init(const void *base, int64_t ld, int r0, int r_end, int k0)
    {
        step = ACROSS ? kStepK<T> * ld : kStepK<T>;
        const T *p = static_cast<const T *>(base);
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const int q = i * kGemmThreads + threadIdx.x, row = q / kPerRow, pc = q % kPerRow;
            if constexpr (ACROSS) {
                const int lc = sizeof(T) == 4 ? pc : ((((pc >> 1) ^ permute(row)) << 1) | (pc & 1));
                const int r = r0 + lc * E;
                krow[i] = row;
                room[i] = r_end - r;
                src[i] = room[i] > 0 ? p + (int64_t)(k0 + row) * ld + r : nullptr;
            } else {
                const int lc = pc ^ (row & 7);
                room[i] = lc * E;
                krow[i] = 0;
                src[i] = r0 + row < r_end ? p + (int64_t)(r0 + row) * ld + k0 + lc * E : nullptr;
            }
        }
    }

    // Fetch the step with `left` k remaining: into LDS, or into registers.
    __device__ __forceinline__ void fetch(lds_byte *lds, int left)
    {
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const int valid = src[i] == nullptr ? 0 : ACROSS ? (krow[i] < left ? room[i] : 0) : left - room[i];
            if constexpr (DIRECT) {
                const void *p = valid > 0 ? (const void *)src[i] : (const void *)zero_chunk;
                lds_byte *to = lds + (i * kGemmThreads + (threadIdx.x & ~63)) * 16;
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t *)p,
                                                 (__attribute__((address_space(3))) uint32_t *)to, 16, 0, 0);
            } else {
                held[i] = load_chunk<T>(src[i], valid);
            }
            if (src[i]) src[i] += step;
        }
    }
    __device__ __forceinline__ void commit(lds_byte *lds) const
    {
        if constexpr (!DIRECT)
#pragma unroll
            for (int i = 0; i < kLoads; i++)
                *(__attribute__((address_space(3))) u32x4 *)(lds + (i * kGemmThreads + threadIdx.x) * 16) = held[i];
    }

    // The fragment of rows r .. r+15 for the s-th half of the step.
    __device__ __forceinline__ static Fragment read(const lds_byte *lds, int r, int s)
    {
        const int lane = threadIdx.x & 63, j = lane & 15, g = lane >> 4;
        Fragment f;
        if constexpr (!ACROSS) {
            const int row = r + j, c = (4 * s + g) ^ (row & 7);
            f.u = *(const __attribute__((address_space(3))) u32x4 *)(lds + (row * 8 + c) * 16);
        } else if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int krow = 16 * s + 4 * g + i;
                f.f[i] = *(const __attribute__((address_space(3))) float *)(lds + (krow * R + r + j) * 4);
            }
        } else {
            // sixteen lanes name four k rows of sixteen elements, and receive a column of four each
#pragma unroll
            for (int t = 0; t < 2; t++) {
                const int krow = 32 * s + 8 * g + 4 * t + (j >> 2);
                const int unit = (r >> 4) ^ permute(krow);
                f.s[t] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (__attribute__((address_space(3))) s16x4 *)(lds + krow * (R * 2) + unit * 32 + (j & 3) * 8));
            }
        }
        return f;
    }
};

// W neighbouring outputs of row m: bias, the value kept for the gradient,
// activation, residual, each rounded once.
template <int ACT, typename T, int W>
__device__ __forceinline__ void finish(const GemmArgs &g, int m, int n, float (&v)[W])
{
    const int left = g.n - n;
    T *out = static_cast<T *>(g.out) + m * g.ldo + n;
    const T *res = g.residual ? static_cast<const T *>(g.residual) + m * g.ldr + n : nullptr;
    T *pre = g.preact ? static_cast<T *>(g.preact) + m * g.ldp + n : nullptr;
    if (left >= W) {
        Vec<T, W> o;
        if (g.bias) {
            const Vec<float, W> b = load_vec<float, W>(g.bias + n);
#pragma unroll
            for (int i = 0; i < W; i++) v[i] += b.v[i];
        }
        if (pre) {
#pragma unroll
            for (int i = 0; i < W; i++) o.v[i] = (T)v[i];
            store_vec<T, W>(pre, o);
        }
#pragma unroll
        for (int i = 0; i < W; i++) v[i] = activate<ACT>(v[i]);
        if (res) {
            const Vec<T, W> r = load_vec<T, W>(res);
#pragma unroll
            for (int i = 0; i < W; i++) v[i] += (float)r.v[i];
        }
#pragma unroll
        for (int i = 0; i < W; i++) o.v[i] = (T)v[i];
        store_vec<T, W>(out, o);
    } else {
#pragma unroll
        for (int i = 0; i < W; i++)
            if (i < left) {
                const float z = v[i] + (g.bias ? g.bias[n + i] : 0.0f);
                if (pre) pre[i] = (T)z;
                out[i] = (T)(activate<ACT>(z) + (res ? (float)res[i] : 0.0f));
            }
    }
}
template <int ACT, typename T>
__device__ __forceinline__ void finish(const GemmArgs &g, int m, int n, f32x4 v)
{
    float w[4] = {v[0], v[1], v[2], v[3]};
    finish<ACT, T, 4>(g, m, n, w);
}

template <typename T, bool A_ACROSS, bool B_ACROSS, bool DIRECT, int ACT>
__global__ __launch_bounds__(kGemmThreads) void k_gemm(GemmArgs g)
{
    using A = Operand<T, A_ACROSS, kTile, DIRECT>;
    using B = Operand<T, B_ACROSS, kTile, DIRECT>;
    __shared__ __align__(1024) unsigned char smem[2][A::kBytes + B::kBytes];
    const int tiles = g.tiles_m * g.tiles_n;
    const int split = blockIdx.x / tiles, tile = xcd_order(blockIdx.x - split * tiles, tiles);
    const int m0 = (tile / g.tiles_n) * kTile, n0 = (tile % g.tiles_n) * kTile;
    const int k0 = split * g.k_split;
    const int len = g.k - k0 < g.k_split ? g.k - k0 : g.k_split;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int wm = (wave >> 1) * 64, wn = (wave & 1) * 64;
    A a;
    B b;
    a.init(g.a, g.lda, m0, g.m, k0);
    b.init(g.b, g.ldb, n0, g.n, k0);
    f32x4 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; i++)
#pragma unroll
        for (int j = 0; j < 4; j++) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    auto buffer = [&](int s) { return (lds_byte *)smem[s]; };
    if (len > 0) {
        a.fetch(buffer(0), len);
        b.fetch(buffer(0) + A::kBytes, len);
        a.commit(buffer(0));
        b.commit(buffer(0) + A::kBytes);
    }
    int cur = 0;
    for (int left = len; left > 0; left -= kStepK<T>, cur ^= 1) {
        __syncthreads();
        const bool more = left > kStepK<T>;
        if (more) {
            a.fetch(buffer(cur ^ 1), left - kStepK<T>);
            b.fetch(buffer(cur ^ 1) + A::kBytes, left - kStepK<T>);
        }
        const lds_byte *la = buffer(cur), *lb = la + A::kBytes;
#pragma unroll
        for (int s = 0; s < 2; s++) {
            Fragment fa[4], fb[4];
#pragma unroll
            for (int i = 0; i < 4; i++) fa[i] = A::read(la, wm + 16 * i, s);
#pragma unroll
            for (int i = 0; i < 4; i++) fb[i] = B::read(lb, wn + 16 * i, s);
#pragma unroll
            for (int i = 0; i < 4; i++)
#pragma unroll
                for (int j = 0; j < 4; j++) acc[i][j] = mma<T>(fb[j], fa[i], acc[i][j]);
        }
        if (more) {
            a.commit(buffer(cur ^ 1));
            b.commit(buffer(cur ^ 1) + A::kBytes);
        }
    }
    const int64_t ldpart = (g.n + 3) / 4 * 4;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int m = m0 + wm + 16 * i + (lane & 15);
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const int n = n0 + wn + 16 * j + 4 * (lane >> 4);
            if (m >= g.m || n >= g.n) continue;
            if (g.splits > 1)
                *reinterpret_cast<f32x4 *>(g.part + ((int64_t)split * g.m + m) * ldpart + n) = acc[i][j];
            else
                finish<ACT, T>(g, m, n, acc[i][j]);
        }
    }
}

// The splits' partial products summed in a fixed order, then the epilogue:
// 16 vectors of four n per workgroup, 16 lanes of splits for each.
template <typename T, int ACT>
__global__ __launch_bounds__(256) void k_gemm_join(GemmArgs g)
{
    __shared__ f32x4 lds[4][16];
    const int quads = (g.n + 3) / 4, at = threadIdx.x & 15, lane = threadIdx.x >> 4;
    const int64_t all = (int64_t)g.m * quads, q = (int64_t)blockIdx.x * 16 + at;
    const int64_t step = all * 4;
    const float *p = g.part + q * 4;
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    if (q < all) {
#pragma unroll 4
        for (int s = lane; s < g.splits; s += 16) v += *reinterpret_cast<const f32x4 *>(p + s * step);
    }
#pragma unroll
    for (int o = 16; o <= 32; o <<= 1)
#pragma unroll
        for (int i = 0; i < 4; i++) v[i] += __shfl_xor(v[i], o);
    if ((threadIdx.x & 63) < 16) lds[threadIdx.x >> 6][at] = v;
    __syncthreads();
    if (threadIdx.x < 16 && q < all) {
        v = (lds[0][at] + lds[1][at]) + (lds[2][at] + lds[3][at]);
        const int m = (int)(q / quads);
        finish<ACT, T>(g, m, (int)(q - (int64_t)m * quads) * 4, v);
    }
}

// Few rows (a served token or a handful): 16 n per workgroup, its waves
// dividing k; fragments come straight from memory, since no other workgroup
// shares the weights and the rows stay in the caches.
template <typename T, int MT, int ACT>
__global__ __launch_bounds__(1024) void k_gemm_rows(GemmArgs g)
{
    __shared__ f32x4 joined[16][MT][64];
    constexpr int E = kChunk<T>, kStep = 4 * E;
    const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6, lane = threadIdx.x & 63;
    const int j = lane & 15, c = lane >> 4, n = blockIdx.x * 16 + j;
    const int steps = (g.k + kStep - 1) / kStep, each = (steps + waves - 1) / waves;
    const int lo = wave * each, hi = lo + each < steps ? lo + each : steps;
    const T *pb = static_cast<const T *>(g.b) + (int64_t)n * g.ldb;
    f32x4 acc[MT];
#pragma unroll
    for (int i = 0; i < MT; i++) acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    constexpr int U = 4;
    for (int s = lo; s < hi; s += U) {
        Fragment fb[U], fa[U][MT];
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int k = (s + u) * kStep + c * E, left = s + u < hi ? g.k - k : 0;
            fb[u].u = load_chunk<T>(pb + k, n < g.n ? left : 0);
#pragma unroll
            for (int i = 0; i < MT; i++) {
                const int m = 16 * i + j;
                fa[u][i].u = load_chunk<T>(static_cast<const T *>(g.a) + m * g.lda + k, m < g.m ? left : 0);
            }
        }
#pragma unroll
        for (int u = 0; u < U; u++)
#pragma unroll
            for (int i = 0; i < MT; i++) acc[i] = mma<T>(fb[u], fa[u][i], acc[i]);
    }
#pragma unroll
    for (int i = 0; i < MT; i++) joined[wave][i][lane] = acc[i];
    __syncthreads();
    if (wave < MT) {
        f32x4 v = joined[0][wave][lane];
        for (int w = 1; w < waves; w++) v += joined[w][wave][lane];
        const int m = 16 * wave + j, n4 = blockIdx.x * 16 + 4 * c;
        if (m < g.m && n4 < g.n) finish<ACT, T>(g, m, n4, v);
    }
}

// Narrow products (a map's projection to its embedding), whose B fits into LDS
// whole: it is laid out there once per workgroup, along k, and the waves stream
// the rows of A past it, 16 at a time, straight from memory into fragments, the
// next strip in flight while the present one is multiplied.  No barrier and no
// LDS traffic for A; every row is read once.
//
// B's rows within a pair of 16-row fragments are taken in the order
// n = 8 (r / 4) + 4 t + r % 4 (fragment t, row r), which leaves each lane
// eight neighbouring n of its row of A: one 16-byte store for 16-bit types.
// Chunk c of row n lies at c ^ swizzle(n), so that eight lanes' reads meet all
// the banks in that order.
template <typename T>
constexpr int kNarrowStep = 4 * kChunk<T>;       // k of one fragment
constexpr int kNarrowLds = 64 << 10;             // most bytes of B
__device__ __forceinline__ int narrow_swizzle(int n) { return (n & 3) | ((n >> 3) & 1) << 2; }

template <typename T, int KS, bool B_ACROSS, int ACT>
__global__ __launch_bounds__(256) void k_gemm_narrow(GemmArgs g)
{
    extern __shared__ __align__(1024) unsigned char narrow_lds[];
    constexpr int E = kChunk<T>, kRow = KS * 4;        // chunks in a row of B
    lds_byte *lds = (lds_byte *)narrow_lds;
    const int pairs = (g.n + 31) / 32, n_pad = pairs * 32;
    for (int q = threadIdx.x; q < n_pad * kRow; q += 256) {
        int n, c;
        Fragment f;
        f.u = u32x4{0, 0, 0, 0};
        if constexpr (B_ACROSS) {       // neighbouring threads read neighbouring n
            c = q / n_pad;
            n = q - c * n_pad;
            T e[E];
#pragma unroll
            for (int i = 0; i < E; i++)
                e[i] = n < g.n && c * E + i < g.k ? static_cast<const T *>(g.b)[(int64_t)(c * E + i) * g.ldb + n]
                                                  : (T)0.0f;
            __builtin_memcpy(&f, e, 16);
        } else {
            n = q / kRow;
            c = q - n * kRow;
            f.u = load_chunk<T>(static_cast<const T *>(g.b) + (int64_t)n * g.ldb + c * E, n < g.n ? g.k - c * E : 0);
        }
        *(__attribute__((address_space(3))) u32x4 *)(lds + (n * kRow + (c ^ narrow_swizzle(n))) * 16) = f.u;
    }
    __syncthreads();
    const int lane = threadIdx.x & 63, j = lane & 15, c = lane >> 4;
    const int strips = (g.m + 15) / 16, step = gridDim.x * 4;
    const int full = g.k / E;                    // whole chunks of a row of A
    auto fetch = [&](int strip, Fragment (&f)[KS]) {
        const int m = strip * 16 + j;
        const T *p = static_cast<const T *>(g.a) + m * g.lda;
        const bool on = m < g.m;
#pragma unroll
        for (int s = 0; s < KS; s++) {
            const int chunk = 4 * s + c;
            f[s].u = u32x4{0, 0, 0, 0};
            if (on && chunk < full) {
                const Vec<T, E> v = load_vec<T, E>(p + chunk * E);
                __builtin_memcpy(&f[s], &v, 16);
            } else if (on && chunk == full) {
                f[s].u = load_chunk<T>(p + chunk * E, g.k - chunk * E);
            }
        }
    };
    Fragment next[KS];
    int strip = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (strip < strips) fetch(strip, next);
    const int row = 8 * (j >> 2) + (j & 3);
    for (; strip < strips; strip += step) {
        Fragment fa[KS];
#pragma unroll
        for (int s = 0; s < KS; s++) fa[s] = next[s];
        if (strip + step < strips) fetch(strip + step, next);
        const int m = strip * 16 + j;
        for (int p = 0; p < pairs; p++) {
            f32x4 acc[2] = {f32x4{0.0f, 0.0f, 0.0f, 0.0f}, f32x4{0.0f, 0.0f, 0.0f, 0.0f}};
#pragma unroll
            for (int s = 0; s < KS; s++)
#pragma unroll
                for (int t = 0; t < 2; t++) {
                    const int n = 32 * p + row + 4 * t;
                    Fragment fb;
                    fb.u = *(const __attribute__((address_space(3))) u32x4 *)(
                        lds + (n * kRow + ((4 * s + c) ^ narrow_swizzle(n))) * 16);
                    acc[t] = mma<T>(fb, fa[s], acc[t]);
                }
            const int n = 32 * p + 8 * c;
            if (m < g.m && n < g.n) {
                float v[8] = {acc[0][0], acc[0][1], acc[0][2], acc[0][3],
                              acc[1][0], acc[1][1], acc[1][2], acc[1][3]};
                finish<ACT, T, 8>(g, m, n, v);
            }
        }
    }
}

// dz = dy act'(preact), rounded (the products' operand), and its column sums
// over this workgroup's rows, unrounded.  A workgroup covers up to 256 vectors
// of V columns (blockIdx.y) and 256 / vectors rows at a time.
template <typename T, int V, int ACT>
__global__ __launch_bounds__(256) void k_act_grad(GradArgs g)
{
    __shared__ float lds[256 * V];
    const int all = g.n / V, first = blockIdx.y * 256, here = all - first < 256 ? all - first : 256;
    const int rows = 256 / here, row = threadIdx.x / here, col = threadIdx.x - row * here;
    const int64_t span = (g.rows + (int64_t)g.blocks - 1) / g.blocks, lo = span * blockIdx.x;
    const int64_t hi = lo + span < g.rows ? lo + span : g.rows;
    float sum[V];
#pragma unroll
    for (int v = 0; v < V; v++) sum[v] = 0.0f;
    if (row < rows) {
        const int n = (first + col) * V;
        const T *pd = static_cast<const T *>(g.dy) + n, *pz = static_cast<const T *>(g.preact) + n;
        T *po = static_cast<T *>(g.dz) + n;
        constexpr int U = 4;
        for (int64_t r = lo + row; r < hi; r += U * rows) {
            Vec<T, V> d[U], z[U];
#pragma unroll
            for (int u = 0; u < U; u++) {
                const int64_t at = r + u * rows;
                if (at < hi) {
                    d[u] = load_vec<T, V>(pd + at * g.ldd);
                    if (ACT != CPE_ACT_NONE) z[u] = load_vec<T, V>(pz + at * g.ldp);
                }
            }
#pragma unroll
            for (int u = 0; u < U; u++) {
                const int64_t at = r + u * rows;
                if (at >= hi) continue;
                Vec<T, V> o;
#pragma unroll
                for (int v = 0; v < V; v++) {
                    float dz = (float)d[u].v[v];
                    if constexpr (ACT != CPE_ACT_NONE) dz *= activate_grad<ACT>((float)z[u].v[v]);
                    sum[v] += dz;
                    o.v[v] = (T)dz;
                }
                if (ACT != CPE_ACT_NONE && g.dz) store_vec<T, V>(po + at * g.ldz, o);
            }
        }
#pragma unroll
        for (int v = 0; v < V; v++) lds[(row * here + col) * V + v] = sum[v];
    }
    __syncthreads();
    if (!g.sums) return;
    for (int i = threadIdx.x; i < here * V; i += 256) {
        float s = 0.0f;
        for (int r = 0; r < rows; r++) s += lds[r * here * V + i];
        g.part[(int64_t)blockIdx.x * g.n + first * V + i] = s;
    }
}

// sums[n] over the workgroups' partials: 32 columns (a cache line) per
// workgroup, 32 lanes of partials each.
__global__ __launch_bounds__(1024) void k_column_join(GradArgs g)
{
    __shared__ double lds[16][32];
    const int at = threadIdx.x & 31, n = blockIdx.x * 32 + at;
    double s = 0.0;
    if (n < g.n) {
#pragma unroll 8
        for (int i = threadIdx.x >> 5; i < g.blocks; i += 32) s += (double)g.part[(int64_t)i * g.n + n];
    }
    s += __shfl_xor(s, 32);
    if ((threadIdx.x & 63) < 32) lds[threadIdx.x >> 6][at] = s;
    __syncthreads();
    if (threadIdx.x < 32 && n < g.n) {
        s = 0.0;
        for (int w = 0; w < 16; w++) s += lds[w][at];
        g.sums[n] = (float)s;
    }
}

// -- launches -----------------------------------------------------------------------

template <typename T>
bool direct_ok(const GemmArgs &g)
{
    constexpr int E = kChunk<T>;
    auto ok = [](const void *p, int64_t ld, int width) {
        return aligned_to(p, 16) && ld % E == 0 && width % E == 0;
    };
    return ok(g.a, g.lda, g.a_cols ? g.m : g.k) && ok(g.b, g.ldb, g.b_cols ? g.n : g.k);
}

// Workgroups dividing k where the tiles alone leave most of the chip idle:
// at most kSplitTiles partial tiles, each of four steps of k or more.
template <typename T>
void choose_splits(GemmArgs &g)
{
    const int64_t tiles = (int64_t)g.tiles_m * g.tiles_n, steps = ceil_div(g.k, kStepK<T>);
    int64_t splits = 1;
    if (g.part && tiles <= kSplitTiles / 4) {
        splits = kSplitTiles / tiles;
        if (splits > steps / 4) splits = steps / 4;
        if (splits < 1) splits = 1;
    }
    const int64_t each = ceil_div(steps > 0 ? steps : 1, splits);
    g.k_split = (int32_t)(each * kStepK<T>);
    g.splits = (int32_t)ceil_div(steps > 0 ? steps : 1, each);
}

template <typename T, bool A_ACROSS, bool B_ACROSS, int ACT>
hipError_t launch_tiles(GemmArgs g, hipStream_t stream)
{
    g.tiles_m = (int32_t)ceil_div(g.m, kTile);
    g.tiles_n = (int32_t)ceil_div(g.n, kTile);
    choose_splits<T>(g);
    const dim3 grid(g.tiles_m * g.tiles_n * g.splits);
    if (direct_ok<T>(g))
        hipLaunchKernelGGL((k_gemm<T, A_ACROSS, B_ACROSS, true, ACT>), grid, dim3(kGemmThreads), 0, stream, g);
    else
        hipLaunchKernelGGL((k_gemm<T, A_ACROSS, B_ACROSS, false, ACT>), grid, dim3(kGemmThreads), 0, stream, g);
    if (hipError_t e = hipGetLastError(); e != hipSuccess || g.splits == 1) return e;
    const int64_t quads = (int64_t)g.m * ((g.n + 3) / 4);
    hipLaunchKernelGGL((k_gemm_join<T, ACT>), dim3((unsigned)ceil_div(quads, 16)), dim3(256), 0, stream, g);
    return hipGetLastError();
}

template <typename T, int ACT>
hipError_t launch_rows(const GemmArgs &g, hipStream_t stream)
{
    const int steps = (int)ceil_div(g.k, 4 * kChunk<T>);
    const int waves = steps >= 64 ? 16 : steps >= 16 ? 8 : 4;
    const dim3 grid((unsigned)ceil_div(g.n, 16)), block(64 * waves);
    if (g.m <= 16)
        hipLaunchKernelGGL((k_gemm_rows<T, 1, ACT>), grid, block, 0, stream, g);
    else if (g.m <= 32)
        hipLaunchKernelGGL((k_gemm_rows<T, 2, ACT>), grid, block, 0, stream, g);
    else
        hipLaunchKernelGGL((k_gemm_rows<T, 4, ACT>), grid, block, 0, stream, g);
    return hipGetLastError();
}

// Fragments of k that hold a row of A (2, 4, 8 or 16), 0 where it is too long.
template <typename T>
int narrow_steps(int k)
{
    for (int ks = 2; ks <= 16; ks *= 2)
        if (k <= ks * kNarrowStep<T>) return ks;
    return 0;
}
template <typename T>
int narrow_bytes(const GemmArgs &g)
{
    return (int)(ceil_div(g.n, 32) * 32 * narrow_steps<T>(g.k) * 64);
}
template <typename T>
bool narrow_fits(const GemmArgs &g)
{
    return narrow_steps<T>(g.k) > 0 && g.n <= 4096 && narrow_bytes<T>(g) <= kNarrowLds;
}

template <typename T, bool B_ACROSS, int ACT>
hipError_t launch_narrow(const GemmArgs &g, hipStream_t stream)
{
    const int bytes = narrow_bytes<T>(g), per_cu = (160 << 10) / (bytes + 1024);
    const int64_t want = ceil_div(ceil_div(g.m, 16), 4), most = 256 * (per_cu < 4 ? per_cu : 4);
    const dim3 grid((unsigned)(want < most ? want : most));
    switch (narrow_steps<T>(g.k)) {
    case 2: hipLaunchKernelGGL((k_gemm_narrow<T, 2, B_ACROSS, ACT>), grid, dim3(256), bytes, stream, g); break;
    case 4: hipLaunchKernelGGL((k_gemm_narrow<T, 4, B_ACROSS, ACT>), grid, dim3(256), bytes, stream, g); break;
    case 8: hipLaunchKernelGGL((k_gemm_narrow<T, 8, B_ACROSS, ACT>), grid, dim3(256), bytes, stream, g); break;
    default: hipLaunchKernelGGL((k_gemm_narrow<T, 16, B_ACROSS, ACT>), grid, dim3(256), bytes, stream, g); break;
    }
    return hipGetLastError();
}

template <typename T, int ACT>
hipError_t launch_forward(const GemmArgs &g, hipStream_t stream)
{
    if (g.m <= 64) return launch_rows<T, ACT>(g, stream);
    if (narrow_fits<T>(g)) return launch_narrow<T, false, ACT>(g, stream);
    return launch_tiles<T, false, false, ACT>(g, stream);
}

// Rows in one launch: the grid stays under kMaxTiles.
template <typename T>
hipError_t launch_gemm_type(const GemmArgs &all, hipStream_t stream)
{
    if (all.a_cols && all.b_cols) return launch_tiles<T, true, true, CPE_ACT_NONE>(all, stream);
    const int64_t tiles_n = ceil_div(all.n, kTile), most = kMaxTiles / tiles_n * kTile;
    for (int64_t m = 0; m < all.m; m += most) {
        GemmArgs g = all;
        g.a = static_cast<const T *>(all.a) + m * all.lda;
        g.out = static_cast<T *>(all.out) + m * all.ldo;
        if (all.residual) g.residual = static_cast<const T *>(all.residual) + m * all.ldr;
        if (all.preact) g.preact = static_cast<T *>(all.preact) + m * all.ldp;
        g.m = (int32_t)(all.m - m < most ? all.m - m : most);
        hipError_t e;
        if (g.b_cols)
            e = narrow_fits<T>(g) ? launch_narrow<T, true, CPE_ACT_NONE>(g, stream)
                                  : launch_tiles<T, false, true, CPE_ACT_NONE>(g, stream);
        else if (g.act == CPE_ACT_RELU)
            e = launch_forward<T, CPE_ACT_RELU>(g, stream);
        else if (g.act == CPE_ACT_SILU)
            e = launch_forward<T, CPE_ACT_SILU>(g, stream);
        else if (g.act == CPE_ACT_GELU)
            e = launch_forward<T, CPE_ACT_GELU>(g, stream);
        else
            e = launch_forward<T, CPE_ACT_NONE>(g, stream);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T, int V>
hipError_t launch_grad_width(GradArgs g, hipStream_t stream)
{
    const int vectors = g.n / V, rows = vectors >= 256 ? 1 : 256 / vectors;
    const int64_t slabs = ceil_div(vectors, 256);
    const int64_t want = ceil_div(g.rows, 4 * (int64_t)rows), cap = kSumBlocks / slabs < 1 ? 1 : kSumBlocks / slabs;
    g.blocks = (int32_t)(want < 1 ? 1 : want < cap ? want : cap);
    const dim3 grid(g.blocks, (unsigned)slabs);
    switch (g.act) {
    case CPE_ACT_RELU: hipLaunchKernelGGL((k_act_grad<T, V, CPE_ACT_RELU>), grid, dim3(256), 0, stream, g); break;
    case CPE_ACT_SILU: hipLaunchKernelGGL((k_act_grad<T, V, CPE_ACT_SILU>), grid, dim3(256), 0, stream, g); break;
    case CPE_ACT_GELU: hipLaunchKernelGGL((k_act_grad<T, V, CPE_ACT_GELU>), grid, dim3(256), 0, stream, g); break;
    default: hipLaunchKernelGGL((k_act_grad<T, V, CPE_ACT_NONE>), grid, dim3(256), 0, stream, g); break;
    }
    if (hipError_t e = hipGetLastError(); e != hipSuccess || !g.sums) return e;
    hipLaunchKernelGGL(k_column_join, dim3((unsigned)ceil_div(g.n, 32)), dim3(1024), 0, stream, g);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_grad_type(const GradArgs &g, hipStream_t stream)
{
    if constexpr (sizeof(T) == 2)
        if (g.n % 8 == 0) return launch_grad_width<T, 8>(g, stream);
    if (g.n % 4 == 0) return launch_grad_width<T, 4>(g, stream);
    if (g.n % 2 == 0) return launch_grad_width<T, 2>(g, stream);
    return launch_grad_width<T, 1>(g, stream);
}

}  // namespace
}  // namespace cpe
