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
// The gradient's products take dz = dy act'(z) as an operand of these
// instructions, so it is rounded to the type first (in 32 bits it stays as it
// is).  To keep more of it would take a second operand for its low half and
// twice the products, which are 145 of the 198 us of a large gradient.  The
// rounding is as large as the outputs' own: dx and dw are off by 2.9e-4 instead
// of 2.1e-4 in f16 and 2.3e-3 instead of 1.7e-3 in bf16 (2-norm of the error
// over that of the result; 409,600 x 256 to 64 and 7744 x 1024 to 4096).
//
// LDS tiles hold 128 bytes of k.  Along k: a row per m (or n) of eight
// 16-byte chunks, chunk c of row r at place c ^ (r & 7).  Across k: a row per
// k, read back through the transposing LDS read (16 bits), its 32-byte units
// permuted by the bits of k that one read's lanes span.
#pragma once

#include "common.hpp"
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
constexpr int kStepK = step_k(sizeof(T));

union Fragment {
    u32x4 u;
    f16x8 h;
    bf16x8 b;
    f32x4 f;
    s16x4 s[2];
};

// The first thread of this wave, as a scalar.
__device__ __forceinline__ int wave_base() { return __builtin_amdgcn_readfirstlane(threadIdx.x & ~63); }

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

// One operand of a workgroup: R rows (m or n) by kStepK of k.  DIRECT: loads
// through a buffer descriptor straight into LDS; a lane out of range has an
// offset beyond the descriptor's, which reads as 0.
constexpr uint32_t kBufferBytes = 0x80000000u;
template <typename T, bool ACROSS, bool DIRECT>
struct Operand {
    static constexpr int E = kChunk<T>, R = kTile, kLoads = R * 8 / kGemmThreads;
    static constexpr int kPerRow = ACROSS ? R / E : 8;    // chunks in an LDS row
    static constexpr int kBytes = R * 128;
    const T *base;          // DIRECT: of the workgroup; else of the first row
    int64_t step;
    uint32_t off[kLoads];   // DIRECT: bytes from the base
    const T *src[DIRECT ? 1 : kLoads];
    int room[DIRECT ? 1 : kLoads];      // staged, across: valid elements of the chunk
    u32x4 held[DIRECT ? 1 : kLoads];

    __device__ __forceinline__ static int permute(int krow)      // of the 32-byte units of a row across k
    {
        if constexpr (sizeof(T) == 4) return 0;
        return (krow & 3) | ((krow >> 3) & 1) << 2;
    }
    // this thread's i-th chunk: its row in LDS, and the chunk of the row
    __device__ __forceinline__ static int row_of(int i) { return (i * kGemmThreads + threadIdx.x) / kPerRow; }
    __device__ __forceinline__ static int chunk_of(int i)
    {
        const int pc = (i * kGemmThreads + threadIdx.x) % kPerRow, row = row_of(i);
        if constexpr (!ACROSS) return pc ^ (row & 7);
        return sizeof(T) == 4 ? pc : ((((pc >> 1) ^ permute(row)) << 1) | (pc & 1));
    }

    __device__ __forceinline__ void init(const void *p, int64_t ld, int r0, int r_end, int k0)
    {
        step = ACROSS ? kStepK<T> * ld : kStepK<T>;
        base = static_cast<const T *>(p) + (ACROSS ? k0 * ld + r0 : r0 * ld + k0);
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const int row = row_of(i), c = chunk_of(i);
            const int left = ACROSS ? r_end - r0 - c * E : r_end - r0 - row;
            if constexpr (DIRECT) {
                off[i] = left > 0 ? (uint32_t)((row * ld + c * E) * (int64_t)sizeof(T)) : kBufferBytes;
            } else {
                room[i] = left;
                src[i] = base + row * ld + c * E;
            }
        }
    }

    // Fetch the next step into LDS, or into registers; TAIL: only `left` k of
    // it exist.
    template <bool TAIL>
    __device__ __forceinline__ void fetch(lds_byte *lds, int left)
    {
        if constexpr (DIRECT) {
#ifdef __HIP_DEVICE_COMPILE__       // (the host's pass does not know the descriptor's type)
            const auto buffer =
                __builtin_amdgcn_make_buffer_rsrc(const_cast<T *>(base), 0, (int)kBufferBytes, 0x00027000);
#pragma unroll
            for (int i = 0; i < kLoads; i++) {
                uint32_t at = off[i];
                if constexpr (TAIL) at = (ACROSS ? row_of(i) : chunk_of(i) * E) < left ? at : kBufferBytes;
                lds_byte *to = lds + (i * kGemmThreads + wave_base()) * 16;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer, (__attribute__((address_space(3))) void *)to, 16, at,
                                                         0, 0, 0);
            }
#endif
            base += step;
        } else {
#pragma unroll
            for (int i = 0; i < kLoads; i++) {
                held[i] = load_chunk<T>(src[i], ACROSS ? (row_of(i) < left ? room[i] : 0)
                                                       : (room[i] > 0 ? left - chunk_of(i) * E : 0));
                src[i] += step;
            }
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

// An operand across k of which each k is a row in 8 bits: bytes come into
// registers, and become elements on their way to LDS, where they lie as
// those of Operand<T, true>.  RAGGED: its columns are no multiple of a chunk.
// (Chunks of columns that are not there repeat the first one: what comes of them
// is not stored.)
template <typename T, bool RAGGED>
struct PackedOperand : Operand<T, true, false> {
    using O = Operand<T, true, false>;
    static constexpr int E = O::E, kLoads = O::kLoads;
    const int8_t *from[kLoads];
    const float *scales;
    int64_t step8;
    int columns[RAGGED ? kLoads : 1];
    Vec<int8_t, E> bytes[kLoads];
    float scale[kLoads];
    uint32_t part;          // the bits of a scale that are taken: all, or sign and exponent

    __device__ __forceinline__ void init(const GemmArgs &g, int r0, int k0)
    {
        step8 = kStepK<T> * g.ldb;
        scales = g.b_scale + k0;
        part = g.fold ? 0xff800000u : 0xffffffffu;
        const int8_t *first = static_cast<const int8_t *>(g.b) + k0 * g.ldb + r0;
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const int row = O::row_of(i), c = O::chunk_of(i), left = g.n - r0 - c * E;
            if constexpr (RAGGED) columns[i] = left;
            from[i] = first + row * g.ldb + (RAGGED || left > 0 ? c * E : 0);
        }
    }
    template <bool TAIL>
    __device__ __forceinline__ void fetch(lds_byte *, int left)
    {
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const bool there = !TAIL || O::row_of(i) < left;
            scale[i] = there ? scales[O::row_of(i)] : 0.0f;
            if (there && (!RAGGED || columns[i] >= E)) {
                bytes[i] = load_vec<int8_t, E>(from[i]);
            } else {
#pragma unroll
                for (int e = 0; e < E; e++)
                    bytes[i].v[e] = RAGGED && there && e < columns[RAGGED ? i : 0] ? from[i][e] : (int8_t)0;
            }
            from[i] += step8;
        }
        scales += kStepK<T>;
    }
    __device__ __forceinline__ void commit(lds_byte *lds) const
    {
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            // (scale_parts' p; scales without a mantissa stay whole)
            const uint32_t b = __builtin_bit_cast(uint32_t, scale[i]);
            const float p = __builtin_bit_cast(float, ((b >> 23) & 255) - 1 < 254 ? b & part : b);
            T e[E];
#pragma unroll
            for (int v = 0; v < E; v++) e[v] = scaled_byte<T>(bytes[i].v[v], p);
            Fragment f;
            __builtin_memcpy(&f, e, 16);
            *(__attribute__((address_space(3))) u32x4 *)(lds + (i * kGemmThreads + threadIdx.x) * 16) = f.u;
        }
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
    if constexpr (ACT == CPE_ACT_NONE && sizeof(T) == 2) {
        if (g.row_scale) {
            const float f = 1.0f / scale_parts<true>(g.row_scale[m]).f;
#pragma unroll
            for (int i = 0; i < W; i++) v[i] *= f;
        }
    }
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

// Wait until no LDS read is in flight, and (LOADS) no load either.  (The fields
// of s_waitcnt: loads in bits 0-3 and 14-15, LDS in 8-11, the rest idle.)
template <bool LOADS>
__device__ __forceinline__ void wait_for_lds()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(LOADS ? 0x0070 : 0xc07f);
    asm volatile("" ::: "memory");
}
__device__ __forceinline__ void meet()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Tiles of 128 x 128 outputs, a wave for each 64 x 64 of them, two LDS tiles of
// kStepK k, two workgroups per CU.  A step's two halves of fragments alternate
// in registers: the second half is read while the first is multiplied, then
// the waves meet and read the next step's first half while the second is
// multiplied.  At the meeting the next step's LDS tile has arrived (DIRECT: its
// loads went straight to LDS) and every wave has read the present one, whose
// place the loads of the step after next take at once.
//
// The epilogue passes through LDS, a row's 16-byte chunks permuted by the
// row, so that every row leaves as whole lines and the code that finishes a
// vector is there once.
//
// Measured (one MI355X, bf16): 4096^3 130 us (1.06 PFLOP/s, matrix units 54 %
// busy at the 1.9 GHz that such products run at); 7744 x 4096 to 1024 (dx) 74 us
// (0.88); 1936 x 1024 to 4096 with GELU and z kept 28 us.  f32 4096^3 970 us
// (0.14).  A smaller share of LDS reads (larger tiles) gains only where no split
// is needed; deeper staging and 32 x 32 instructions gain nothing.
constexpr int kBand = 8;
// PACKED: B is rows in 8 bits; 1: of whole chunks, 2: ragged.
template <typename T, bool A_ACROSS, bool B_ACROSS, bool DIRECT, int ACT, int PACKED = 0>
__global__ __launch_bounds__(kGemmThreads, 2) void k_gemm(GemmArgs g)
{
    using A = Operand<T, A_ACROSS, DIRECT>;
    using B = std::conditional_t<PACKED != 0, PackedOperand<T, PACKED == 2>, Operand<T, B_ACROSS, DIRECT>>;
    constexpr int kStage = A::kBytes + B::kBytes, W = kTile / 32;       // fragments of a wave's rows
    __shared__ __align__(1024) unsigned char smem[2 * kStage];
    static_assert(2 * kStage >= kTile * kTile * 4, "the epilogue's tile fits");
    const int tiles = g.tiles_m * g.tiles_n;
    const int split = blockIdx.x / tiles, tile = xcd_order(blockIdx.x - split * tiles, tiles);
    // bands of eight rows of tiles, down then across: tiles at work together
    // share both operands in the XCD's L2
    const int band = tile / (kBand * g.tiles_n), in_band = tile - band * kBand * g.tiles_n;
    const int high = g.tiles_m - band * kBand < kBand ? g.tiles_m - band * kBand : kBand;
    const int m0 = (band * kBand + in_band % high) * kTile, n0 = in_band / high * kTile;
    const int k0 = split * g.k_split;
    const int len = g.k - k0 < g.k_split ? g.k - k0 : g.k_split;
    const int steps = len > 0 ? (len + kStepK<T> - 1) / kStepK<T> : 0;
    const int whole = len / kStepK<T>;      // steps without a tail
    const int wave = wave_base() >> 6, lane = threadIdx.x & 63;
    const int wm = (wave >> 1) * 64, wn = (wave & 1) * 64;
    lds_byte *lds = (lds_byte *)smem;
    A a;
    B b;
    a.init(g.a, g.lda, m0, g.m, k0);
    if constexpr (PACKED)
        b.init(g, n0, k0);
    else
        b.init(g.b, g.ldb, n0, g.n, k0);
    f32x4 acc[W][W];
#pragma unroll
    for (int i = 0; i < W; i++)
#pragma unroll
        for (int j = 0; j < W; j++) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    auto fetch = [&](auto tail, int step) __attribute__((always_inline)) {
        constexpr bool TAIL = decltype(tail)::value;
        lds_byte *to = lds + (step & 1) * kStage;
        a.template fetch<TAIL>(to, len - step * kStepK<T>);
        b.template fetch<TAIL>(to + A::kBytes, len - step * kStepK<T>);
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
    Fragment fa[2][W], fb[2][W];
    auto read = [&](int step, int half) {
        const lds_byte *la = lds + (step & 1) * kStage, *lb = la + A::kBytes;
#pragma unroll
        for (int i = 0; i < W; i++) fa[half][i] = A::read(la, wm + 16 * i, half);
#pragma unroll
        for (int j = 0; j < W; j++) fb[half][j] = B::read(lb, wn + 16 * j, half);
    };
    auto multiply = [&](int half) {
#pragma unroll
        for (int i = 0; i < W; i++)
#pragma unroll
            for (int j = 0; j < W; j++) acc[i][j] = mma<T>(fb[half][j], fa[half][i], acc[i][j]);
    };
    // step t's first half of fragments is in flight; its LDS tile and (DIRECT) the
    // next one's loads, or the next one's values in registers
    if (steps > 0) {
        fetch_any(0);
        commit(0);
        wait_for_lds<true>();
        meet();
        if (steps > 1) fetch_any(1);
        read(0, 0);
    }
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
    // no load is in flight, and every wave has read its last fragments
    typedef __attribute__((address_space(3))) f32x4 lds_quad;
    auto place = [&](int m, int n) { return (lds_quad *)(lds + (m * (kTile / 4) + ((n >> 2) ^ (m & 15))) * 16); };
#pragma unroll
    for (int i = 0; i < W; i++)
#pragma unroll
        for (int j = 0; j < W; j++) *place(wm + 16 * i + (lane & 15), wn + 16 * j + 4 * (lane >> 4)) = acc[i][j];
    __syncthreads();
    const int64_t ldpart = (g.n + 3) / 4 * 4;
    for (int q = threadIdx.x; q < kTile * kTile / 8; q += kGemmThreads) {
        const int r = q / (kTile / 8), c = q % (kTile / 8) * 8, m = m0 + r, n = n0 + c;
        if (m >= g.m || n >= g.n) continue;
        const f32x4 v0 = *place(r, c), v1 = *place(r, c + 4);
        if (g.splits > 1) {
            float *p = g.part + ((int64_t)split * g.m + m) * ldpart + n;
            *reinterpret_cast<f32x4 *>(p) = v0;
            if (n + 4 < g.n) *reinterpret_cast<f32x4 *>(p + 4) = v1;
        } else {
            float v[8] = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
            finish<ACT, T, 8>(g, m, n, v);
        }
    }
}

// The splits' partial products summed in a fixed order, then the epilogue:
// LANES neighbours-by-256/LANES share a vector of four n where there are many
// splits.
template <typename T, int LANES, int ACT>
__global__ __launch_bounds__(256) void k_gemm_join(GemmArgs g)
{
    constexpr int kVectors = 256 / LANES;
    __shared__ f32x4 lds[LANES][kVectors];
    const int quads = (g.n + 3) / 4, at = threadIdx.x % kVectors, lane = threadIdx.x / kVectors;
    const int64_t all = (int64_t)g.m * quads, q = (int64_t)blockIdx.x * kVectors + at;
    const int64_t step = all * 4;
    const float *p = g.part + q * 4;
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    if (q < all) {
#pragma unroll 4
        for (int s = lane; s < g.splits; s += LANES) v += *reinterpret_cast<const f32x4 *>(p + s * step);
    }
    if constexpr (LANES > 1) {
        lds[lane][at] = v;
        __syncthreads();
        if (lane > 0) return;
#pragma unroll
        for (int l = 1; l < LANES; l++) v += lds[l][at];
    }
    if (q < all) {
        const int m = (int)(q / quads);
        finish<ACT, T>(g, m, (int)(q - (int64_t)m * quads) * 4, v);
    }
}

// Few rows (a served token or a handful): 16 n per workgroup, its waves
// dividing k; fragments come straight from memory, since no other workgroup
// shares the weights and the rows stay in the caches.  One row of 1024 to 1024
// in f16: 4.1 us, the latency of a launch, one round of loads and the join.
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
// whole: it is laid out there once per workgroup, along k, and the workgroup
// streams strips of 64 MT rows of A past it, each read once, in whole lines,
// with the next strip's loads in flight.  A strip passes through LDS only to
// turn its rows into fragments: once the waves have theirs (16 MT rows each)
// its place is free again.
//
// B's rows within a pair of 16-row fragments are taken in the order
// n = 8 (r / 4) + 4 t + r % 4 (fragment t, row r), which leaves each lane
// eight neighbouring n of its row of A: one 16-byte store for 16-bit types.
// Bound by memory: f16 409,600 x 256 to 64 52 us (5.0 TB/s); with A's rows
// loaded straight into fragments 72 us, sixteen lines to a quarter wave.
// Chunk c of row n lies at c ^ swizzle(n), so that eight lanes' reads meet all
// the banks in that order.
template <typename T>
constexpr int kNarrowStep = 4 * kChunk<T>;       // k of one fragment
constexpr int kNarrowLds = 64 << 10;             // most bytes of B
constexpr int narrow_tiles(int ks) { return ks >= 8 ? 1 : 8 / ks; }             // MT
constexpr int narrow_strip_bytes(int ks) { return 64 * narrow_tiles(ks) * ks * 64; }
__device__ __forceinline__ int narrow_swizzle(int n) { return (n & 3) | ((n >> 3) & 1) << 2; }

// FULL: k fills the fragments.  Otherwise a row's last chunk is its last 16
// bytes, the elements that the chunk before has too masked to 0 (in B as well),
// and chunks beyond it are 0: no load leaves the row, and none is conditional.
template <typename T, int KS, bool FULL, bool B_ACROSS, int ACT>
__global__ __launch_bounds__(256, 2) void k_gemm_narrow(GemmArgs g)
{
    extern __shared__ __align__(1024) unsigned char narrow_lds[];
    constexpr int E = kChunk<T>, kRow = KS * 4;        // chunks in a row of A or B
    constexpr int MT = narrow_tiles(KS), kRows = 64 * MT, kLoads = kRows * kRow / 256, kStep = 256 / kRow;
    lds_byte *strip_lds = (lds_byte *)narrow_lds, *lds = strip_lds + narrow_strip_bytes(KS);
    const int pairs = (g.n + 31) / 32, n_pad = pairs * 32;
    // the first element of chunk c, and how many of its elements are not its own
    auto start = [&](int c) { return FULL || c * E <= g.k - E ? c * E : g.k - E; };
    auto extra = [&](int c) { return c * E - start(c); };
    // B's chunks, kSetup of a thread's in flight at a time
    constexpr int kSetup = 4;
    for (int q0 = threadIdx.x; q0 < n_pad * kRow; q0 += kSetup * 256) {
        T e[kSetup][E];
        int place[kSetup];
#pragma unroll
        for (int u = 0; u < kSetup; u++) {
            const int q = q0 + u * 256;
            // (across k neighbouring threads read neighbouring n)
            const int n = B_ACROSS ? q % n_pad : q / kRow, c = B_ACROSS ? q / n_pad : q % kRow;
            const bool on = q < n_pad * kRow && n < g.n;
            const int k0 = start(c), skip = on ? extra(c) : E;
            const T *p = static_cast<const T *>(g.b) + (B_ACROSS ? (int64_t)k0 * g.ldb + n : (int64_t)n * g.ldb + k0);
            place[u] = q < n_pad * kRow ? (n * kRow + (c ^ narrow_swizzle(n))) * 16 : -1;
            if constexpr (B_ACROSS) {
#pragma unroll
                for (int i = 0; i < E; i++) e[u][i] = i >= skip ? p[i * g.ldb] : (T)0.0f;
            } else {
                Vec<T, E> v;
                if (on) v = load_vec<T, E>(p);
#pragma unroll
                for (int i = 0; i < E; i++) e[u][i] = i >= skip ? v.v[i] : (T)0.0f;
            }
        }
#pragma unroll
        for (int u = 0; u < kSetup; u++) {
            Fragment f;
            __builtin_memcpy(&f, e[u], 16);
            if (place[u] >= 0) *(__attribute__((address_space(3))) u32x4 *)(lds + place[u]) = f.u;
        }
    }
    const int lane = threadIdx.x & 63, j = lane & 15, c = lane >> 4;
    const int row0 = (wave_base() >> 6) * 16 * MT;       // this wave's rows of a strip
    const int strips = (int)(((int64_t)g.m + kRows - 1) / kRows);
    // this thread's chunk of a row, and its rows of a strip
    const int my_chunk = threadIdx.x % kRow, my_row = threadIdx.x / kRow;
    const int my_start = start(my_chunk), my_extra = extra(my_chunk);
    Vec<T, E> next[kLoads];
    auto fetch = [&](int strip) {
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const int m = strip * kRows + my_row + i * kStep;       // (rows beyond the last repeat it)
            next[i] = load_vec<T, E>(static_cast<const T *>(g.a) + (m < g.m ? m : g.m - 1) * g.lda + my_start);
        }
    };
    int strip = blockIdx.x;
    if (strip < strips) fetch(strip);
    const int row = 8 * (j >> 2) + (j & 3);
    for (; strip < strips; strip += gridDim.x) {
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const int r = my_row + i * kStep;
            Fragment f;
            __builtin_memcpy(&f, &next[i], 16);
            if constexpr (!FULL) {
#pragma unroll
                for (int d = 0; d < 4; d++) {
                    if constexpr (sizeof(T) == 4)
                        f.u[d] = d >= my_extra ? f.u[d] : 0u;
                    else
                        f.u[d] &= (2 * d >= my_extra ? 0xffffu : 0u) | (2 * d + 1 >= my_extra ? 0xffff0000u : 0u);
                }
            }
            *(__attribute__((address_space(3))) u32x4 *)(strip_lds + (r * kRow + (my_chunk ^ (r & 7))) * 16) = f.u;
        }
        wait_for_lds<false>();
        meet();
        if (strip + (int)gridDim.x < strips) fetch(strip + gridDim.x);
        Fragment fa[MT][KS];
#pragma unroll
        for (int t = 0; t < MT; t++)
#pragma unroll
            for (int s = 0; s < KS; s++) {
                const int r = row0 + 16 * t + j;
                fa[t][s].u = *(const __attribute__((address_space(3))) u32x4 *)(
                    strip_lds + (r * kRow + ((4 * s + c) ^ (r & 7))) * 16);
            }
        wait_for_lds<false>();
        meet();
        for (int p = 0; p < pairs; p++) {
            f32x4 acc[MT][2];
#pragma unroll
            for (int t = 0; t < MT; t++) acc[t][0] = acc[t][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int s = 0; s < KS; s++)
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    const int n = 32 * p + row + 4 * h;
                    Fragment fb;
                    fb.u = *(const __attribute__((address_space(3))) u32x4 *)(
                        lds + (n * kRow + ((4 * s + c) ^ narrow_swizzle(n))) * 16);
#pragma unroll
                    for (int t = 0; t < MT; t++) acc[t][h] = mma<T>(fb, fa[t][s], acc[t][h]);
                }
            const int n = 32 * p + 8 * c;
#pragma unroll
            for (int t = 0; t < MT; t++) {
                const int m = strip * kRows + row0 + 16 * t + j;
                if (m < g.m && n < g.n) {
                    float v[8] = {acc[t][0][0], acc[t][0][1], acc[t][0][2], acc[t][0][3],
                                  acc[t][1][0], acc[t][1][1], acc[t][1][2], acc[t][1][3]};
                    finish<ACT, T, 8>(g, m, n, v);
                }
            }
        }
    }
}

// dz = dy act'(preact), rounded (the products' operand), and its column sums
// over this workgroup's rows, unrounded.  Bound by memory and, for GELU, the
// vector unit (61 % busy): 46 us for 7744 x 4096 in bf16 (4.1 TB/s).  A workgroup
// covers g.slab vectors of V columns (blockIdx.y) and 256 / vectors rows at a time.
// PACKED: preact is rows in 8 bits, and dz is multiplied by the mantissa of its
// row's scale of x where the products take it so.
template <typename T, int V, int ACT, bool PACKED>
__global__ __launch_bounds__(256) void k_act_grad(GradArgs g)
{
    using Z = std::conditional_t<PACKED, int8_t, T>;
    __shared__ float lds[256 * V];
    const int all = g.n / V, first = blockIdx.y * g.slab, here = all - first < g.slab ? all - first : g.slab;
    const int rows = 256 / here, row = threadIdx.x / here, col = threadIdx.x - row * here;
    const int64_t span = (g.rows + (int64_t)g.blocks - 1) / g.blocks, lo = span * blockIdx.x;
    const int64_t hi = lo + span < g.rows ? lo + span : g.rows;
    float sum[V];
#pragma unroll
    for (int v = 0; v < V; v++) sum[v] = 0.0f;
    if (row < rows) {
        const int n = (first + col) * V;
        const T *pd = static_cast<const T *>(g.dy) + n;
        const Z *pz = static_cast<const Z *>(g.preact) + n;
        T *po = static_cast<T *>(g.dz) + n;
        constexpr int U = kSumUnroll;
        for (int64_t r = lo + row; r < hi; r += U * rows) {
            Vec<T, V> d[U];
            Vec<Z, V> z[U];
            [[maybe_unused]] float z_scale[U], x_scale[U];
#pragma unroll
            for (int u = 0; u < U; u++) {
                const int64_t at = r + u * rows;
                if (at < hi) {
                    d[u] = load_vec<T, V>(pd + at * g.ldd);
                    if (ACT != CPE_ACT_NONE) z[u] = load_vec<Z, V>(pz + at * g.ldp);
                    if constexpr (PACKED) {
                        z_scale[u] = g.z_scale[at];
                        x_scale[u] = folds(ACT, sizeof(T)) ? g.x_scale[at] : 1.0f;
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < U; u++) {
                const int64_t at = r + u * rows;
                if (at >= hi) continue;
                Vec<T, V> o;
                [[maybe_unused]] const float f = PACKED ? scale_parts<true>(x_scale[u]).f : 1.0f;
#pragma unroll
                for (int v = 0; v < V; v++) {
                    float dz = (float)d[u].v[v];
                    if constexpr (ACT != CPE_ACT_NONE)
                        dz *= activate_grad<ACT>(PACKED ? (float)z[u].v[v] * z_scale[u] : (float)z[u].v[v]);
                    sum[v] += dz;
                    if constexpr (PACKED && folds(ACT, sizeof(T))) dz *= f;
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
    float *out = g.blocks == 1 ? g.sums : g.part + (int64_t)blockIdx.x * g.n;
    for (int i = threadIdx.x; i < here * V; i += 256) {
        float s = 0.0f;
        for (int r = 0; r < rows; r++) s += lds[r * here * V + i];
        out[first * V + i] = s;
    }
}

// sums[n] over the workgroups' partials: 32 columns (a cache line) per
// workgroup, 32 lanes of partials each.
[[maybe_unused]] __global__ __launch_bounds__(1024) void k_column_join(GradArgs g)
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

// The whole gradient of a narrow product in one pass over its rows: x, dy and
// preact are read once and dx is written, which is all the memory it needs (the
// three products apart read x and dz again and write dz).  A workgroup of eight
// waves takes strips of 64 rows: it forms dz in registers (and its column sums,
// unrounded), writes dz, rounded, and x to LDS, and from there
//   dx = dz w      each wave for its 16 KT columns of dx, w in registers;
//   dw += dz^T x   each wave for the same columns, all n, over the strip's rows
//                  read back transposed; summed in registers to the end.
// The next strip's loads are in flight meanwhile, and the LDS tiles are
// double, so the waves meet once a strip.  Bound by memory: f16 409,600 rows, 256
// to 64 with SiLU, 104 us (5.0 TB/s), and 5 us for the join of the partial dw.
//
// LDS rows of 16-byte chunks, chunk c of row r at c ^ f(r) (rows of 128 bytes)
// or c ^ 2 f(r): f differs over eight rows in a row and over the rows r .. r+3,
// r+8 .. r+11 that half a transposing read's lanes name.
constexpr int kNarrowThreads = 512;
__device__ __forceinline__ int strip_swizzle(int row, int chunks)
{
    const int f = (row & 3) | (((row >> 3) ^ (row >> 2)) & 1) << 2;
    return chunks == 8 ? f : 2 * f;
}

// PACKED: x and preact are rows in 8 bits, which become elements on their way
// to LDS; where dz is rounded anyway it takes the mantissas of x's scales, and
// dx is divided by them.
template <typename T, int NT, int KT, int ACT, bool PACKED>
__global__ __launch_bounds__(kNarrowThreads, 2) void k_narrow_grad(WholeGradArgs a)
{
    using X = std::conditional_t<PACKED, int8_t, T>;
    constexpr bool kFold = PACKED && folds(ACT, sizeof(T));
    constexpr int kZChunks = NT * 2, kXChunks = KT * 16;                  // chunks of an LDS row
    constexpr int kZBytes = kStripRows * kZChunks * 16, kXBytes = kStripRows * kXChunks * 16;
    constexpr int kZLoads = kStripRows * kZChunks / kNarrowThreads, kXLoads = kStripRows * kXChunks / kNarrowThreads;
    constexpr int NS = NT / 2;                                            // fragments of n
    static_assert(sizeof(T) == 2 && kZLoads >= 1, "");
    __shared__ __align__(1024) unsigned char smem[2 * (kZBytes + kXBytes)];
    __shared__ float inverse[2][kFold ? kStripRows : 1];       // 1 / the mantissas of a strip's rows
    lds_byte *lds = (lds_byte *)smem;
    const int lane = threadIdx.x & 63, j = lane & 15, c = lane >> 4;
    const int k_wave = (wave_base() >> 6) * 16 * KT;
    const int strips = (a.rows + kStripRows - 1) / kStripRows;
    // w as the first operand, k along the fragment's rows (in the order that
    // leaves a lane 8 neighbouring k where KT is even), n along the reduction
    Fragment fw[KT][NS];
    auto k_of = [&](int kt, int row) {
        return k_wave + (KT % 2 == 0 ? 32 * (kt >> 1) + 8 * (row >> 2) + 4 * (kt & 1) + (row & 3) : 16 * kt + row);
    };
#pragma unroll
    for (int kt = 0; kt < KT; kt++)
#pragma unroll
        for (int s = 0; s < NS; s++) {
            T e[8];
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const int n = 32 * s + 8 * c + i, k = k_of(kt, j);
                e[i] = a.dx && n < a.n && k < a.k ? static_cast<const T *>(a.w)[n * a.ldw + k] : (T)0.0f;
            }
            __builtin_memcpy(&fw[kt][s], e, 16);
        }
    // this thread's chunks of a strip: their rows and columns
    const int z_col = threadIdx.x % kZChunks * 8, z_row = threadIdx.x / kZChunks;
    const int x_col = threadIdx.x % kXChunks * 8, x_row = threadIdx.x / kXChunks;
    constexpr int kZStep = kNarrowThreads / kZChunks, kXStep = kNarrowThreads / kXChunks;
    const bool z_on = z_col < a.n, x_on = x_col < a.k && a.dw;
    Vec<T, 8> vd[kZLoads];
    Vec<X, 8> vz[kZLoads], vx[kXLoads];
    [[maybe_unused]] float z_scale[kZLoads], z_row_scale[kZLoads], x_scale[kXLoads];
    auto fetch = [&](int strip) {
        // rows and columns that are not there repeat others, and are set to 0 later
        const int r0 = strip * kStripRows;
#pragma unroll
        for (int i = 0; i < kZLoads; i++) {
            const int r = r0 + z_row + i * kZStep, rr = r < a.rows ? r : a.rows - 1, cc = z_on ? z_col : 0;
            vd[i] = load_vec<T, 8>(static_cast<const T *>(a.dy) + rr * a.ldd + cc);
            if (ACT != CPE_ACT_NONE) vz[i] = load_vec<X, 8>(static_cast<const X *>(a.preact) + rr * a.ldp + cc);
            if constexpr (PACKED && ACT != CPE_ACT_NONE) z_scale[i] = a.z_scale[rr];
            if constexpr (kFold) z_row_scale[i] = a.x_scale[rr];
        }
        if (!a.dw) return;
#pragma unroll
        for (int i = 0; i < kXLoads; i++) {
            const int r = r0 + x_row + i * kXStep, rr = r < a.rows ? r : a.rows - 1;
            vx[i] = load_vec<X, 8>(static_cast<const X *>(a.x) + rr * a.ldx + (x_on ? x_col : 0));
            if constexpr (PACKED) x_scale[i] = a.x_scale[rr];
        }
    };
    f32x4 acc[NT][KT];
    float sums[8];
#pragma unroll
    for (int n = 0; n < NT; n++)
#pragma unroll
        for (int k = 0; k < KT; k++) acc[n][k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 8; i++) sums[i] = 0.0f;
    int strip = blockIdx.x, turn = 0;
    if (strip < strips) fetch(strip);
    for (; strip < strips; strip += gridDim.x, turn ^= 1) {
        lds_byte *lz = lds + turn * (kZBytes + kXBytes), *lx = lz + kZBytes;
        const int r0 = strip * kStripRows;
#pragma unroll
        for (int i = 0; i < kZLoads; i++) {
            const int r = z_row + i * kZStep;
            const bool on = z_on && r0 + r < a.rows;
            [[maybe_unused]] float factor = 1.0f;
            if constexpr (kFold) {
                factor = scale_parts<true>(z_row_scale[i]).f;
                if (z_col == 0) inverse[turn][r] = 1.0f / factor;
            }
            T e[8];
#pragma unroll
            for (int v = 0; v < 8; v++) {
                float dz = (float)vd[i].v[v];
                if constexpr (ACT != CPE_ACT_NONE) {
                    if constexpr (PACKED)
                        dz *= activate_grad<ACT>((float)vz[i].v[v] * z_scale[i]);
                    else
                        dz *= activate_grad<ACT>((float)vz[i].v[v]);
                }
                dz = on ? dz : 0.0f;
                sums[v] += dz;
                if constexpr (kFold) dz *= factor;
                e[v] = (T)dz;
            }
            Fragment f;
            __builtin_memcpy(&f, e, 16);
            *(__attribute__((address_space(3))) u32x4 *)(
                lz + (r * kZChunks + ((z_col >> 3) ^ strip_swizzle(r, kZChunks))) * 16) = f.u;
        }
        if (a.dw) {
#pragma unroll
            for (int i = 0; i < kXLoads; i++) {
                const int r = x_row + i * kXStep;
                Fragment f;
                if constexpr (PACKED) {
                    const float p = scale_parts<kFold>(x_scale[i]).p;
                    T e[8];
#pragma unroll
                    for (int v = 0; v < 8; v++) e[v] = scaled_byte<T>(vx[i].v[v], p);
                    __builtin_memcpy(&f, e, 16);
                } else {
                    __builtin_memcpy(&f, &vx[i], 16);
                }
                if (!x_on || r0 + r >= a.rows) f.u = u32x4{0, 0, 0, 0};
                *(__attribute__((address_space(3))) u32x4 *)(
                    lx + (r * kXChunks + ((x_col >> 3) ^ strip_swizzle(r, kXChunks))) * 16) = f.u;
            }
        }
        wait_for_lds<false>();
        meet();
        if (strip + (int)gridDim.x < strips) fetch(strip + gridDim.x);
        if (a.dw && k_wave < a.k) {
            // the fragment of sixteen columns from `col` on over rows 32 s .. 32 s + 31, transposed
            auto column = [&](const lds_byte *tile, int chunks, int col, int s) {
                Fragment f;
#pragma unroll
                for (int t = 0; t < 2; t++) {
                    const int r = 32 * s + 8 * c + 4 * t + (j >> 2), chunk = (col >> 3) + ((j & 3) >> 1);
                    f.s[t] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(
                        tile + (r * chunks + (chunk ^ strip_swizzle(r, chunks))) * 16 + (j & 1) * 8));
                }
                return f;
            };
#pragma unroll
            for (int s = 0; s < kStripRows / 32; s++) {
                Fragment fz[NT], fx[KT];
#pragma unroll
                for (int k = 0; k < KT; k++) fx[k] = column(lx, kXChunks, k_wave + 16 * k, s);
#pragma unroll
                for (int n = 0; n < NT; n++) fz[n] = column(lz, kZChunks, 16 * n, s);
#pragma unroll
                for (int n = 0; n < NT; n++)
#pragma unroll
                    for (int k = 0; k < KT; k++) acc[n][k] = mma<T>(fx[k], fz[n], acc[n][k]);
            }
        }
        if (a.dx && k_wave < a.k) {
#pragma unroll
            for (int t = 0; t < kStripRows / 16; t++) {
                const int r = 16 * t + j;
                [[maybe_unused]] const float f = kFold ? inverse[turn][r] : 1.0f;
                Fragment fz[NS];
#pragma unroll
                for (int s = 0; s < NS; s++)
                    fz[s].u = *(const __attribute__((address_space(3))) u32x4 *)(
                        lz + (r * kZChunks + ((4 * s + c) ^ strip_swizzle(r, kZChunks))) * 16);
                constexpr int P = KT % 2 == 0 ? 2 : 1;
#pragma unroll
                for (int kt = 0; kt < KT; kt += P) {
                    Vec<T, 4 * P> o;
#pragma unroll
                    for (int h = 0; h < P; h++) {
                        f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                        for (int s = 0; s < NS; s++) v = mma<T>(fw[kt + h][s], fz[s], v);
#pragma unroll
                        for (int i = 0; i < 4; i++) o.v[4 * h + i] = (T)(kFold ? v[i] * f : v[i]);
                    }
                    const int k = k_of(kt, 4 * c);
                    if (r0 + r < a.rows && k < a.k)
                        store_vec<T, 4 * P>(static_cast<T *>(a.dx) + (r0 + r) * a.lddx + k, o);
                }
            }
        }
    }
    if (a.dw) {
#pragma unroll
        for (int n = 0; n < NT; n++)
#pragma unroll
            for (int k = 0; k < KT; k++) {
                const int nn = 16 * n + j, kk = k_wave + 16 * k + 4 * c;
                if (nn < a.n && kk < a.k)
                    *reinterpret_cast<f32x4 *>(a.part + ((int64_t)blockIdx.x * a.n + nn) * a.k + kk) = acc[n][k];
            }
    }
    if (a.dbias) {
        float *row = reinterpret_cast<float *>(smem);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; i++) row[z_row * (kZChunks * 8) + z_col + i] = sums[i];
        __syncthreads();
        if ((int)threadIdx.x < a.n) {
            float s = 0.0f;
            for (int r = 0; r < kZStep; r++) s += row[r * (kZChunks * 8) + threadIdx.x];
            a.part_sums[(int64_t)blockIdx.x * a.n + threadIdx.x] = s;
        }
    }
}

// The gradient of few rows (at most 64): dz is formed where it is needed, since
// there is little of it, and neither scratch nor a join is.
//
// dx: 16 columns per workgroup, its waves dividing n; w's column of each lane is
// gathered, sixteen lanes side by side.
template <typename T, int MT, int ACT, bool PACKED>
__global__ __launch_bounds__(1024) void k_rows_dx(WholeGradArgs a)
{
    constexpr bool kFold = PACKED && folds(ACT, sizeof(T));
    __shared__ f32x4 joined[16][MT][64];
    constexpr int E = kChunk<T>, kStep = 4 * E;
    const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6, lane = threadIdx.x & 63;
    const int j = lane & 15, c = lane >> 4, k = blockIdx.x * 16 + j;
    const int steps = (a.n + kStep - 1) / kStep, each = (steps + waves - 1) / waves;
    const int lo = wave * each, hi = lo + each < steps ? lo + each : steps;
    const T *w = static_cast<const T *>(a.w) + (k < a.k ? k : a.k - 1);      // (columns that are not there: the last)
    f32x4 acc[MT];
#pragma unroll
    for (int i = 0; i < MT; i++) acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int s = lo; s < hi; s++) {
        const int n0 = s * kStep + c * E, left = a.n - n0;
        Fragment fw, fz[MT];
        T e[E];
#pragma unroll
        for (int i = 0; i < E; i++) e[i] = i < left ? w[(n0 + i) * a.ldw] : (T)0.0f;
        __builtin_memcpy(&fw, e, 16);
#pragma unroll
        for (int t = 0; t < MT; t++) {
            const int m = 16 * t + j, here = m < a.rows ? left : 0;
            fz[t].u = load_chunk<T>(static_cast<const T *>(a.dy) + m * a.ldd + n0, here);
            if constexpr (ACT != CPE_ACT_NONE) {
                float z[E];
                [[maybe_unused]] float f = 1.0f;
                if constexpr (PACKED) {
                    const int8_t *pz = static_cast<const int8_t *>(a.preact) + m * a.ldp + n0;
                    const float s = here > 0 ? a.z_scale[m] : 0.0f;
                    if (kFold && here > 0) f = scale_parts<true>(a.x_scale[m]).f;
#pragma unroll
                    for (int i = 0; i < E; i++) z[i] = i < here ? (float)pz[i] * s : 0.0f;
                } else {
                    Fragment raw;
                    raw.u = load_chunk<T>(static_cast<const T *>(a.preact) + m * a.ldp + n0, here);
                    T ez[E];
                    __builtin_memcpy(ez, &raw, 16);
#pragma unroll
                    for (int i = 0; i < E; i++) z[i] = (float)ez[i];
                }
                __builtin_memcpy(e, &fz[t], 16);
#pragma unroll
                for (int i = 0; i < E; i++) {
                    const float dz = (float)e[i] * activate_grad<ACT>(z[i]);
                    e[i] = (T)(kFold ? dz * f : dz);
                }
                __builtin_memcpy(&fz[t], e, 16);
            }
        }
#pragma unroll
        for (int t = 0; t < MT; t++) acc[t] = mma<T>(fw, fz[t], acc[t]);
    }
#pragma unroll
    for (int t = 0; t < MT; t++) joined[wave][t][lane] = acc[t];
    __syncthreads();
    if (wave < MT) {
        f32x4 v = joined[0][wave][lane];
        for (int i = 1; i < waves; i++) v += joined[i][wave][lane];
        const int m = 16 * wave + j, k4 = blockIdx.x * 16 + 4 * c;
        if (m < a.rows) {
            T *out = static_cast<T *>(a.dx) + m * a.lddx + k4;
            if constexpr (kFold) v *= 1.0f / scale_parts<true>(a.x_scale[m]).f;
#pragma unroll
            for (int i = 0; i < 4; i++)
                if (k4 + i < a.k) out[i] = (T)v[i];
        }
    }
}

// dw and dbias: 64 n by 64 k per workgroup, 16 n of them per wave.
template <typename T, int ACT, bool PACKED>
__global__ __launch_bounds__(256) void k_rows_dw(WholeGradArgs a)
{
    constexpr bool kFold = PACKED && folds(ACT, sizeof(T));
    constexpr int E = kChunk<T>, kStep = 4 * E;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, j = lane & 15, c = lane >> 4;
    const int n = blockIdx.y * 64 + wave * 16 + j, k0 = blockIdx.x * 64;
    const bool n_on = n < a.n;
    f32x4 acc[4];
    float sum = 0.0f;
#pragma unroll
    for (int t = 0; t < 4; t++) acc[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int m0 = c * E; m0 < (a.rows + kStep - 1) / kStep * kStep; m0 += kStep) {
        Fragment fz, fx[4];
        T e[E];
#pragma unroll
        for (int i = 0; i < E; i++) {
            const int m = m0 + i;
            float dz = 0.0f;
            [[maybe_unused]] float f = 1.0f;
            if (n_on && m < a.rows) {
                dz = (float)static_cast<const T *>(a.dy)[m * a.ldd + n];
                if constexpr (ACT != CPE_ACT_NONE) {
                    if constexpr (PACKED)
                        dz *= activate_grad<ACT>((float)static_cast<const int8_t *>(a.preact)[m * a.ldp + n] * a.z_scale[m]);
                    else
                        dz *= activate_grad<ACT>((float)static_cast<const T *>(a.preact)[m * a.ldp + n]);
                }
                if constexpr (kFold) f = scale_parts<true>(a.x_scale[m]).f;
            }
            sum += dz;
            e[i] = (T)(kFold ? dz * f : dz);
        }
        __builtin_memcpy(&fz, e, 16);
        if (!a.dw) continue;
#pragma unroll
        for (int t = 0; t < 4; t++) {
            const int k = k0 + 16 * t + j;
#pragma unroll
            for (int i = 0; i < E; i++) {
                const bool there = k < a.k && m0 + i < a.rows;
                if constexpr (PACKED)
                    e[i] = there ? scaled_byte<T>(static_cast<const int8_t *>(a.x)[(m0 + i) * a.ldx + k],
                                              scale_parts<kFold>(a.x_scale[m0 + i]).p)
                                 : (T)0.0f;
                else
                    e[i] = there ? static_cast<const T *>(a.x)[(m0 + i) * a.ldx + k] : (T)0.0f;
            }
            __builtin_memcpy(&fx[t], e, 16);
        }
#pragma unroll
        for (int t = 0; t < 4; t++) acc[t] = mma<T>(fx[t], fz, acc[t]);
    }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (a.dbias && blockIdx.x == 0 && c == 0 && n_on) a.dbias[n] = sum;
    if (!a.dw || !n_on) return;
#pragma unroll
    for (int t = 0; t < 4; t++) {
        const int k = k0 + 16 * t + 4 * c;
        T *out = static_cast<T *>(a.dw) + n * a.lddw + k;
        if (k + 4 <= a.k) {
            Vec<T, 4> o;
#pragma unroll
            for (int i = 0; i < 4; i++) o.v[i] = (T)acc[t][i];
            store_vec<T, 4>(out, o);
        } else {
#pragma unroll
            for (int i = 0; i < 4; i++)
                if (k + i < a.k) out[i] = (T)acc[t][i];
        }
    }
}

// -- launches -----------------------------------------------------------------------

template <typename T>
bool direct_ok(const GemmArgs &g)
{
    constexpr int E = kChunk<T>;
    auto ok = [](const void *p, int64_t ld, int width) {     // (a tile's offsets stay in the buffer)
        return aligned_to(p, 16) && ld % E == 0 && width % E == 0 && ld < (int64_t)kBufferBytes / 2048;
    };
    return ok(g.a, g.lda, g.a_cols ? g.m : g.k) && (g.b_scale || ok(g.b, g.ldb, g.b_cols ? g.n : g.k));
}

// Workgroups dividing k where the tiles alone leave half or more of the chip
// empty.  A split's partial tiles are written, read again and joined in a
// launch of their own, 5 us or more: so each split has at least kLeast steps
// (bf16 2048 x 1024 to 512: 11 us in one piece, 22 in splits of four steps;
// binary32 steps take four times as long), and the splits fill one place per
// CU, both places only where 2 kLeast steps are left to each (1936 x 4096 to
// 1024: 35 us on 512 places, 40 on 256, 53 in one piece).
template <typename T>
void choose_splits(GemmArgs &g)
{
    constexpr int kLeast = least_steps(sizeof(T));
    const int64_t tiles = (int64_t)g.tiles_m * g.tiles_n, steps = g.k > 0 ? ceil_div(g.k, kStepK<T>) : 1;
    int64_t splits = kSplitTiles / tiles;
    if (splits > 1 && steps / splits < 2 * kLeast) {
        splits = kSplitTiles / 2 / tiles;
        if (splits > steps / kLeast) splits = steps / kLeast;
    }
    const int64_t one = (int64_t)g.m * ceil_div(g.n, 4) * 16;      // a split's partial outputs, in the scratch
    if (splits > g.part_bytes / one) splits = g.part_bytes / one;
    if (splits < 1) splits = 1;
    const int64_t each = ceil_div(steps, splits);
    g.k_split = (int32_t)(each * kStepK<T>);
    g.splits = (int32_t)ceil_div(steps, each);
}

template <typename T, bool A_ACROSS, bool B_ACROSS, int ACT, int PACKED = 0>
hipError_t launch_tiles(GemmArgs g, hipStream_t stream)
{
    g.tiles_m = (int32_t)ceil_div(g.m, kTile);
    g.tiles_n = (int32_t)ceil_div(g.n, kTile);
    choose_splits<T>(g);
    const dim3 grid(g.tiles_m * g.tiles_n * g.splits);
    if (direct_ok<T>(g))
        hipLaunchKernelGGL((k_gemm<T, A_ACROSS, B_ACROSS, true, ACT, PACKED>), grid, dim3(kGemmThreads), 0, stream, g);
    else
        hipLaunchKernelGGL((k_gemm<T, A_ACROSS, B_ACROSS, false, ACT, PACKED>), grid, dim3(kGemmThreads), 0, stream, g);
    if (hipError_t e = hipGetLastError(); e != hipSuccess || g.splits == 1) return e;
    const int64_t quads = (int64_t)g.m * ((g.n + 3) / 4);
    if (g.splits <= 8)
        hipLaunchKernelGGL((k_gemm_join<T, 1, ACT>), dim3((unsigned)ceil_div(quads, 256)), dim3(256), 0, stream, g);
    else
        hipLaunchKernelGGL((k_gemm_join<T, 16, ACT>), dim3((unsigned)ceil_div(quads, 16)), dim3(256), 0, stream, g);
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
// In f16, 200,000 rows: 256 to 64 34 us against 47 in tiles, 100 to 65 31 against
// 49; with more columns the strips' epilogues outlast their loads (64 to 256 65
// against 60, 128 to 256 96 against 70).
template <typename T>
bool narrow_fits(const GemmArgs &g)
{
    return g.k >= kChunk<T> && narrow_steps<T>(g.k) > 0 && g.n <= 128 && narrow_bytes<T>(g) <= kNarrowLds;
}

template <typename T, bool B_ACROSS, int ACT>
hipError_t launch_narrow(const GemmArgs &g, hipStream_t stream)
{
    // as many workgroups as run at once, by LDS and registers
    const int ks = narrow_steps<T>(g.k), bytes = narrow_bytes<T>(g) + narrow_strip_bytes(ks);
    const int64_t strips = ceil_div(g.m, 64 * narrow_tiles(ks)), by_lds = (160 << 10) / bytes;
    const int64_t most = 256 * (by_lds < 2 ? by_lds : 2);
    const dim3 grid((unsigned)(strips < most ? strips : most));
    auto launch = [&](auto steps) {
        constexpr int KS = decltype(steps)::value;
        if (g.k == KS * kNarrowStep<T>)
            hipLaunchKernelGGL((k_gemm_narrow<T, KS, true, B_ACROSS, ACT>), grid, dim3(256), bytes, stream, g);
        else
            hipLaunchKernelGGL((k_gemm_narrow<T, KS, false, B_ACROSS, ACT>), grid, dim3(256), bytes, stream, g);
    };
    switch (narrow_steps<T>(g.k)) {
    case 2: launch(std::integral_constant<int, 2>{}); break;
    case 4: launch(std::integral_constant<int, 4>{}); break;
    case 8: launch(std::integral_constant<int, 8>{}); break;
    default: launch(std::integral_constant<int, 16>{}); break;
    }
    return hipGetLastError();
}

template <typename T, int ACT>
hipError_t launch_forward(const GemmArgs &g, hipStream_t stream)
{
    // few rows: 10 us against 13 at 64 x 1024 to 1024; with more than 16 rows only
    // while w stays in the caches (64 x 4096 to 4096: 23 us, in tiles 16)
    if (g.m <= 16 || (g.m <= 64 && (int64_t)g.n * g.k <= (int64_t)1 << 22)) return launch_rows<T, ACT>(g, stream);
    if (narrow_fits<T>(g)) return launch_narrow<T, false, ACT>(g, stream);
    return launch_tiles<T, false, false, ACT>(g, stream);
}

// Rows in one launch: the grid stays under kMaxTiles.
template <typename T>
hipError_t launch_gemm_type(const GemmArgs &all, hipStream_t stream)
{
    if (all.a_cols && all.b_cols)
        return !all.b_scale                  ? launch_tiles<T, true, true, CPE_ACT_NONE>(all, stream)
               : all.n % kChunk<T> == 0 ? launch_tiles<T, true, true, CPE_ACT_NONE, 1>(all, stream)
                                             : launch_tiles<T, true, true, CPE_ACT_NONE, 2>(all, stream);
    const int64_t tiles_n = ceil_div(all.n, kTile), most = kMaxTiles / tiles_n * kTile;
    for (int64_t m = 0; m < all.m; m += most) {
        GemmArgs g = all;
        g.a = static_cast<const T *>(all.a) + m * all.lda;
        g.out = static_cast<T *>(all.out) + m * all.ldo;
        if (all.residual) g.residual = static_cast<const T *>(all.residual) + m * all.ldr;
        if (all.preact) g.preact = static_cast<T *>(all.preact) + m * all.ldp;
        if (all.row_scale) g.row_scale = all.row_scale + m;
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
    // few enough rows for one workgroup per slab of 32 vectors: no join
    const int vectors = g.n / V;
    g.slab = 32;
    int rows = 256 / (vectors < g.slab ? vectors : g.slab);
    g.blocks = 1;
    if (g.rows > 16 * rows) {
        g.slab = 256;
        rows = vectors >= 256 ? 1 : 256 / vectors;
        const int64_t slabs = ceil_div(vectors, 256);
        const int64_t want = ceil_div(g.rows, kSumUnroll * (int64_t)rows);
        const int64_t cap = kSumBlocks / slabs < 1 ? 1 : kSumBlocks / slabs;
        g.blocks = (int32_t)(want < 1 ? 1 : want < cap ? want : cap);
    }
    const int64_t slabs = ceil_div(vectors, g.slab);
    const dim3 grid(g.blocks, (unsigned)slabs);
    auto launch = [&](auto act) {
        constexpr int ACT = decltype(act)::value;
        if (ACT != CPE_ACT_NONE && g.z_scale)
            hipLaunchKernelGGL((k_act_grad<T, V, ACT, ACT != CPE_ACT_NONE>), grid, dim3(256), 0, stream, g);
        else
            hipLaunchKernelGGL((k_act_grad<T, V, ACT, false>), grid, dim3(256), 0, stream, g);
    };
    switch (g.act) {
    case CPE_ACT_RELU: launch(std::integral_constant<int, CPE_ACT_RELU>{}); break;
    case CPE_ACT_SILU: launch(std::integral_constant<int, CPE_ACT_SILU>{}); break;
    case CPE_ACT_GELU: launch(std::integral_constant<int, CPE_ACT_GELU>{}); break;
    default: launch(std::integral_constant<int, CPE_ACT_NONE>{}); break;
    }
    if (hipError_t e = hipGetLastError(); e != hipSuccess || !g.sums || g.blocks == 1) return e;
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

// dw and dbias over the workgroups' partials, four values per 16 lanes.
template <typename T>
__global__ __launch_bounds__(256) void k_narrow_grad_join(WholeGradArgs a)
{
    __shared__ f32x4 lds[16][16];
    const int at = threadIdx.x & 15, lane = threadIdx.x >> 4;
    const int64_t of_dw = a.dw ? (int64_t)a.n * (a.k / 4) : 0, all = of_dw + (a.dbias ? a.n / 4 : 0);
    const int64_t q = (int64_t)blockIdx.x * 16 + at;
    const bool is_dw = q < of_dw;
    const float *p = is_dw ? a.part + q * 4 : a.part_sums + (q - of_dw) * 4;
    const int64_t step = is_dw ? (int64_t)a.n * a.k : a.n;
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    if (q < all) {
#pragma unroll 8
        for (int s = lane; s < a.blocks; s += 16) v += *reinterpret_cast<const f32x4 *>(p + s * step);
    }
    lds[lane][at] = v;
    __syncthreads();
    if (lane > 0 || q >= all) return;
#pragma unroll
    for (int l = 1; l < 16; l++) v += lds[l][at];
    if (is_dw) {
        const int quads = a.k / 4, n = (int)(q / quads), k = (int)(q - (int64_t)n * quads) * 4;
        Vec<T, 4> o;
#pragma unroll
        for (int i = 0; i < 4; i++) o.v[i] = (T)v[i];
        store_vec<T, 4>(static_cast<T *>(a.dw) + n * a.lddw + k, o);
    } else {
        *reinterpret_cast<Vec<float, 4> *>(a.dbias + (q - of_dw) * 4) = Vec<float, 4>{{v[0], v[1], v[2], v[3]}};
    }
}

template <typename T, int NT, int KT>
hipError_t launch_narrow_grad_size(const WholeGradArgs &a, hipStream_t stream)
{
    const dim3 grid(a.blocks), block(kNarrowThreads);
    auto launch = [&](auto act) {
        constexpr int ACT = decltype(act)::value;
        if (a.x_scale)
            hipLaunchKernelGGL((k_narrow_grad<T, NT, KT, ACT, true>), grid, block, 0, stream, a);
        else
            hipLaunchKernelGGL((k_narrow_grad<T, NT, KT, ACT, false>), grid, block, 0, stream, a);
    };
    switch (a.act) {
    case CPE_ACT_RELU: launch(std::integral_constant<int, CPE_ACT_RELU>{}); break;
    case CPE_ACT_SILU: launch(std::integral_constant<int, CPE_ACT_SILU>{}); break;
    case CPE_ACT_GELU: launch(std::integral_constant<int, CPE_ACT_GELU>{}); break;
    default: launch(std::integral_constant<int, CPE_ACT_NONE>{}); break;
    }
    return hipGetLastError();
}

template <typename T>
hipError_t launch_narrow_grad_type(WholeGradArgs a, hipStream_t stream)
{
    // one workgroup per CU: a second one would double the partial dw
    const int64_t strips = ceil_div(a.rows, kStripRows);
    a.blocks = (int32_t)(strips < kNarrowGradBlocks ? strips : kNarrowGradBlocks);
    const bool wide_n = a.n > 64;
    hipError_t e;
    if (a.k <= 128)
        e = wide_n ? launch_narrow_grad_size<T, 8, 1>(a, stream) : launch_narrow_grad_size<T, 4, 1>(a, stream);
    else if (a.k <= 256)
        e = wide_n ? launch_narrow_grad_size<T, 8, 2>(a, stream) : launch_narrow_grad_size<T, 4, 2>(a, stream);
    else
        e = launch_narrow_grad_size<T, 4, 4>(a, stream);
    if (e != hipSuccess || (!a.dw && !a.dbias)) return e;
    const int64_t quads = (a.dw ? (int64_t)a.n * (a.k / 4) : 0) + (a.dbias ? a.n / 4 : 0);
    hipLaunchKernelGGL(k_narrow_grad_join<T>, dim3((unsigned)ceil_div(quads, 16)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

template <typename T, int ACT, bool PACKED>
hipError_t launch_rows_grad_form(const WholeGradArgs &a, hipStream_t stream)
{
    if (a.dx) {
        const int steps = (int)ceil_div(a.n, 4 * kChunk<T>);
        const int waves = steps >= 64 ? 16 : steps >= 16 ? 8 : 4;
        const dim3 grid((unsigned)ceil_div(a.k, 16)), block(64 * waves);
        if (a.rows <= 16)
            hipLaunchKernelGGL((k_rows_dx<T, 1, ACT, PACKED>), grid, block, 0, stream, a);
        else if (a.rows <= 32)
            hipLaunchKernelGGL((k_rows_dx<T, 2, ACT, PACKED>), grid, block, 0, stream, a);
        else
            hipLaunchKernelGGL((k_rows_dx<T, 4, ACT, PACKED>), grid, block, 0, stream, a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    if (!a.dw && !a.dbias) return hipSuccess;
    const dim3 grid(a.dw ? (unsigned)ceil_div(a.k, 64) : 1u, (unsigned)ceil_div(a.n, 64));
    hipLaunchKernelGGL((k_rows_dw<T, ACT, PACKED>), grid, dim3(256), 0, stream, a);
    return hipGetLastError();
}

template <typename T, int ACT>
hipError_t launch_rows_grad(const WholeGradArgs &a, hipStream_t stream)
{
    return a.x_scale ? launch_rows_grad_form<T, ACT, true>(a, stream) : launch_rows_grad_form<T, ACT, false>(a, stream);
}

template <typename T>
hipError_t launch_rows_grad_type(const WholeGradArgs &a, hipStream_t stream)
{
    switch (a.act) {
    case CPE_ACT_RELU: return launch_rows_grad<T, CPE_ACT_RELU>(a, stream);
    case CPE_ACT_SILU: return launch_rows_grad<T, CPE_ACT_SILU>(a, stream);
    case CPE_ACT_GELU: return launch_rows_grad<T, CPE_ACT_GELU>(a, stream);
    default: return launch_rows_grad<T, CPE_ACT_NONE>(a, stream);
    }
}

}  // namespace
}  // namespace cpe
