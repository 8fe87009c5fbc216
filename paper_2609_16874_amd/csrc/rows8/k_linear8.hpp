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
// matter and splits of k join exactly.  They are rounded to binary32 once, then
// scaled, twice: three roundings of 2^-24 in all, the last one with the bias.
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
// PAIRS: the rows of two fragments t = 0, 1 are n = 8 (r / 4) + 4 t + r % 4, which
// leaves a lane eight neighbouring n of its row of sums; the chunks' places then
// go by the bits of the row that eight lanes' reads span.
template <int R, int THREADS, bool DIRECT, bool PAIRS = false>
struct ByteOperand {
    static constexpr int kLoads = R * 8 / THREADS, kBytes = R * kStep8;
    const int8_t *base;
    uint32_t off[DIRECT ? kLoads : 1];
    const int8_t *src[DIRECT ? 1 : kLoads];
    bool there[DIRECT ? 1 : kLoads];
    u32x4 held[DIRECT ? 1 : kLoads];

    __device__ __forceinline__ static int row_of(int i) { return (i * THREADS + threadIdx.x) / 8; }
    __device__ __forceinline__ static int swizzle(int r) { return PAIRS ? (r & 3) | ((r >> 3) & 1) << 2 : r & 7; }
    __device__ __forceinline__ static int chunk_of(int i) { return (threadIdx.x & 7) ^ swizzle(row_of(i)); }

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
    // the t-th fragment of the rows from r on, for the s-th half of the step
    __device__ __forceinline__ static Bytes16 read(const lds_byte *lds, int r, int t, int s)
    {
        const int lane = threadIdx.x & 63, j = lane & 15;
        const int row = r + (PAIRS ? 32 * (t >> 1) + 8 * (j >> 2) + 4 * (t & 1) + (j & 3) : 16 * t + j);
        const int c = (4 * s + (lane >> 4)) ^ swizzle(row);
        Bytes16 f;
        f.u = *(const __attribute__((address_space(3))) u32x4 *)(lds + (row * 8 + c) * 16);
        return f;
    }
};

// W neighbouring values before the activation of row m, `left` of which exist.
// PAST: whole vectors of the outputs are stored past the caches.
template <int ACT, bool PAST, typename T, int W>
__device__ __forceinline__ void finish_scaled(const GemmArgs &g, int m, int n, int left, const float (&z)[W])
{
    T *out = static_cast<T *>(g.out) + m * g.ldo + n;
    const T *res = g.residual ? static_cast<const T *>(g.residual) + m * g.ldr + n : nullptr;
    T *pre = g.preact ? static_cast<T *>(g.preact) + m * g.ldp + n : nullptr;
    if (left >= W) {
        Vec<T, W> o, r;
        if (res) r = load_vec<T, W>(res);
        if (pre) {
#pragma unroll
            for (int i = 0; i < W; i++) o.v[i] = (T)z[i];
            store_words<PAST>(pre, o);
        }
#pragma unroll
        for (int i = 0; i < W; i++) {
            const float y = activate<ACT>(z[i]);
            o.v[i] = (T)(res ? y + (float)r.v[i] : y);
        }
        store_words<PAST>(out, o);
    } else {
#pragma unroll
        for (int i = 0; i < W; i++)
            if (i < left) {
                if (pre) pre[i] = (T)z[i];
                out[i] = (T)(activate<ACT>(z[i]) + (res ? (float)res[i] : 0.0f));
            }
    }
}

// The scales and biases of W neighbouring n, `left` of which exist.
template <int W>
struct ColumnTerms {
    float scale[W], bias[W];
    __device__ __forceinline__ ColumnTerms(const Gemm8Args &a, int n, int left)
    {
        if (left >= W) {
            const Vec<float, W> t = load_vec<float, W>(a.b_scale + n);
            Vec<float, W> b;
            if (a.g.bias) b = load_vec<float, W>(a.g.bias + n);
#pragma unroll
            for (int i = 0; i < W; i++) {
                scale[i] = t.v[i];
                bias[i] = a.g.bias ? b.v[i] : 0.0f;
            }
        } else {
#pragma unroll
            for (int i = 0; i < W; i++) {
                scale[i] = i < left ? a.b_scale[n + i] : 0.0f;
                bias[i] = a.g.bias && i < left ? a.g.bias[n + i] : 0.0f;
            }
        }
    }
};

// W neighbouring sums of row m, whose scale is s.
template <int ACT, bool PAST, typename T, int W>
__device__ __forceinline__ void finish8(const Gemm8Args &a, int m, int n, float s, const ColumnTerms<W> &c,
                                        const int32_t (&sum)[W])
{
    float z[W];
#pragma unroll
    for (int i = 0; i < W; i++) z[i] = fmaf((float)sum[i] * s, c.scale[i], c.bias[i]);
    finish_scaled<ACT, PAST, T>(a.g, m, n, a.g.n - n, z);
}

// Tiles of TM x TN outputs, two LDS tiles of kStep8 k, WM x WN waves.  The
// steps go as in the products of 16 bits: a step's two halves of fragments
// alternate in registers, the waves meet once a step, and at the meeting the
// next step's LDS tile has arrived.  A half's LDS reads (and the next tile's
// loads) are spread over its multiplies: left to itself the compiler puts them
// last, and the waves wait for them (6 % of 16384 x 4096 to 4096).
//
// WIDE: tiles of 256 x 256 and waves of 128 x 64, one workgroup per CU, for
// products that fill the chip with them.  What bounds the tiles is LDS: a step
// reads and writes 96 KB for 128 x 128 outputs and 256 KB for 256 x 256, four times
// as many (at 128 bytes a clock 2048 clocks, as long as the multiplies take).
// Their sums leave from the registers, a lane's eight neighbours at a time, PAST
// the caches where rows are whole lines, and the operands stay there (16384 x 4096 to
// 4096 with SiLU 222 us, 233 through the caches); those of 128 x 128 tiles pass
// through LDS, so that rows leave as whole lines (straight from registers 409,600 x
// 512 to 256 took 6 % longer in such tiles).
//
// Measured (one MI355X, bf16 out, other data from call to call): 16384 x 4096 to 4096
// with SiLU 222 us (2.5 POP/s), with a residual, whose 134 MB arrive while nothing is
// multiplied, 262; 7744 x 1024 to 4096 with GELU 50; 409,600 x 512 to 256 in f16 121
// to 131; in 128 x 128 tiles 7744 x 4096 to 1024 38, 2048^3 18 us.
template <bool WIDE, bool PAST, bool DIRECT, typename T, int ACT>
__global__ __launch_bounds__(WIDE ? 512 : 256, 2) void k_gemm8(Gemm8Args args)
{
    static_assert((DIRECT || !WIDE) && (WIDE || !PAST), "");
    constexpr int TM = WIDE ? 256 : 128, TN = TM, WM = 2, WN = WIDE ? 4 : 2, kThreads = WM * WN * 64;
    using A = ByteOperand<TM, kThreads, DIRECT>;
    using B = ByteOperand<TN, kThreads, DIRECT, WIDE>;
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
        for (int i = 0; i < FM; i++) fa[half][i] = A::read(la, wm, i, half);
#pragma unroll
        for (int j = 0; j < FN; j++) fb[half][j] = B::read(lb, wn, j, half);
    };
    auto multiply = [&](int half) {
#pragma unroll
        for (int i = 0; i < FM; i++)
#pragma unroll
            for (int j = 0; j < FN; j++) acc[i][j] = mma8(fb[half][j], fa[half][i], acc[i][j]);
    };
    // one LDS read before every two multiplies, and one load where there are some
    auto spread = [&](auto loads) __attribute__((always_inline)) {
        if constexpr (WIDE)
#pragma unroll
            for (int u = 0; u < FM + FN; u++) {
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
                if (u < decltype(loads)::value) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
            }
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
        spread(std::integral_constant<int, 0>{});
        __builtin_amdgcn_sched_barrier(0);
        commit(t + 1);
        wait_for_lds<true>();
        meet();
        __builtin_amdgcn_sched_barrier(0);
        fetch(std::false_type{}, t + 2);
        read(t + 1, 0);
        multiply(1);
        spread(std::integral_constant<int, A::kLoads + B::kLoads>{});
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
    if constexpr (WIDE) {       // (never split)
        const int row = lane & 15, group = lane >> 4;
        float s[FM];
#pragma unroll
        for (int i = 0; i < FM; i++) {
            const int m = m0 + wm + 16 * i + row;
            s[i] = args.a_scale[m < g.m ? m : g.m - 1];
        }
        if (m0 + TM <= g.m && n0 + TN <= g.n) {
            // A whole tile: both halves of a line follow one another, and the
            // residual's loads of two rows are in flight together (the halves apart
            // cost 16384 x 4096 to 4096 5 %, one load at a time 12 %).
            static_assert(FN == 4 || !WIDE, "");
            constexpr int kBatch = 2;
            const T *res = static_cast<const T *>(g.residual) + (m0 + wm + row) * g.ldr + n0 + wn + 8 * group;
            T *out = static_cast<T *>(g.out) + (m0 + wm + row) * g.ldo + n0 + wn + 8 * group;
            T *pre = static_cast<T *>(g.preact) + (m0 + wm + row) * g.ldp + n0 + wn + 8 * group;
            const ColumnTerms<8> c[2] = {ColumnTerms<8>(args, n0 + wn + 8 * group, 8),
                                         ColumnTerms<8>(args, n0 + wn + 32 + 8 * group, 8)};
#pragma unroll
            for (int i0 = 0; i0 < FM; i0 += kBatch) {
                Vec<T, 8> r[kBatch][2];
                if (g.residual)
#pragma unroll
                    for (int i = 0; i < kBatch; i++)
#pragma unroll
                        for (int p = 0; p < 2; p++) r[i][p] = load_vec<T, 8>(res + 16 * (i0 + i) * g.ldr + 32 * p);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < kBatch; i++)
#pragma unroll
                    for (int p = 0; p < 2; p++) {
                        Vec<T, 8> o;
                        float z[8];
#pragma unroll
                        for (int v = 0; v < 8; v++) {
                            z[v] = fmaf((float)acc[i0 + i][2 * p + v / 4][v % 4] * s[i0 + i], c[p].scale[v], c[p].bias[v]);
                            const float y = activate<ACT>(z[v]);
                            o.v[v] = (T)(g.residual ? y + (float)r[i][p].v[v] : y);
                        }
                        store_words<PAST>(out + 16 * (i0 + i) * g.ldo + 32 * p, o);
                        if (g.preact) {
#pragma unroll
                            for (int v = 0; v < 8; v++) o.v[v] = (T)z[v];
                            store_words<PAST>(pre + 16 * (i0 + i) * g.ldp + 32 * p, o);
                        }
                    }
                __builtin_amdgcn_sched_barrier(0);
            }
            return;
        }
#pragma unroll
        for (int p = 0; p < FN / 2; p++) {
            const int n = n0 + wn + 32 * p + 8 * group;
            if (n >= g.n) continue;
            const ColumnTerms<8> c(args, n, g.n - n);
#pragma unroll
            for (int i = 0; i < FM; i++) {
                const int m = m0 + wm + 16 * i + row;
                const i32x4 v0 = acc[i][2 * p], v1 = acc[i][2 * p + 1];
                const int32_t v[8] = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
                if (m < g.m) finish8<ACT, PAST, T>(args, m, n, s[i], c, v);
            }
        }
        return;
    }
    // no load is in flight, and every wave has read its last fragments: the sums
    // pass through LDS
    typedef __attribute__((address_space(3))) i32x4 lds_quad;
    auto place = [&](int m, int n) { return (lds_quad *)(lds + (m * (TN / 4) + ((n >> 2) ^ (m & 15))) * 16); };
    static_assert(WIDE || TM * TN * 4 <= 2 * kStage, "");
    const int64_t ldpart = (g.n + 3) / 4 * 4;
#pragma unroll
    for (int i = 0; i < FM; i++)
#pragma unroll
        for (int j = 0; j < FN; j++) *place(wm + 16 * i + (lane & 15), wn + 16 * j + 4 * (lane >> 4)) = acc[i][j];
    __syncthreads();
    for (int q = threadIdx.x; q < TM * TN / 8; q += kThreads) {
        const int r = q / (TN / 8), c = q % (TN / 8) * 8, m = m0 + r, n = n0 + c;
        if (m >= g.m || n >= g.n) continue;
        const i32x4 v0 = *place(r, c), v1 = *place(r, c + 4);
        if (g.splits > 1) {
            int32_t *to = reinterpret_cast<int32_t *>(g.part) + ((int64_t)split * g.m + m) * ldpart + n;
            *reinterpret_cast<i32x4 *>(to) = v0;
            if (n + 4 < g.n) *reinterpret_cast<i32x4 *>(to + 4) = v1;
        } else {
            const int32_t v[8] = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
            finish8<ACT, false, T>(args, m, n, args.a_scale[m], ColumnTerms<8>(args, n, g.n - n), v);
        }
    }
}

// Narrow products (a map's projection to its embedding), whose B fits into LDS
// whole, as those of 16 bits: B is laid out once per workgroup, strips of 64 rows
// of A stream past it, each read once, in whole lines, with the next strip's loads
// in flight.  Bound by memory: 409,600 x 256 to 64 in f16 38 us (4.1 TB/s; in tiles
// 72).  On the same rows again and again, which the last cache holds in part, 30 with
// four workgroups per CU; three 33, strips of 128 rows 33 to 36 (a round of them more
// or less is then a sixth of the work).
constexpr int kStrip8 = 64;
constexpr int narrow8_bytes(int n, int ks) { return ((n + 31) / 32 * 32 + kStrip8) * ks * 64; }

// FULL: k fills the fragments.  Otherwise a row's last chunk is its last 16
// bytes, those that the chunk before has too masked to 0, and chunks beyond it
// are 0.
template <int KS, bool FULL, typename T, int ACT>
__global__ __launch_bounds__(256, KS < 8 ? 4 : 2) void k_gemm8_narrow(Gemm8Args args)
{
    extern __shared__ __align__(1024) unsigned char gemm8_lds[];
    const GemmArgs &g = args.g;
    constexpr int kRow = KS * 4;        // chunks in a row of A or B
    constexpr int kRows = kStrip8, kLoads = kRows * kRow / 256, kStep = 256 / kRow;
    lds_byte *strip_lds = (lds_byte *)gemm8_lds, *lds = strip_lds + kRows * KS * 64;
    const int pairs = (g.n + 31) / 32, n_pad = pairs * 32;
    // the first byte of chunk c, and how many of its bytes are not its own
    auto start = [&](int c) { return FULL || c * 16 <= g.k - 16 ? c * 16 : g.k - 16; };
    auto extra = [&](int c) { return c * 16 - start(c); };
    auto masked = [&](Bytes16 f, int skip) {
        if constexpr (!FULL)
#pragma unroll
            for (int d = 0; d < 4; d++) {
                const int gone = skip - 4 * d;
                f.u[d] &= gone <= 0 ? 0xffffffffu : gone >= 4 ? 0u : 0xffffffffu << (8 * gone);
            }
        return f;
    };
    for (int q = threadIdx.x; q < n_pad * kRow; q += 256) {
        const int n = q / kRow, c = q % kRow;
        Bytes16 f;
        f.u = u32x4{0, 0, 0, 0};
        if (n < g.n) {
            const Vec<int8_t, 16> v = load_vec<int8_t, 16>(static_cast<const int8_t *>(g.b) + (int64_t)n * g.ldb + start(c));
            __builtin_memcpy(&f, &v, 16);
            f = masked(f, extra(c));
        }
        *(__attribute__((address_space(3))) u32x4 *)(lds + (n * kRow + (c ^ narrow_swizzle(n))) * 16) = f.u;
    }
    const int lane = threadIdx.x & 63, j = lane & 15, c = lane >> 4;
    const int row0 = (wave_base() >> 6) * 16;       // this wave's rows of a strip
    const int strips = (int)(((int64_t)g.m + kRows - 1) / kRows);
    const int my_chunk = threadIdx.x % kRow, my_row = threadIdx.x / kRow;
    const int my_start = start(my_chunk), my_extra = extra(my_chunk);
    Vec<int8_t, 16> next[kLoads];
    auto fetch = [&](int strip) {
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const int m = strip * kRows + my_row + i * kStep;       // (rows beyond the last repeat it)
            next[i] = load_vec<int8_t, 16>(static_cast<const int8_t *>(g.a) + (m < g.m ? m : g.m - 1) * g.lda + my_start);
        }
    };
    int strip = blockIdx.x;
    if (strip < strips) fetch(strip);
    const int row = 8 * (j >> 2) + (j & 3);
    for (; strip < strips; strip += gridDim.x) {
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const int r = my_row + i * kStep;
            Bytes16 f;
            __builtin_memcpy(&f, &next[i], 16);
            f = masked(f, my_extra);
            *(__attribute__((address_space(3))) u32x4 *)(strip_lds + (r * kRow + (my_chunk ^ (r & 7))) * 16) = f.u;
        }
        const int m = strip * kRows + row0 + j;
        const float s = args.a_scale[m < g.m ? m : g.m - 1];
        wait_for_lds<false>();
        meet();
        if (strip + (int)gridDim.x < strips) fetch(strip + gridDim.x);
        Bytes16 fa[KS];
#pragma unroll
        for (int k = 0; k < KS; k++) {
            const int r = row0 + j;
            fa[k].u = *(const __attribute__((address_space(3))) u32x4 *)(
                strip_lds + (r * kRow + ((4 * k + c) ^ (r & 7))) * 16);
        }
        wait_for_lds<false>();
        meet();
        for (int p = 0; p < pairs; p++) {
            i32x4 acc[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
            for (int k = 0; k < KS; k++)
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    const int n = 32 * p + row + 4 * h;
                    Bytes16 fb;
                    fb.u = *(const __attribute__((address_space(3))) u32x4 *)(
                        lds + (n * kRow + ((4 * k + c) ^ narrow_swizzle(n))) * 16);
                    acc[h] = mma8(fb, fa[k], acc[h]);
                }
            const int n = 32 * p + 8 * c;
            if (n >= g.n || m >= g.m) continue;
            const int32_t v[8] = {acc[0][0], acc[0][1], acc[0][2], acc[0][3], acc[1][0], acc[1][1], acc[1][2], acc[1][3]};
            finish8<ACT, false, T>(args, m, n, s, ColumnTerms<8>(args, n, g.n - n), v);
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
    const int n = (int)(q - (int64_t)m * quads) * 4;
    finish8<ACT, false, T>(a, m, n, a.a_scale[m], ColumnTerms<4>(a, n, a.g.n - n), w);
}

// Few rows: 16 n per workgroup, its waves dividing k; fragments come straight
// from memory, since no other workgroup shares the weights and the rows stay in
// the caches.  One row of 1024 to 4096 3.9 us: a launch, two rounds of loads, the
// join of eight waves.
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
        if (m < g.m && n4 < g.n) finish8<ACT, false, T>(a, m, n4, a.a_scale[m], ColumnTerms<4>(a, n4, g.n - n4), sum);
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

// Rounds of tiles that the chip goes through: a round of wide ones (256 at
// once) takes 1.15 to 1.7 times as long as one of the others (512 at once):
// 7744 x 4096 to 1024 42 against 37 us, a round each; 4096^3 57 against 71, one
// against two; 7744 x 1024 to 4096 40 against 51, two against four; 409,600 x 512 to
// 256 in f16 121 against 170, seven against thirteen.
inline bool wide8_pays(const GemmArgs &g)
{
    const int64_t wide = ceil_div(ceil_div(g.m, 256) * ceil_div(g.n, 256), 256);
    const int64_t others = ceil_div(ceil_div(g.m, 128) * ceil_div(g.n, 128), 512);
    return 10 * others > 17 * wide;
}

// Whether rows of T are whole cache lines, so that wide tiles store past the
// caches: halves of lines cost more there where they are not (38,884 x 1088 to 1264
// with the value before the activation 155 us, 113 through the caches; to 1280 91
// and 103, without that value 68 and 77), and in binary32 (169, 131).
template <typename T>
bool whole_lines8(const void *p, int64_t ld)
{
    return !p || (aligned_to(p, 128) && ld * (int64_t)sizeof(T) % 128 == 0);
}

template <typename T, int ACT>
hipError_t launch_tiles8(Gemm8Args a, hipStream_t stream)
{
    const bool direct = direct8_ok(a.g), wide = direct && wide8_pays(a.g);
    const int tile = wide ? 256 : 128;
    a.g.tiles_m = (int32_t)ceil_div(a.g.m, tile);
    a.g.tiles_n = (int32_t)ceil_div(a.g.n, tile);
    a.g.splits = 1;
    a.g.k_split = a.g.k;
    if (!wide) choose_splits8(a.g);
    const dim3 grid(a.g.tiles_m * a.g.tiles_n * a.g.splits);
    const int lds = 4 * tile * kStep8;
    constexpr bool kPast = sizeof(T) == 2;
    if (wide && kPast && whole_lines8<T>(a.g.out, a.g.ldo) && whole_lines8<T>(a.g.preact, a.g.ldp))
        hipLaunchKernelGGL((k_gemm8<true, kPast, true, T, ACT>), grid, dim3(512), lds, stream, a);
    else if (wide)
        hipLaunchKernelGGL((k_gemm8<true, false, true, T, ACT>), grid, dim3(512), lds, stream, a);
    else if (direct)
        hipLaunchKernelGGL((k_gemm8<false, false, true, T, ACT>), grid, dim3(256), lds, stream, a);
    else
        hipLaunchKernelGGL((k_gemm8<false, false, false, T, ACT>), grid, dim3(256), lds, stream, a);
    if (hipError_t e = hipGetLastError(); e != hipSuccess || a.g.splits == 1) return e;
    const int64_t quads = (int64_t)a.g.m * ((a.g.n + 3) / 4);
    hipLaunchKernelGGL((k_gemm8_join<T, ACT>), dim3((unsigned)ceil_div(quads, 256)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

// Fragments of k that hold a row (2, 4 or 8), 0 where it is too long.
inline int narrow8_steps(int k) { return k <= 128 ? 2 : k <= 256 ? 4 : k <= 512 ? 8 : 0; }
// Where two workgroups or more fit a CU: 409,600 x 512 to 96 in f16 74 us (in tiles
// 95), to 128, of which one fits, 124 (100).
inline bool narrow8_fits(const GemmArgs &g)
{
    const int ks = narrow8_steps(g.k);
    return g.k >= 16 && ks > 0 && g.n <= 128 && 2 * narrow8_bytes(g.n, ks) <= 160 << 10;
}

template <typename T, int ACT>
hipError_t launch_narrow8(const Gemm8Args &a, hipStream_t stream)
{
    const int ks = narrow8_steps(a.g.k), bytes = narrow8_bytes(a.g.n, ks), by_lds = (160 << 10) / bytes;
    const int64_t strips = ceil_div(a.g.m, kStrip8), most = 256 * (by_lds < 4 ? by_lds : 4);
    const dim3 grid((unsigned)(strips < most ? strips : most));
    auto launch = [&](auto steps) {
        constexpr int KS = decltype(steps)::value;
        if (a.g.k == KS * 64)
            hipLaunchKernelGGL((k_gemm8_narrow<KS, true, T, ACT>), grid, dim3(256), bytes, stream, a);
        else
            hipLaunchKernelGGL((k_gemm8_narrow<KS, false, T, ACT>), grid, dim3(256), bytes, stream, a);
    };
    switch (ks) {
    case 2: launch(std::integral_constant<int, 2>{}); break;
    case 4: launch(std::integral_constant<int, 4>{}); break;
    default: launch(std::integral_constant<int, 8>{}); break;
    }
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
    if (narrow8_fits(a.g)) return launch_narrow8<T, ACT>(a, stream);
    return launch_tiles8<T, ACT>(a, stream);
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
