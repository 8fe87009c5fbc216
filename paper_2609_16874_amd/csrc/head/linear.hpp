// linear.hpp -- arguments of the matrix product kernels (private to the library).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "cpe_head.h"

namespace cpe {

constexpr int kGemmThreads = 256;
constexpr int kTile = 128;                    // output rows and columns of a workgroup
constexpr int kSplitTiles = 512;              // partial tiles of a split product
constexpr int64_t kSplitBytes = (int64_t)kSplitTiles * kTile * kTile * 4;       // and their scratch
constexpr int step_k(size_t element) { return 128 / (int)element; }             // k of one LDS tile
constexpr int least_steps(size_t element) { return element == 4 ? 4 : 8; }      // of a split
constexpr int64_t kMaxTiles = (int64_t)1 << 22;
constexpr int kSumBlocks = 1024;              // workgroups along the rows of the bias gradient
constexpr int kStripRows = 64;                // rows that a workgroup of the one-pass gradient takes at a time
constexpr int kNarrowGradBlocks = 256;        // and its workgroups
constexpr int kSumUnroll = 4;                 // rows of a thread of the bias gradient in flight

// out[m][n] = act(sum_k A(m, k) B(n, k) + bias[n]) + residual[m][n].
// A(m, k) is a[m lda + k], or a[k lda + m] where a_cols is set; B alike.
struct GemmArgs {
    const void *a, *b;
    int64_t lda, ldb;
    int32_t m, n, k;
    bool a_cols, b_cols;
    void *out;
    int64_t ldo;
    const float *bias;                        // may be null
    const void *residual;                     // may be null
    int64_t ldr;
    void *preact;                             // may be null: the value before the activation
    int64_t ldp;
    int act;
    const float *row_scale;                   // may be null: out[m] /= the mantissa of row m's scale
    const float *b_scale;                     // not null: B is bytes across k, with a scale for each k
    bool fold;                                // of which A has the mantissas already
    float *part;                              // scratch of a split product: [splits][m][n rounded up to 4]
    int64_t part_bytes;
    int32_t splits, k_split;                  // splits > 1: each sums k_split of the k
    int32_t tiles_m, tiles_n;
};

// dz = dy act'(preact) (dz may be null) and column sums of it (sums may be null).
struct GradArgs {
    const void *dy, *preact;
    int64_t ldd, ldp, ldz;
    void *dz;
    const float *z_scale, *x_scale;           // not null: preact is bytes with these scales; dz is times x's mantissas
    float *part, *sums;                       // scratch [blocks][n]; out [n]
    int32_t rows, n, blocks, slab;            // workgroups along the rows, vectors of columns of each
    int act;
};

// A narrow or few-row product's whole gradient: dz = dy act'(preact), dx = dz w,
// dw = dz^T x, dbias = column sums of dz; those whose pointer is not null.
struct WholeGradArgs {
    const void *x, *w, *dy, *preact;
    int64_t ldx, ldw, ldd, ldp, lddx, lddw;
    void *dx, *dw;
    float *dbias;
    const float *x_scale, *z_scale;           // x_scale not null: x and preact are bytes with these scales
    float *part, *part_sums;                  // scratch: [blocks][n][k], [blocks][n]
    int32_t rows, n, k, blocks;
    int act;
};

// Whether a gradient from rows in 8 bits has the mantissas of x's scales in dz:
// where dz is rounded to 16 bits anyway, x then need not be.
constexpr bool folds(int act, size_t element) { return element == 2 && (act == CPE_ACT_SILU || act == CPE_ACT_GELU); }

hipError_t launch_gemm_f32(const GemmArgs &g, hipStream_t stream);
hipError_t launch_gemm_f16(const GemmArgs &g, hipStream_t stream);
hipError_t launch_gemm_bf16(const GemmArgs &g, hipStream_t stream);
hipError_t launch_grad_f32(const GradArgs &g, hipStream_t stream);
hipError_t launch_grad_f16(const GradArgs &g, hipStream_t stream);
hipError_t launch_grad_bf16(const GradArgs &g, hipStream_t stream);
// in one pass over the rows (16-bit types)
hipError_t launch_narrow_grad_f16(WholeGradArgs a, hipStream_t stream);
hipError_t launch_narrow_grad_bf16(WholeGradArgs a, hipStream_t stream);
// of few rows
hipError_t launch_rows_grad_f32(const WholeGradArgs &a, hipStream_t stream);
hipError_t launch_rows_grad_f16(const WholeGradArgs &a, hipStream_t stream);
hipError_t launch_rows_grad_bf16(const WholeGradArgs &a, hipStream_t stream);

}  // namespace cpe
