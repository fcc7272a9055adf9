// Launchers of the row operators (linear.hip, residual_norm.hip), called by rows_api.hip after its checks.
#pragma once
#include "rows.h"

// A first operand in two parts (`a_lo` is there): HIGH_PART x = a + a_lo / LOW_PART.  fp16 so holds x, an fp32 value, to 22 bits: no |x| up
// to 1.13 times its largest overflows, and what is below its normal values keeps its digits in the low part.  bf16, which has fp32's range, holds
// 16 bits, and no low part or sum of them is infinite where the high ones are not.
template <class T> constexpr float HIGH_PART = 1.f;
template <class T> constexpr float LOW_PART = 1.f;
template <> inline constexpr float HIGH_PART<_Float16> = 0.5f;
template <> inline constexpr float LOW_PART<_Float16> = 2048.f;

// C[m][n] = sum over k < K of A(m, k) B(n, k).  An operand is stored with its k contiguous ([m][k], `lda` elements from row to
// row) or with its rows contiguous ([k][m]); which of the two is part of the kernel chosen.
struct ProductArgs {
    corr_dtype type;
    const void* a; const void* b;
    const void* a_lo;          // laid out as a; null but for 16-bit types whose second operand has its rows contiguous
    int64_t lda, ldb;
    int a_rows, b_rows;        // 1: rows contiguous ([k][m] / [k][n])
    int M, N, K;
    int gated;                 // 1: b has 2 N rows, y = act(first N) * (second N); bias, pre and part have 2 N columns, no residual
    // epilogue: z = C + bias (to `pre`, if there), y = act(z) + res
    const float* bias;
    const void* res; int64_t ld_res;
    void* pre;                 // [M][N]
    void* y; int64_t ldy;
    int act;
    bool past;                 // set by launch_product: y and pre are stored past the caches
    float* part;               // [splits][M][N] fp32, where the plan says more than one split
};
struct ProductPlan { int tile, splits, steps; };   // steps of the k loop per split
ProductPlan product_plan(corr_dtype type, int a_rows, int b_rows, int M, int N, int K);
void product_tile(const ProductPlan& p, int& rows, int& cols);   // no rows: few rows, without tiles
void gated_tile(corr_dtype type, int M, int N, int K, int& rows, int& cols, int& splits);      // of both halves' columns; 128 x 64: rows with a short k
static inline size_t product_part_bytes(const ProductPlan& p, int M, int N) {
    return p.splits > 1 ? (size_t)p.splits * M * N * 4 : 0;
}
hipError_t launch_product(const ProductArgs& p, hipStream_t s);
// dst[r][0 .. ld_dst) = src[r][0 .. cols), zeros behind (16-bit elements, ld_dst a multiple of eight); no rows: nothing to do
struct Pack16 { const void* src; int64_t ld_src; void* dst; int64_t ld_dst, rows, cols; };
hipError_t launch_pack16(const Pack16& one, const Pack16& two, hipStream_t s);
// dz = dy * act'(z) as `type` (dz may be null; in two parts if dz_lo is there), and the column sums of the unrounded dz by parts (part may be null)
int slope_parts(int64_t M);
hipError_t launch_slope(corr_dtype t, int act, const void* dy, int64_t ld_dy, const void* z, void* dz, void* dz_lo, int64_t ld_dz,
                        float* part, int64_t M, int N, hipStream_t s);

// gated: z is [M][2 N], dz and part have 2 N columns
hipError_t launch_slope_gated(corr_dtype t, int act, const void* dy, int64_t ld_dy, const void* z, void* dz, void* dz_lo, int64_t ld_dz,
                              float* part, int64_t M, int N, hipStream_t s);

// ---- norms around a block (residual_norm.hip)
struct NormArgs {
    corr_residual_norm_args a;
    void* h_out; void* n_out;
    const void* d_h_out; const void* d_n_out;      // gradient: either may be null (zero)
    void* d_h; void* d_y; void* d_gate;            // each may be null
    float* part;                                   // [parts][5][cols]: scale, post weight, post bias, pre weight, pre bias
    int parts;
};
int norm_backward_parts(int64_t rows, int64_t cols, bool full);
// one instantiation of residual_norm.hip per pair of stream and row types
#define NORM_PAIRS(X) X(F32, F32, f32_f32) X(F32, BF16, f32_bf16) X(F32, F16, f32_f16) X(BF16, BF16, bf16_bf16) X(F16, F16, f16_f16)
#define CORR_DECLARE_NORM(S, T, name)                                          \
    hipError_t launch_residual_norm_##name(const NormArgs& n, hipStream_t s);  \
    hipError_t launch_residual_norm_backward_##name(const NormArgs& n, hipStream_t s);
NORM_PAIRS(CORR_DECLARE_NORM)
#undef CORR_DECLARE_NORM
