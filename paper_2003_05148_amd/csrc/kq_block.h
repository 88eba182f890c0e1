// Fully-connected layers in 8-bit floats (e4m3) with a power of two for each block of 128: what the translation
// units share.
//
// Every product is out[j][i] = sum_c A[i][c] B[j][c] of two operands held the same way (but for W^T): rows of e4m3 values along the
// contraction, their pitch a multiple of 128 bytes with zeros past the end, and one exponent byte for 128 of them.  So
// a kernel has no edges along the contraction, every row is aligned, and a block's exponent is one byte of the scaled
// matrix instruction (or one factor of a decoded operand).
//   linear       Y[m][n]   i = n, j = m, c = k   A = W (128 x 128 blocks), B = X
//   grad input   dX[m][k]  i = k, j = m, c = n   A = W^T (read as W lies, the same blocks), B = dY
//   grad weight  dW[n][k]  i = k, j = n, c = m   A = X^T, B = dY^T, both quantized along m
#pragma once

#include "kq_group.h"

namespace kq {

constexpr int kBlock = KQ_BLOCK;

inline __host__ __device__ int64_t block_pitch(int64_t k) { return (k + kBlock - 1) / kBlock * kBlock; }

// The biased exponent of a block from the bits of its largest magnitude (255: not finite).
__device__ __forceinline__ unsigned block_exponent(unsigned a) {
    if (a >= 0x7f800000u) return 255u;
    const int e = (int)(a >> 23) - 8 + ((a & 0x7fffffu) > 0x600000u ? 1 : 0);
    return (unsigned)(e < 1 ? 1 : e);
}
// 2^-e, for 1 <= biased <= 254
__device__ __forceinline__ float block_inverse(unsigned biased) { return __builtin_bit_cast(float, (254u - biased) << 23); }

// Four fp32 values times inv (exact: a power of two) to four bytes.  Their magnitude is at most 448 then.
__device__ __forceinline__ unsigned encode4(float a, float b, float c, float d, float inv) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, w, true);
}
constexpr unsigned kNaN4 = 0x7f7f7f7fu;

// Eight bytes times a power of two as bf16, which holds them exactly (but for magnitudes below 2^-126).
__device__ __forceinline__ u32x4 decode8(unsigned lo, unsigned hi, float scale) {
    return u32x4{__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false)),
                 __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true)),
                 __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false)),
                 __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true))};
}

// ---- device parameters and launchers (checked by the C entry points before) ------------------------

struct BlockQuantizeParams {
    const void* X;
    int64_t ldx;
    int type;
    int64_t m;
    int64_t k, kp;
    uint8_t* values;
    uint8_t* exps;
};
hipError_t launch_quantize_blocks(const BlockQuantizeParams& p, int rows, hipStream_t s);

struct BlockReconstructParams {
    const uint8_t* values;
    const uint8_t* exps;
    int64_t m, k, kp;
    int rows;
    void* X_hat;
    int64_t ldx;
    int type;
};
hipError_t launch_reconstruct_blocks(const BlockReconstructParams& p, hipStream_t s);

// out[c][r], r along the 128-row blocks of X, pitch rp (a multiple of 128, zeros past m): quantized along r (again, where X is
// bytes).
struct BlockTransposeParams {
    const void* X;        // [m][cols], or bytes of pitch ldx with in_exps [m][ldx / 128]
    int64_t ldx;
    int type;             // KQ_T_*
    const uint8_t* in_exps;
    int64_t m, cols, rp;
    uint8_t* values;      // [cols][rp]
    uint8_t* exps;        // [cols][rp / 128]
    float* sums;          // [rp / 128][cols]: sums over each 128 rows, or NULL
};
// X's values and dY, transposed and quantized along the rows
hipError_t launch_grad_weight_operands(const BlockTransposeParams& x, const BlockTransposeParams& dy, hipStream_t s);

struct BlockOperand {
    const uint8_t* v;
    int64_t pitch;
    const uint8_t* e;        // exponent of row r, block b: e[r * e_row + b * e_col], r / 128 for r in the 128 x 128 form
    int64_t e_row, e_col;
};
// How A lies: rows with an exponent for 128 x 128 of them, rows with their own, or columns A[i][c] at v[c * pitch + i] (128 x 128)
enum { kFormBlocks, kFormRows, kFormColumns };
struct BlockGemmParams {
    BlockOperand A, B;
    int64_t I, J;
    int64_t depth, a_cols;   // kFormColumns: rows c that there are, and columns of each (a multiple of 128)
    int steps;               // blocks of the contraction
    const float* bias;       // [I] or NULL
    void* out;
    int type;                // of out
    int64_t ldo;
    float* part;             // partial sums of a split contraction, or NULL
    int splits, steps_per_split;
    int itiles, jtiles;
    float* dbias;            // [J] or NULL: the sum of bias_parts rows of bias_part [bias_parts][J]
    const float* bias_part;
    int bias_parts;
};
struct BlockGemmPlan {
    int bi, bj;              // output tile
    int splits, steps_per_split;
    size_t part_bytes;
    int64_t rest_from;       // columns i from here on have a tile of their own, or 0
    int rest_bi, rest_bj;
    float us;                // as modelled
};
// exact: products on the 16-bit matrix instructions
BlockGemmPlan block_gemm_plan(bool exact, int64_t I, int64_t J, int64_t C);
hipError_t launch_block_gemm(bool exact, int form, const BlockGemmPlan& plan, BlockGemmParams p, void* part, hipStream_t s);

// Y = X W^T for few rows of X: up to kBlockMatvecRows always, up to kBlockMatvecMost where the plan is the faster one.
constexpr int kBlockMatvecRows = 16, kBlockMatvecMost = 1024;
struct BlockMatvecParams {
    const uint8_t* values;   // W
    const uint8_t* exps;
    int64_t n, k, kp;
    const void* X;           // of x_type; KQ_T_E4M3 with x_exps
    int x_type;
    int64_t ldx;
    const uint8_t* x_exps;
    int m;
    const float* bias;
    void* Y;
    int y_type;
    int64_t ldy;
    float* part;             // partial sums [splits][m][n], or NULL
    int splits, blocks_per_split;
};
struct BlockMatvecPlan {
    int row_tiles, waves, splits, blocks_per_split;
    size_t ws_bytes;
    float us;                // as modelled, above kBlockMatvecRows rows
};
BlockMatvecPlan block_matvec_plan(int m, int64_t n, int64_t k);              // up to kBlockMatvecRows rows
BlockMatvecPlan block_matvec_plan(int x_type, int m, int64_t n, int64_t k);  // more of them
hipError_t launch_block_matvec(const BlockMatvecPlan& plan, BlockMatvecParams p, hipStream_t s);

// What kq_block_linear of a size takes, and its workspace.
struct BlockLinearPlan {
    bool few;
    BlockMatvecPlan few_plan;
    BlockGemmPlan plan;
    size_t x, x_exps, total;  // X quantized, where it is not already
};
BlockLinearPlan block_linear_plan(int x_type, int y_type, int64_t m, int64_t n, int64_t k);

}  // namespace kq
