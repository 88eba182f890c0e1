// Fully-connected layers in 4 bits with group scales, and 8-bit activation checkpoints: what the
// translation units share.
//
// Packed codes.  W is cut into tiles of 16 rows by 128 columns of 1 KB, row tiles outermost:
// [ceil(n/16)][ceil(k/128)][16 rows][64 bytes].  In a row's 64 bytes, dword 4 q + i holds columns
// 32 i + 8 q + 0..7, and in a dword nibble (j & 1) * 4 + j / 2 holds column j of its eight.  So
//   * a wave that loads 16 bytes a lane (lane = row + 16 q ... in the matrix instruction's own order)
//     reads one contiguous kilobyte, and dword i of lane (row, q) is exactly that lane's operand of
//     the i-th 16x16x32 matrix instruction of the tile: columns 8 q .. 8 q + 7 of 32-column block i;
//   * nibbles r and r + 4 are the neighbours 2 r and 2 r + 1, so one shift and one mask leave a pair
//     of neighbouring columns in the two halves of a register, where 16-bit values are wanted.
// Rows and columns past the matrix hold code 0 and are never used with a non-zero factor.
#pragma once

#include "kq_internal.h"

namespace kq {

constexpr int kTileRows = 16;
constexpr int kTileCols = 128;
constexpr int kTileBytes = kTileRows * kTileCols / 2;
constexpr int kCkGroup = KQ_CHECKPOINT_GROUP;

inline __host__ __device__ int ceil_div(int a, int b) { return (a + b - 1) / b; }
inline __host__ __device__ int64_t ceil_div64(int64_t a, int64_t b) { return (a + b - 1) / b; }

using f32x4 = __attribute__((ext_vector_type(4))) float;
using f32x2 = __attribute__((ext_vector_type(2))) float;
using bf16x8 = __attribute__((ext_vector_type(8))) __bf16;
using bf16x2 = __attribute__((ext_vector_type(2))) __bf16;
using f16x8 = __attribute__((ext_vector_type(8))) _Float16;
using f16x2 = __attribute__((ext_vector_type(2))) _Float16;
using u32x4 = __attribute__((ext_vector_type(4))) unsigned;
using u32x2 = __attribute__((ext_vector_type(2))) unsigned;

__device__ __forceinline__ float bf16_bits_to_f32(unsigned h) { return __builtin_bit_cast(float, h << 16); }

// A checkpoint group's step from its exponent; 0 gives 0, and 255 NaN.
__device__ __forceinline__ float checkpoint_step(unsigned e) {
    return __builtin_bit_cast(float, e == 255u ? 0x7fc00000u : e << 23);
}

// The two 16-bit activation types.
template <bool BF>
struct Act {
    static __device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
        if constexpr (BF)
            return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
        else
            return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
    // two fp32 values rounded to nearest into the halves of a register
    static __device__ __forceinline__ unsigned pack(float lo, float hi) {
        const f32x2 v = {lo, hi};
        if constexpr (BF) return __builtin_bit_cast(unsigned, __builtin_convertvector(v, bf16x2));
        else return __builtin_bit_cast(unsigned, __builtin_convertvector(v, f16x2));
    }
    // the same for values that bf16 holds exactly (to fp16 they are rounded, beyond its range to infinity)
    static __device__ __forceinline__ unsigned pack_bf16_value(float lo, float hi) {
        if constexpr (BF)
            return __builtin_amdgcn_perm(__builtin_bit_cast(unsigned, hi), __builtin_bit_cast(unsigned, lo), 0x07060302u);
        else
            return pack(lo, hi);
    }
    static __device__ __forceinline__ float lo(unsigned v) {
        if constexpr (BF) return __builtin_bit_cast(float, v << 16);
        else return (float)__builtin_bit_cast(f16x2, v).x;
    }
    static __device__ __forceinline__ float hi(unsigned v) {
        if constexpr (BF) return __builtin_bit_cast(float, v & 0xffff0000u);
        else return (float)__builtin_bit_cast(f16x2, v).y;
    }
    static __device__ __forceinline__ unsigned short one(float v) { return (unsigned short)(pack(v, 0.0f) & 0xffffu); }
};

// 16 levels as two byte tables of 16 entries in registers; a look-up is four byte permutes.
// In fp16 they are levels 2^shift, with the largest in [2^14, 2^15): every bf16 level down to 2^-31 of it is exact
// and what lies below is off by at most 2^-39 of it (fp16's subnormals), whatever the table's own range is.
struct LevelTable {
    unsigned lo[4], hi[4];  // low and high bytes of the 16-bit levels, four a register
    int shift;
};

template <bool BF>
__device__ __forceinline__ LevelTable load_levels(const uint16_t* levels) {
    LevelTable t;
    t.shift = 0;
    if constexpr (!BF) {
        unsigned top = 1u << 7;  // (at least the smallest normal number)
#pragma unroll
        for (int j = 0; j < 16; ++j) top = max(top, (unsigned)levels[j] & 0x7fffu);
        t.shift = 14 + 127 - (int)(top >> 7);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        unsigned a, b;  // levels 4 r .. 4 r + 3 in two registers
        if constexpr (BF) {
            a = (unsigned)levels[4 * r] | (unsigned)levels[4 * r + 1] << 16;
            b = (unsigned)levels[4 * r + 2] | (unsigned)levels[4 * r + 3] << 16;
        } else {
            auto level = [&](int j) { return __builtin_ldexpf(bf16_bits_to_f32(levels[j]), t.shift); };
            a = Act<false>::pack(level(4 * r), level(4 * r + 1));
            b = Act<false>::pack(level(4 * r + 2), level(4 * r + 3));
        }
        t.lo[r] = __builtin_amdgcn_perm(b, a, 0x06040200u);
        t.hi[r] = __builtin_amdgcn_perm(b, a, 0x07050301u);
    }
    return t;
}

// the bytes of a 16-entry table at four indices (0..15, one a byte)
__device__ __forceinline__ unsigned look_up(const unsigned (&t)[4], unsigned low3, unsigned pick) {
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(t[3], t[2], low3), __builtin_amdgcn_perm(t[1], t[0], low3), pick);
}

// Memory of the two kinds as the direct load to LDS takes it.
using lds_ptr = __attribute__((address_space(3))) void*;
using global_ptr = const __attribute__((address_space(1))) void*;

// Workgroups are dealt to the eight XCDs in turn; tile numbers are dealt so that an XCD's workgroups take
// neighbouring tiles (their operands meet in its L2).  A bijection for any count.
__device__ __forceinline__ int xcd_tile(int b, int count) {
    const int per = count >> 3, rest = count & 7, x = b & 7;
    return x * per + min(x, rest) + (b >> 3);
}

// ---- device parameters and launchers (checked by the C entry points before) ------------------------

struct GroupWeights {
    const uint8_t* codes;
    const uint16_t* scales;  // bf16 [n][groups]
    const uint16_t* levels;  // bf16 [16], or NULL: -8 .. 7
    int n, k;
    int log_group;           // 5, 6 or 7
    int groups;              // ceil(k / group)
    int ktiles;              // ceil(k / 128)
    int ntiles;              // ceil(n / 16)
};

struct QuantizeParams {
    const void* W;
    int64_t ldw;
    int type;
    int n, k, log_group, groups, ktiles;
    const uint16_t* levels;
    uint8_t* codes;
    uint16_t* scales;
};
hipError_t launch_quantize_groups(const QuantizeParams& p, hipStream_t s);

struct ReconstructGroupsParams {
    GroupWeights w;
    int type;
    void* W_hat;
    int64_t ldw;
};
hipError_t launch_reconstruct_groups(const ReconstructGroupsParams& p, hipStream_t s);

struct CheckpointParams {
    void* X;       // read by pack, written by restore
    int64_t ldx;
    int type;
    int64_t m;
    int k, kq;     // kq = k rounded up to the group: the pitch of q
    int8_t* q;
    uint8_t* exps;
};
hipError_t launch_checkpoint_pack(const CheckpointParams& p, hipStream_t s);
hipError_t launch_checkpoint_restore(const CheckpointParams& p, hipStream_t s);

// The products.  `i` is the contiguous dimension of the output, `j` its rows, `c` the contraction:
//   linear      Y[m][n]  = sum_k X[m][k] W[n][k]     i = n, j = m, c = k
//   grad input  dX[m][k] = sum_n dY[m][n] W[n][k]    i = k, j = m, c = n
//   grad weight dW[n][k] = sum_m dY[m][n] X^[m][k]   i = k, j = n, c = m   (scales: reduced in the epilogue)
enum class Product { Linear = 0, GradInput = 1, GradWeight = 2, GradScales = 3 };

struct GemmParams {
    GroupWeights w;          // Linear, GradInput, GradScales (codes and levels only)
    const void* B;           // X (Linear) or dY; in the kernel [J][C] in aligned rows
    int64_t ldb;
    const int8_t* q;         // the checkpoint: GradWeight, GradScales
    const uint8_t* exps;
    int kq;
    int64_t I, J, C;         // sizes along i, j, c
    const float* bias;
    void* out;               // 16-bit (Linear, GradInput) or fp32
    int64_t ldo;
    float* dbias;            // column sums of dY, or NULL: from bias_parts partial ones [bias_parts][J]
    float* bias_part;
    int bias_parts;
    float* part;             // partial sums of a split contraction, or NULL
    int splits;
    int steps_per_split;     // 64-deep steps of the contraction a workgroup takes
    int itiles, jtiles;
};
struct GemmPlan {
    int bi, bj;              // output tile
    int splits, steps_per_split;
    bool stage_b;            // B is transposed or copied into the workspace, rows of `pitch` values
    int64_t pitch;
    int bias_parts;
    size_t part_bytes, b_bytes, ws_bytes;  // workspace: partial sums, B, partial column sums
};
// B and ldb: X or dY as the call gets it (only its alignment counts; the gradients from a checkpoint take any)
GemmPlan gemm_plan(Product mode, const void* B, int64_t ldb, int64_t I, int64_t J, int64_t C, int groups);
hipError_t launch_gemm(Product mode, bool bf16, const GemmPlan& plan, GemmParams p, void* ws, hipStream_t s);

struct StageBParams {
    const void* in;
    int64_t ld;
    int64_t J, C;
    void* out;
    int64_t pitch;
    float* bias_part;
};

// out[r][c] = sum over the splits of part[split][r][c], in order, + bias[c]
struct JoinParams {
    const float* part;
    int splits;
    int64_t rows, cols;
    const float* bias;
    void* out;
    int64_t ldo;
    int type;
};
hipError_t launch_join(const JoinParams& p, hipStream_t s);

// Y = X W^T for at most kMatvecRows rows of X.
constexpr int kMatvecRows = 16;
constexpr int kMatvecLdsRows = 4;         // up to so many rows of X go through LDS
constexpr int kMatvecLdsBytes = 65536;
struct MatvecParams {
    GroupWeights w;
    const void* X;
    int64_t ldx;
    int m;
    const float* bias;
    void* Y;
    int64_t ldy;
    float* part;             // partial sums [splits][m][n], or NULL
    int splits, blocks_per_split;  // 128-column blocks a workgroup takes
    int chunk;
};
struct MatvecPlan {
    int row_tiles, waves, splits, blocks_per_split;
    size_t ws_bytes;
};
MatvecPlan matvec_plan(int m, int64_t n, int64_t k);
hipError_t launch_matvec(bool bf16, const MatvecPlan& plan, MatvecParams p, hipStream_t s);

}  // namespace kq
