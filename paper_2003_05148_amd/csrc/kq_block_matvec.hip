// Y = X W^T for few rows of X (one token, a small batch): a stream of the weight's bytes past the matrix cores.
//
// A wave multiplies 16 rows of W by 16 rows of X, a block of 128 columns at a time.  Lane (row r = l % 16, q = l / 16)
// takes columns 16 q .. 16 q + 15 and 64 more of both, so a wave's two loads of W are 16 rows of 64 neighbouring bytes;
// the bytes become bf16 on the way to the 16 x 16 x 32 matrix instruction, which is exact, and a block's fp32 sum
// takes both exponents at once.  A row's block of X lies in four lanes: its largest magnitude is two exchanges away,
// so X is quantized where it is used.  The waves of a workgroup take the blocks of its rows in turn and add their
// sums through LDS in order.  Where there are few rows of W the columns are also split over workgroups, joined by a
// second kernel.
#include "kq_block.h"
#include "kq_values.h"

namespace kq {

// 16 columns at c0 of a row, zeros past k
template <int TYPE>
__device__ __forceinline__ void load16(const void* X, int64_t row_at, int c0, int k, float* v) {
    float a[8], b[8];
    load_columns<TYPE>(X, row_at, c0, k, a);
    load_columns<TYPE>(X, row_at, c0 + 8, k, b);
#pragma unroll
    for (int t = 0; t < 8; ++t) {
        v[t] = a[t];
        v[8 + t] = b[t];
    }
}

template <int TYPE, int WAVES, int RT>
__global__ __launch_bounds__(64 * WAVES) void block_matvec_kernel(const BlockMatvecParams p) {
    __shared__ f32x4 s_sum[RT * WAVES * 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r16 = lane & 15, q = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * RT * 16;
    const int blocks = (int)(p.kp >> 7);
    const int b_begin = blockIdx.y * p.blocks_per_split, b_end = min(b_begin + p.blocks_per_split, blocks);
    // rows past the last repeat it: what they give is not stored
    const uint8_t* w_row[RT];
    const uint8_t* w_exp[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        w_row[t] = p.values + min(n0 + 16 * t + r16, p.n - 1) * p.kp;
        w_exp[t] = p.exps + (min(n0 + 16 * t, p.n - 1) >> 7) * blocks;  // (16 rows lie in one block)
    }
    const int64_t xr = min(r16, p.m - 1);
    f32x4 y[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) y[t] = f32x4{0, 0, 0, 0};

    for (int b = b_begin + wave; b < b_end; b += WAVES) {
        u32x4 w[RT][2];
        unsigned ew[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            w[t][0] = *(const u32x4*)(w_row[t] + (int64_t)b * kBlock + 16 * q);
            w[t][1] = *(const u32x4*)(w_row[t] + (int64_t)b * kBlock + 64 + 16 * q);
            ew[t] = w_exp[t][b];
        }
        u32x4 x[2];
        unsigned ex;
        if constexpr (TYPE == KQ_T_E4M3) {
            const uint8_t* row = (const uint8_t*)p.X + xr * p.kp + (int64_t)b * kBlock;
            x[0] = *(const u32x4*)(row + 16 * q);
            x[1] = *(const u32x4*)(row + 64 + 16 * q);
            ex = p.x_exps[xr * blocks + b];
        } else {
            float v[2][16];
#pragma unroll
            for (int h = 0; h < 2; ++h) load16<TYPE>(p.X, xr * p.ldx, b * kBlock + 64 * h + 16 * q, (int)p.k, v[h]);
            unsigned a = 0;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int t = 0; t < 16; ++t) a = max(a, __builtin_bit_cast(unsigned, v[h][t]) & 0x7fffffffu);
            a = max(a, (unsigned)__shfl_xor(a, 16));
            a = max(a, (unsigned)__shfl_xor(a, 32));
            ex = block_exponent(a);
            const float inv = ex == 255u ? 0.0f : block_inverse(ex);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int t = 0; t < 4; ++t) x[h][t] = encode4(v[h][4 * t], v[h][4 * t + 1], v[h][4 * t + 2], v[h][4 * t + 3], inv);
        }
        u32x4 xd[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) xd[i] = decode8(x[i >> 1][2 * (i & 1)], x[i >> 1][2 * (i & 1) + 1], 1.0f);
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            f32x4 acc = {0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < 4; ++i) acc = Act<true>::mfma(decode8(w[t][i >> 1][2 * (i & 1)], w[t][i >> 1][2 * (i & 1) + 1], 1.0f), xd[i], acc);
            const int shift = (int)(ew[t] + ex) - 254;
            const float one = ew[t] == 255u || ex == 255u ? __builtin_bit_cast(float, 0x7fc00000u) : 1.0f;
#pragma unroll
            for (int r = 0; r < 4; ++r) y[t][r] = __builtin_fmaf(__builtin_ldexpf(acc[r], shift), one, y[t][r]);
        }
    }

    // lane holds Y[r16][n0 + 16 t + 4 q + r]: the waves' sums in order
#pragma unroll
    for (int t = 0; t < RT; ++t) s_sum[(t * WAVES + wave) * 64 + lane] = y[t];
    __syncthreads();
    if (wave < RT) {
        f32x4 v = s_sum[wave * WAVES * 64 + lane];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v += s_sum[(wave * WAVES + w) * 64 + lane];
        if (r16 < p.m) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int64_t n = n0 + 16 * wave + 4 * q + r;
                if (n >= p.n) break;
                if (p.part) {
                    p.part[((int64_t)blockIdx.y * p.m + r16) * p.n + n] = v[r];
                    continue;
                }
                const float o = v[r] + (p.bias ? p.bias[n] : 0.0f);
                const int64_t at = (int64_t)r16 * p.ldy + n;
                if (p.y_type == KQ_T_F32) ((float*)p.Y)[at] = o;
                else ((uint16_t*)p.Y)[at] = p.y_type == KQ_T_BF16 ? Act<true>::one(o) : Act<false>::one(o);
            }
        }
    }
}

BlockMatvecPlan block_matvec_plan(int m, int64_t n, int64_t k) {
    BlockMatvecPlan v = {};
    const int64_t blocks = block_pitch(k) / kBlock, tiles = ceil_div64(n, 16);
    v.row_tiles = 1;
    v.waves = 4;
    const int64_t room = tiles < 256 ? 256 / tiles : 1, long_enough = blocks >= 64 ? blocks / 16 : 1;
    const int64_t splits = room < long_enough ? room : long_enough;
    v.blocks_per_split = (int)ceil_div64(blocks, splits);
    v.splits = (int)ceil_div64(blocks, v.blocks_per_split);
    v.ws_bytes = v.splits > 1 ? (size_t)v.splits * (size_t)m * (size_t)n * sizeof(float) : 0;
    return v;
}

hipError_t launch_block_matvec(const BlockMatvecPlan& plan, BlockMatvecParams p, hipStream_t s) {
    p.splits = plan.splits;
    p.blocks_per_split = plan.blocks_per_split;
    if (p.splits == 1) p.part = nullptr;
    const dim3 grid((unsigned)ceil_div64(ceil_div64(p.n, 16), plan.row_tiles), (unsigned)p.splits), block(64 * plan.waves);
    if (plan.row_tiles != 1 || plan.waves != 4) return hipErrorInvalidValue;
    if (p.x_type == KQ_T_E4M3) block_matvec_kernel<KQ_T_E4M3, 4, 1><<<grid, block, 0, s>>>(p);
    else if (p.x_type == KQ_T_F32) block_matvec_kernel<KQ_T_F32, 4, 1><<<grid, block, 0, s>>>(p);
    else if (p.x_type == KQ_T_BF16) block_matvec_kernel<KQ_T_BF16, 4, 1><<<grid, block, 0, s>>>(p);
    else block_matvec_kernel<KQ_T_F16, 4, 1><<<grid, block, 0, s>>>(p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.splits == 1) return e;
    const JoinParams j = {p.part, p.splits, p.m, p.n, p.bias, p.Y, p.ldy, p.y_type};
    return launch_join(j, s);
}

}  // namespace kq
