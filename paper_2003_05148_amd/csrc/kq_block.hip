// The quantizer of 128-blocks in e4m3, what its values stand for, and the transposed forms that the gradients
// contract along: passes over memory.
#include "kq_block.h"
#include "kq_values.h"

namespace kq {

// ---- blocks of one row -------------------------------------------------------------------------------------
// Sixteen lanes a block, 8 columns a lane.  a 2^-e is exact, so the conversion's rounding is the only one.
template <int TYPE>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const BlockQuantizeParams p) {
    const unsigned per_row = (unsigned)(p.kp >> 3);       // 8-column pieces
    const unsigned id = blockIdx.x * 256u + threadIdx.x;  // (at most 2^34 values and their padding: fewer than 2^32 threads)
    const int64_t row = id / per_row;
    const bool live = row < p.m;                          // (blocks are whole: the lanes of one agree)
    const int c0 = live ? (int)(id - (unsigned)row * per_row) * 8 : 0;
    float v[8];
    load_columns<TYPE>(p.X, live ? row * p.ldx : 0, c0, live ? (int)p.k : 0, v);
    unsigned a = max_bits(v);
#pragma unroll
    for (int off = 1; off <= 8; off <<= 1) {
        const unsigned o = __shfl_xor(a, off);
        a = o > a ? o : a;
    }
    if (!live) return;
    const unsigned e = block_exponent(a);
    u32x2 w;
    if (e == 255u) {
        w = u32x2{0, 0};
#pragma unroll
        for (int t = 0; t < 8; ++t)
            if (c0 + t < p.k) w[t >> 2] |= 0x7fu << (8 * (t & 3));
    } else {
        const float inv = block_inverse(e);
        w = u32x2{encode4(v[0], v[1], v[2], v[3], inv), encode4(v[4], v[5], v[6], v[7], inv)};
    }
    *(u32x2*)(p.values + row * p.kp + c0) = w;
    if ((threadIdx.x & 15) == 0) p.exps[row * (p.kp >> 7) + (c0 >> 7)] = (uint8_t)e;
}

// ---- blocks of 128 rows ------------------------------------------------------------------------------------
// A workgroup a block, 16 lanes a row of it, eight rows a thread.
template <int TYPE>
__global__ __launch_bounds__(256) void quantize_tiles_kernel(const BlockQuantizeParams p) {
    __shared__ unsigned s_max[4];
    const unsigned ktiles = (unsigned)(p.kp >> 7);
    const unsigned kt = blockIdx.x % ktiles;
    const int64_t mt = blockIdx.x / ktiles;
    const int c0 = (int)kt * kBlock + 8 * (threadIdx.x & 15), r0 = threadIdx.x >> 4;
    float v[8][8];
    unsigned a = 0;
#pragma unroll
    for (int t = 0; t < 8; ++t) {
        const int64_t row = mt * kBlock + 16 * t + r0;
        const bool live = row < p.m;
        load_columns<TYPE>(p.X, live ? row * p.ldx : 0, c0, live ? (int)p.k : 0, v[t]);
    }
#pragma unroll
    for (int t = 0; t < 8; ++t) a = max(a, max_bits(v[t]));
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) a = max(a, (unsigned)__shfl_xor(a, off));
    if ((threadIdx.x & 63) == 0) s_max[threadIdx.x >> 6] = a;
    __syncthreads();
    a = max(max(s_max[0], s_max[1]), max(s_max[2], s_max[3]));
    const unsigned e = block_exponent(a);
    const float inv = e == 255u ? 0.0f : block_inverse(e);
#pragma unroll
    for (int t = 0; t < 8; ++t) {
        const int64_t row = mt * kBlock + 16 * t + r0;
        if (row >= p.m) break;
        u32x2 w;
        if (e == 255u) {
            w = u32x2{0, 0};
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c0 + j < p.k) w[j >> 2] |= 0x7fu << (8 * (j & 3));
        } else {
            w = u32x2{encode4(v[t][0], v[t][1], v[t][2], v[t][3], inv), encode4(v[t][4], v[t][5], v[t][6], v[t][7], inv)};
        }
        *(u32x2*)(p.values + row * p.kp + c0) = w;
    }
    if (threadIdx.x == 0) p.exps[blockIdx.x] = (uint8_t)e;
}

hipError_t launch_quantize_blocks(const BlockQuantizeParams& p, int rows, hipStream_t s) {
    const dim3 block(256);
    if (rows == 1) {
        const dim3 grid((unsigned)ceil_div64(p.m * (p.kp >> 3), 256));
        if (p.type == KQ_T_F32) quantize_rows_kernel<KQ_T_F32><<<grid, block, 0, s>>>(p);
        else if (p.type == KQ_T_BF16) quantize_rows_kernel<KQ_T_BF16><<<grid, block, 0, s>>>(p);
        else quantize_rows_kernel<KQ_T_F16><<<grid, block, 0, s>>>(p);
    } else {
        const dim3 grid((unsigned)(ceil_div64(p.m, kBlock) * (p.kp >> 7)));
        if (p.type == KQ_T_F32) quantize_tiles_kernel<KQ_T_F32><<<grid, block, 0, s>>>(p);
        else if (p.type == KQ_T_BF16) quantize_tiles_kernel<KQ_T_BF16><<<grid, block, 0, s>>>(p);
        else quantize_tiles_kernel<KQ_T_F16><<<grid, block, 0, s>>>(p);
    }
    return hipGetLastError();
}

// ---- reconstruction ----------------------------------------------------------------------------------------
// Sixteen lanes a block, four neighbouring columns at a time: a block's lanes write contiguous memory.
template <int TYPE>
__global__ __launch_bounds__(256) void reconstruct_blocks_kernel(const BlockReconstructParams p) {
    const unsigned per_row = (unsigned)(p.kp >> 3), id = blockIdx.x * 256u + threadIdx.x;  // (fewer than 2^32 threads)
    const int64_t row = id / per_row;
    if (row >= p.m) return;
    const unsigned piece = id - (unsigned)row * per_row;
    const int kb = (int)(piece >> 4);
    const float step = checkpoint_step(p.exps[(p.rows == 1 ? row : row >> 7) * (p.kp >> 7) + kb]);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int c0 = kb * kBlock + 64 * h + 4 * (int)(piece & 15);
        if (c0 >= p.k) break;
        const int w = *(const int*)(p.values + row * p.kp + c0);
        const float v[4] = {__builtin_amdgcn_cvt_f32_fp8(w, 0) * step, __builtin_amdgcn_cvt_f32_fp8(w, 1) * step,
                            __builtin_amdgcn_cvt_f32_fp8(w, 2) * step, __builtin_amdgcn_cvt_f32_fp8(w, 3) * step};
        store_values<TYPE, 4>(p.X_hat, row * p.ldx + c0, v, (int)(p.k - c0));
    }
}

hipError_t launch_reconstruct_blocks(const BlockReconstructParams& p, hipStream_t s) {
    const dim3 grid((unsigned)ceil_div64(p.m * (p.kp >> 3), 256)), block(256);
    if (p.type == KQ_T_F32) reconstruct_blocks_kernel<KQ_T_F32><<<grid, block, 0, s>>>(p);
    else if (p.type == KQ_T_BF16) reconstruct_blocks_kernel<KQ_T_BF16><<<grid, block, 0, s>>>(p);
    else reconstruct_blocks_kernel<KQ_T_F16><<<grid, block, 0, s>>>(p);
    return hipGetLastError();
}

// ---- transposed, and quantized along the other direction ---------------------------------------------------
// A workgroup takes 128 rows by 128 columns; a thread 8 neighbouring rows of 8 neighbouring columns, so that what it
// writes to LDS transposed are 8-byte pieces.  Piece q of column c lies at q ^ (c / 8): the sixteen column groups of a
// wave's store fall on sixteen different pieces.
template <int TYPE>
__device__ __forceinline__ void load_bytes_or_columns(const BlockTransposeParams& p, int64_t row, int64_t c0, float (&v)[8]) {
    if (row >= p.m || c0 >= p.cols) {
#pragma unroll
        for (int t = 0; t < 8; ++t) v[t] = 0.0f;
    } else if constexpr (TYPE == KQ_T_E4M3) {
        const u32x2 w = *(const u32x2*)((const uint8_t*)p.X + row * p.ldx + c0);
        const float step = checkpoint_step(p.in_exps[row * (p.ldx >> 7) + (c0 >> 7)]);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            v[4 * h] = __builtin_amdgcn_cvt_f32_fp8((int)w[h], 0) * step;
            v[4 * h + 1] = __builtin_amdgcn_cvt_f32_fp8((int)w[h], 1) * step;
            v[4 * h + 2] = __builtin_amdgcn_cvt_f32_fp8((int)w[h], 2) * step;
            v[4 * h + 3] = __builtin_amdgcn_cvt_f32_fp8((int)w[h], 3) * step;
        }
    } else {
        load_columns<TYPE>(p.X, row * p.ldx, (int)c0, (int)p.cols, v);
    }
}

// 128 columns of 128 bytes, from LDS to memory
__device__ __forceinline__ void store_transposed(const BlockTransposeParams& p, const u32x2* s_t, int64_t r0, int64_t c0) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const int id = t * 256 + threadIdx.x, c = id >> 3, q = 2 * (id & 7), sw = c >> 3;
        const u32x2 a = s_t[c * 16 + (q ^ sw)], b = s_t[c * 16 + ((q + 1) ^ sw)];
        if (c0 + c < p.cols) *(u32x4*)(p.values + (c0 + c) * p.rp + r0 + 8 * q) = u32x4{a.x, a.y, b.x, b.y};
    }
}

template <int TYPE>
__global__ __launch_bounds__(256) void transpose_quantize_kernel(const BlockTransposeParams p) {
    __shared__ u32x2 s_t[128 * 16];
    __shared__ unsigned s_max[4][128];
    __shared__ float s_sum[4][128];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = tid & 15, rg = tid >> 4;
    const unsigned ctiles = (unsigned)((p.cols + 127) >> 7), rt = blockIdx.x / ctiles;
    const int64_t c0 = (int64_t)(blockIdx.x - rt * ctiles) * 128, r0 = (int64_t)rt * 128;
    float v[8][8];
#pragma unroll
    for (int t = 0; t < 8; ++t) load_bytes_or_columns<TYPE>(p, r0 + 8 * rg + t, c0 + 8 * l16, v[t]);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        unsigned a = 0;
#pragma unroll
        for (int t = 0; t < 8; ++t) a = max(a, __builtin_bit_cast(unsigned, v[t][j]) & 0x7fffffffu);
        a = max(a, (unsigned)__shfl_xor(a, 16));
        a = max(a, (unsigned)__shfl_xor(a, 32));
        if (lane < 16) s_max[wave][8 * l16 + j] = a;
    }
    if (p.sums) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float s = 0.0f;
#pragma unroll
            for (int t = 0; t < 8; ++t) s += v[t][j];
            s += __shfl_xor(s, 16);
            s += __shfl_xor(s, 32);
            if (lane < 16) s_sum[wave][8 * l16 + j] = s;
        }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int c = 8 * l16 + j;
        const unsigned e = block_exponent(max(max(s_max[0][c], s_max[1][c]), max(s_max[2][c], s_max[3][c])));
        u32x2 w = {kNaN4, kNaN4};
        if (e != 255u) {
            const float inv = block_inverse(e);
            w = u32x2{encode4(v[0][j], v[1][j], v[2][j], v[3][j], inv), encode4(v[4][j], v[5][j], v[6][j], v[7][j], inv)};
        }
        s_t[c * 16 + (rg ^ l16)] = w;
    }
    __syncthreads();
    store_transposed(p, s_t, r0, c0);
    if (tid < 128 && c0 + tid < p.cols) {
        p.exps[(c0 + tid) * (p.rp >> 7) + rt] =
            (uint8_t)block_exponent(max(max(s_max[0][tid], s_max[1][tid]), max(s_max[2][tid], s_max[3][tid])));
        if (p.sums) p.sums[(int64_t)rt * p.cols + c0 + tid] = ((s_sum[0][tid] + s_sum[1][tid]) + s_sum[2][tid]) + s_sum[3][tid];
    }
}

// The same bytes transposed.
__global__ __launch_bounds__(256) void transpose_bytes_kernel(const BlockTransposeParams p) {
    __shared__ u32x2 s_t[128 * 16];
    const int tid = threadIdx.x, l16 = tid & 15, rg = tid >> 4;
    const unsigned ctiles = (unsigned)((p.cols + 127) >> 7), rt = blockIdx.x / ctiles;
    const int64_t c0 = (int64_t)(blockIdx.x - rt * ctiles) * 128, r0 = (int64_t)rt * 128;
    u32x2 v[8];
#pragma unroll
    for (int t = 0; t < 8; ++t) {  // (a column piece past the matrix is inside the padded row)
        const int64_t row = r0 + 8 * rg + t;
        v[t] = row < p.m ? *(const u32x2*)((const uint8_t*)p.X + row * p.ldx + c0 + 8 * l16) : u32x2{0, 0};
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        // 4 x 4 bytes: rows 4 g .. 4 g + 3 of columns 4 h .. 4 h + 3
        unsigned o[4][2];
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const unsigned a = v[4 * g][h], b = v[4 * g + 1][h], c = v[4 * g + 2][h], d = v[4 * g + 3][h];
            const unsigned ab0 = __builtin_amdgcn_perm(b, a, 0x05010400u), ab1 = __builtin_amdgcn_perm(b, a, 0x07030602u);
            const unsigned cd0 = __builtin_amdgcn_perm(d, c, 0x05010400u), cd1 = __builtin_amdgcn_perm(d, c, 0x07030602u);
            o[0][g] = __builtin_amdgcn_perm(cd0, ab0, 0x05040100u);
            o[1][g] = __builtin_amdgcn_perm(cd0, ab0, 0x07060302u);
            o[2][g] = __builtin_amdgcn_perm(cd1, ab1, 0x05040100u);
            o[3][g] = __builtin_amdgcn_perm(cd1, ab1, 0x07060302u);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) s_t[(8 * l16 + 4 * h + j) * 16 + (rg ^ l16)] = u32x2{o[j][0], o[j][1]};
    }
    __syncthreads();
    store_transposed(p, s_t, r0, c0);
}

hipError_t launch_transpose_blocks(const BlockTransposeParams& p, hipStream_t s) {
    const dim3 grid((unsigned)(ceil_div64(p.cols, 128) * (p.rp >> 7))), block(256);
    if (p.exps == nullptr) transpose_bytes_kernel<<<grid, block, 0, s>>>(p);
    else if (p.type == KQ_T_E4M3) transpose_quantize_kernel<KQ_T_E4M3><<<grid, block, 0, s>>>(p);
    else if (p.type == KQ_T_F32) transpose_quantize_kernel<KQ_T_F32><<<grid, block, 0, s>>>(p);
    else if (p.type == KQ_T_BF16) transpose_quantize_kernel<KQ_T_BF16><<<grid, block, 0, s>>>(p);
    else transpose_quantize_kernel<KQ_T_F16><<<grid, block, 0, s>>>(p);
    return hipGetLastError();
}

}  // namespace kq
