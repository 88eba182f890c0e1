// The quantizer of 128-blocks in e4m3, what its values stand for, and the transposed forms that the gradients
// contract along: passes over memory.
#include "kq_block.h"
#include "kq_values.h"

namespace kq {

// ---- blocks of one row -------------------------------------------------------------------------------------
// Sixteen lanes a block, 8 columns a lane: a block's largest magnitude is four exchanges away.  x 2^-e is exact, so the
// conversion's rounding is the only one.  Memory bounds it (4096 x 4096 bf16: 10.2 us, 50 MB), a launch where it is small (33 x
// 1000 fp32: 2.5 us).
template <int TYPE>
__device__ __forceinline__ void quantize_rows(const BlockQuantizeParams& p, unsigned workgroup) {
    const unsigned per_row = (unsigned)(p.kp >> 3);       // 8-column pieces
    const unsigned id = workgroup * 256u + threadIdx.x;  // (at most 2^34 values and their padding: fewer than 2^32 threads)
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
template <int TYPE>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const BlockQuantizeParams p) {
    quantize_rows<TYPE>(p, blockIdx.x);
}
static unsigned quantize_rows_workgroups(const BlockQuantizeParams& p) { return (unsigned)ceil_div64(p.m * (p.kp >> 3), 256); }

// ---- blocks of 128 rows ------------------------------------------------------------------------------------
// A workgroup a block, 16 lanes a row of it, eight rows a thread: the block stays in registers between its largest magnitude
// and the conversion, so it is read once.  Memory bounds it (4096 x 25088 fp32: 87 us, 5.9 TB/s).
template <int TYPE>
__global__ __launch_bounds__(256) void quantize_tiles_kernel(const BlockQuantizeParams p) {
    __shared__ unsigned s_max[4];
    const unsigned ktiles = (unsigned)(p.kp >> 7);
    const unsigned kt = blockIdx.x % ktiles;
    const int64_t mt = blockIdx.x / ktiles;
    const int c0 = (int)kt * kBlock + 8 * (threadIdx.x & 15), r0 = threadIdx.x >> 4;
    float v[8][8];
    unsigned a = 0;
    const int rows = (int)min(p.m - mt * kBlock, (int64_t)kBlock);
    const int64_t first = mt * kBlock * p.ldx;
    // (rows and columns past the last: loads at clamped places, all of a thread's on their way before the first is looked at;
    // 4096 x 4095 bf16 14.1 us, 17.9 with a branch for each row)
    if (c0 + 8 <= p.k) {
#pragma unroll
        for (int t = 0; t < 8; ++t) load_values<TYPE, 8>(p.X, first + min(16 * t + r0, rows - 1) * p.ldx + c0, v[t]);
    } else {
#pragma unroll
        for (int t = 0; t < 8; ++t)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[t][j] = load_value_as<TYPE>(p.X, first + min(16 * t + r0, rows - 1) * p.ldx + min((int64_t)c0 + j, p.k - 1));
#pragma unroll
        for (int t = 0; t < 8; ++t)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[t][j] = c0 + j < p.k ? v[t][j] : 0.0f;
    }
#pragma unroll
    for (int t = 0; t < 8; ++t) a = max(a, max_bits(v[t]));  // (a row again: the same magnitudes)
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
        const dim3 grid(quantize_rows_workgroups(p));
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
// Sixteen lanes a block, four neighbouring columns at a time: a block's lanes write contiguous memory.  v 2^e has 4 significant
// bits, so only 16-bit outputs round (beyond fp16's range, or below a type's smallest normal number).  Memory bounds it
// (4096 x 25088 to fp32: 76 us, 6.8 TB/s, its stores past the caches' normal ways; rows that do not begin on 16 bytes have
// ordinary ones, 4096 x 25087: 120 us, 168 streamed).
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
// wave's store fall on sixteen different pieces.  All of a thread's loads are on their way before the first is used.
// Memory bounds it where it is large (dY 4096 x 4096 bf16 and X 4096 x 25088 in one launch: 53 us, 256 MB at 4.8 TB/s), and a
// workgroup's own latency, about 4 us, where it is small (2047 x 1000 and 2047 x 4095: 10.5 us for 640 workgroups).
struct TransposeShared {
    u32x2 t[128 * 16];
    unsigned exps[4][64];   // of two neighbouring columns
    float sum[4][128];
};
__device__ __forceinline__ unsigned tile_of(const BlockTransposeParams& p, unsigned workgroup, int64_t& r0, int64_t& c0) {
    const unsigned ctiles = (unsigned)((p.cols + 127) >> 7), rt = workgroup / ctiles;
    c0 = (int64_t)(workgroup - rt * ctiles) * 128;
    r0 = (int64_t)rt * 128;
    return rt;
}
static unsigned transpose_workgroups(const BlockTransposeParams& p) { return (unsigned)(ceil_div64(p.cols, 128) * (p.rp >> 7)); }

// 128 columns of 128 bytes, from LDS to memory
__device__ __forceinline__ void store_transposed(const BlockTransposeParams& p, const u32x2* s_t, int64_t r0, int64_t c0) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const int id = t * 256 + threadIdx.x, c = id >> 3, q = 2 * (id & 7), sw = c >> 3;
        const u32x2 a = s_t[c * 16 + (q ^ sw)], b = s_t[c * 16 + ((q + 1) ^ sw)];
        if (c0 + c < p.cols) *(u32x4*)(p.values + (c0 + c) * p.rp + r0 + 8 * q) = u32x4{a.x, a.y, b.x, b.y};
    }
}

// A thread's 8 x 8 values as they lie in memory: zeros past the matrix.
template <int TYPE>
struct RawTile {
    static constexpr int kWords = TYPE == KQ_T_F32 ? 8 : TYPE == KQ_T_E4M3 ? 2 : 4;
    static constexpr int kBytes = TYPE == KQ_T_F32 ? 4 : TYPE == KQ_T_E4M3 ? 1 : 2;
    unsigned w[8][kWords];
    float step[8];   // KQ_T_E4M3: the row's power of two
    __device__ __forceinline__ void load(const BlockTransposeParams& p, int64_t r0, int64_t c0) {
        const int64_t first = min(r0, p.m - 1);
        const int last = (int)min(p.m - 1 - first, (int64_t)7);  // (rows past it: again, and cleared below)
        const char* at = (const char*)p.X + first * p.ldx * kBytes;
        if (TYPE == KQ_T_E4M3 || c0 + 8 <= p.cols) {  // (bytes: whole padded rows)
            at += c0 * kBytes;
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                __builtin_memcpy(w[t], at, 4 * kWords);
                at += t < last ? p.ldx * kBytes : 0;
            }
        } else {  // a row's end: loads at clamped places, all at once
#pragma unroll
            for (int t = 0; t < 8; ++t) {
#pragma unroll
                for (int j = 0; j < kWords; ++j) {
                    if constexpr (TYPE == KQ_T_F32) {
                        const unsigned v = ((const unsigned*)at)[min(c0 + j, p.cols - 1)];
                        w[t][j] = c0 + j < p.cols ? v : 0u;
                    } else {
                        const unsigned lo = ((const uint16_t*)at)[min(c0 + 2 * j, p.cols - 1)], hi = ((const uint16_t*)at)[min(c0 + 2 * j + 1, p.cols - 1)];
                        w[t][j] = (c0 + 2 * j < p.cols ? lo : 0u) | (c0 + 2 * j + 1 < p.cols ? hi << 16 : 0u);
                    }
                }
                at += t < last ? p.ldx * kBytes : 0;
            }
        }
        if constexpr (TYPE == KQ_T_E4M3) {
            const int64_t pitch = p.ldx >> 7;
            const uint8_t* e = p.in_exps + first * pitch + (c0 >> 7);
            unsigned x[8];
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                x[t] = *e;
                e += t < last ? pitch : 0;
            }
#pragma unroll
            for (int t = 0; t < 8; ++t) step[t] = checkpoint_step(x[t]);
        }
        if (r0 + 8 > p.m) {
#pragma unroll
            for (int t = 0; t < 8; ++t)
                if (r0 + t >= p.m) {
                    step[t] = 0.0f;
#pragma unroll
                    for (int j = 0; j < kWords; ++j) w[t][j] = 0;
                }
        }
    }
    // columns 2 j and 2 j + 1 of row t
    __device__ __forceinline__ void pair(int t, int j, float& a, float& b) const {
        if constexpr (TYPE == KQ_T_F32) {
            a = __builtin_bit_cast(float, w[t][2 * j]);
            b = __builtin_bit_cast(float, w[t][2 * j + 1]);
        } else if constexpr (TYPE == KQ_T_E4M3) {
            const f32x2 v = j & 1 ? __builtin_amdgcn_cvt_pk_f32_fp8((int)w[t][j >> 1], true) : __builtin_amdgcn_cvt_pk_f32_fp8((int)w[t][j >> 1], false);
            a = v.x * step[t];
            b = v.y * step[t];
        } else {
            a = Act<TYPE == KQ_T_BF16>::lo(w[t][j]);
            b = Act<TYPE == KQ_T_BF16>::hi(w[t][j]);
        }
    }
};

__device__ __forceinline__ unsigned max_u16x2(unsigned a, unsigned b) {
    using u16x2 = __attribute__((ext_vector_type(2))) unsigned short;
    return __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}

template <int TYPE, bool SUMS>
__device__ __forceinline__ void transpose_quantize(const BlockTransposeParams& p, unsigned workgroup, TransposeShared& s) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = tid & 15, rg = tid >> 4;
    int64_t r0, c0;
    const unsigned rt = tile_of(p, workgroup, r0, c0);
    RawTile<TYPE> raw;
    raw.load(p, r0 + 8 * rg, c0 + 8 * l16);
    // A block's exponent is the largest of its rows' (it never falls as the magnitude grows), so exponents are exchanged, two
    // columns a register.
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float a = 0.0f, b = 0.0f, sa = 0.0f, sb = 0.0f;
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            float x, y;
            raw.pair(t, j, x, y);
            a = __builtin_elementwise_maximum(a, __builtin_fabsf(x));  // (a NaN stays)
            b = __builtin_elementwise_maximum(b, __builtin_fabsf(y));
            if constexpr (SUMS) {
                sa += x;
                sb += y;
            }
        }
        unsigned e = block_exponent(__builtin_bit_cast(unsigned, a) & 0x7fffffffu) | block_exponent(__builtin_bit_cast(unsigned, b) & 0x7fffffffu) << 16;
        e = max_u16x2(e, (unsigned)__shfl_xor(e, 16));
        e = max_u16x2(e, (unsigned)__shfl_xor(e, 32));
        if (lane < 16) s.exps[wave][4 * l16 + j] = e;
        if constexpr (SUMS) {
            sa += __shfl_xor(sa, 16);
            sb += __shfl_xor(sb, 16);
            sa += __shfl_xor(sa, 32);
            sb += __shfl_xor(sb, 32);
            if (lane < 16) {
                s.sum[wave][8 * l16 + 2 * j] = sa;
                s.sum[wave][8 * l16 + 2 * j + 1] = sb;
            }
        }
    }
    __syncthreads();
    auto exponents = [&](int pair) { return max_u16x2(max_u16x2(s.exps[0][pair], s.exps[1][pair]), max_u16x2(s.exps[2][pair], s.exps[3][pair])); };
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int c = 8 * l16 + 2 * j;
        const unsigned e = exponents(4 * l16 + j), ea = e & 0xffffu, eb = e >> 16;
        float x[8], y[8];
#pragma unroll
        for (int t = 0; t < 8; ++t) raw.pair(t, j, x[t], y[t]);
        const float ia = block_inverse(ea == 255u ? 127u : ea), ib = block_inverse(eb == 255u ? 127u : eb);
        u32x2 a = {encode4(x[0], x[1], x[2], x[3], ia), encode4(x[4], x[5], x[6], x[7], ia)};
        u32x2 b = {encode4(y[0], y[1], y[2], y[3], ib), encode4(y[4], y[5], y[6], y[7], ib)};
        if (ea == 255u) a = u32x2{kNaN4, kNaN4};
        if (eb == 255u) b = u32x2{kNaN4, kNaN4};
        s.t[c * 16 + (rg ^ l16)] = a;
        s.t[(c + 1) * 16 + (rg ^ l16)] = b;
    }
    __syncthreads();
    store_transposed(p, s.t, r0, c0);
    if (tid < 128 && c0 + tid < p.cols) {
        p.exps[(c0 + tid) * (p.rp >> 7) + rt] = (uint8_t)(exponents(tid >> 1) >> (16 * (tid & 1)));
        if constexpr (SUMS) p.sums[(int64_t)rt * p.cols + c0 + tid] = ((s.sum[0][tid] + s.sum[1][tid]) + s.sum[2][tid]) + s.sum[3][tid];
    }
}

// Both operands of a gradient in one launch, the first `first` workgroups the first of them: two short passes after each
// other leave half the chip idle at their ends, and each launch costs 2 to 3 us.
template <int TYPE>
__global__ __launch_bounds__(256) void grad_weight_operands_kernel(const BlockTransposeParams x, const BlockTransposeParams dy, unsigned first) {
    __shared__ TransposeShared s;
    if (blockIdx.x < first) transpose_quantize<KQ_T_E4M3, false>(x, blockIdx.x, s);
    else if (dy.sums) transpose_quantize<TYPE, true>(dy, blockIdx.x - first, s);
    else transpose_quantize<TYPE, false>(dy, blockIdx.x - first, s);
}

hipError_t launch_grad_weight_operands(const BlockTransposeParams& x, const BlockTransposeParams& dy, hipStream_t s) {
    const unsigned first = transpose_workgroups(x);
    const dim3 grid(first + transpose_workgroups(dy)), block(256);
    if (dy.type == KQ_T_F32) grad_weight_operands_kernel<KQ_T_F32><<<grid, block, 0, s>>>(x, dy, first);
    else if (dy.type == KQ_T_BF16) grad_weight_operands_kernel<KQ_T_BF16><<<grid, block, 0, s>>>(x, dy, first);
    else grad_weight_operands_kernel<KQ_T_F16><<<grid, block, 0, s>>>(x, dy, first);
    return hipGetLastError();
}

}  // namespace kq
