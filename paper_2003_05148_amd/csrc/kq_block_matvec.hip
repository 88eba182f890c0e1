// Y = X W^T for few rows of X (one token, a small batch, a small layer): a stream of the weight's bytes past the matrix cores.
//
// A wave multiplies 16 rows of W by 16 rows of X, a block of 128 columns at a time.  Lane (row r = l % 16, q = l / 16)
// takes columns 16 q .. 16 q + 15 and 64 more of both, so a wave's two loads of W are 16 rows of 64 neighbouring bytes;
// the bytes become bf16 on the way to the 16 x 16 x 32 matrix instruction, which is exact, and a block's fp32 sum
// takes both exponents at once.  A row's block of X lies in four lanes: its largest magnitude is two exchanges away,
// so X is quantized where it is used.  The waves of a workgroup take the blocks of its rows in turn and add their
// sums through LDS in order.  Where there are few rows of W the columns are also split over workgroups, joined by a
// second kernel.  One row of bf16 through 4096 x 25088 takes 21 us (103 MB at 4.9 TB/s, the rate of a copy; 18 for
// this kernel and 2.5 for the joining one), through 1000 x 512 about 4: a launch and three dependent loads.
#include "kq_block.h"
#include "kq_values.h"

namespace kq {

// A lane's 32 columns of a block of a row of X: 16 from 16 q and 16 from 64 + 16 q, as they lie in memory.  ODD: 16-bit rows that
// begin between two dwords.
using u32x4_a4 = __attribute__((ext_vector_type(4), aligned(4))) unsigned;
template <int TYPE, bool ODD>
struct XBlock {
    static constexpr int kRegs = TYPE == KQ_T_E4M3 ? 2 : TYPE == KQ_T_F32 ? 8 : 4;  // of 16 bytes
    static constexpr int kBytes = TYPE == KQ_T_E4M3 ? 1 : TYPE == KQ_T_F32 ? 4 : 2;
    u32x4 r[kRegs];
    unsigned e;   // KQ_T_E4M3: the exponent
    __device__ __forceinline__ void load(const char* row, int b, int q, int64_t k) {
        const int64_t c0 = (int64_t)b * kBlock + 16 * q;
        if (TYPE == KQ_T_E4M3 || c0 + 80 + ODD <= k) {
            if constexpr (!ODD) {
#pragma unroll
                for (int i = 0; i < kRegs; ++i)
                    __builtin_memcpy(&r[i], row + (c0 + i / (kRegs / 2) * 64) * kBytes + i % (kRegs / 2) * 16, 16);
            } else {
                // A 16-byte load takes several times as long there: the first value alone, the others (and one more) from the next
                // dword on, moved up (16 rows through 1000 x 1023: 5.5 us, 7.3 without; but 5.6 and 4.6 where no row begins
                // so).
                const char* const at = row + c0 * 2;
                const unsigned odd = (unsigned)(uintptr_t)at & 2u;
                unsigned lead[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    lead[h] = *(const uint16_t*)(at + 128 * h);
#pragma unroll
                    for (int i = 0; i < 2; ++i) r[2 * h + i] = *(const u32x4_a4*)(at + 128 * h + 16 * i + odd);
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    unsigned last = lead[h] << 16;
#pragma unroll
                    for (int t = 0; t < 8; ++t) {
                        const unsigned w = r[2 * h + t / 4][t & 3];
                        r[2 * h + t / 4][t & 3] = odd ? __builtin_amdgcn_alignbit(w, last, 16) : w;
                        last = w;
                    }
                }
            }
        } else {  // the row ends here
#pragma unroll
            for (int i = 0; i < kRegs; ++i) {
                constexpr int kIn = 16 / kBytes;   // values of a register
                const int64_t c = c0 + i / (kRegs / 2) * 64 + i % (kRegs / 2) * kIn;
                if (c + kIn <= k) {
                    __builtin_memcpy(&r[i], row + c * kBytes, 16);
                    continue;
                }
                // (loads at clamped places, all at once: a branch for each would wait for the one before)
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    if constexpr (TYPE == KQ_T_F32) {
                        const unsigned v = ((const unsigned*)row)[min(c + t, k - 1)];
                        r[i][t] = c + t < k ? v : 0u;
                    } else if constexpr (TYPE != KQ_T_E4M3) {
                        const unsigned lo = ((const uint16_t*)row)[min(c + 2 * t, k - 1)], hi = ((const uint16_t*)row)[min(c + 2 * t + 1, k - 1)];
                        r[i][t] = (c + 2 * t < k ? lo : 0u) | (c + 2 * t + 1 < k ? hi << 16 : 0u);
                    }
                }
            }
        }
    }
    // its bytes (x[0] the first 16 columns) and the block's exponent: the largest magnitude of four lanes
    __device__ __forceinline__ unsigned quantize(u32x4 (&x)[2]) const {
        if constexpr (TYPE == KQ_T_E4M3) {
            x[0] = r[0];
            x[1] = r[1];
            return e;
        } else {
            unsigned a = 0;
            if constexpr (TYPE == KQ_T_F32) {
#pragma unroll
                for (int i = 0; i < kRegs; ++i)
#pragma unroll
                    for (int t = 0; t < 4; ++t) a = max(a, r[i][t] & 0x7fffffffu);
            } else {  // the magnitudes of 16-bit floats order like integers, two at a time
                using u16x2 = __attribute__((ext_vector_type(2))) unsigned short;
                u16x2 m = {0, 0};
#pragma unroll
                for (int i = 0; i < kRegs; ++i)
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        const unsigned v = r[i][t] & 0x7fff7fffu;
                        m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, v));
                    }
                const unsigned h = m.x > m.y ? m.x : m.y;
                a = __builtin_bit_cast(unsigned, TYPE == KQ_T_BF16 ? Act<true>::lo(h) : Act<false>::lo(h));
            }
            a = max(a, (unsigned)__shfl_xor(a, 16));
            a = max(a, (unsigned)__shfl_xor(a, 32));
            const unsigned ex = block_exponent(a);
            const float scale = __builtin_bit_cast(float, (ex == 255u ? 127u : ex) << 23);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int t = 0; t < 4; ++t) {  // four bytes; the conversion divides by the power of two
                    using s16x2 = __attribute__((ext_vector_type(2))) short;
                    s16x2 w = {0, 0};
                    if constexpr (TYPE == KQ_T_F32) {
                        const unsigned v0 = r[4 * h + t][0], v1 = r[4 * h + t][1], v2 = r[4 * h + t][2], v3 = r[4 * h + t][3];
                        w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, __builtin_bit_cast(float, v0), __builtin_bit_cast(float, v1), scale, false);
                        w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, __builtin_bit_cast(float, v2), __builtin_bit_cast(float, v3), scale, true);
                    } else {
                        const unsigned v0 = r[2 * h + t / 2][2 * (t & 1)], v1 = r[2 * h + t / 2][2 * (t & 1) + 1];
                        if constexpr (TYPE == KQ_T_BF16) {
                            w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2, v0), scale, false);
                            w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2, v1), scale, true);
                        } else {
                            w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(w, __builtin_bit_cast(f16x2, v0), scale, false);
                            w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(w, __builtin_bit_cast(f16x2, v1), scale, true);
                        }
                    }
                    x[h][t] = __builtin_bit_cast(unsigned, w);
                }
            return ex;
        }
    }
};

// RT: 16-row tiles of W a workgroup takes; they share what a wave does to X.
template <int TYPE, int WAVES, int RT, bool ODD>
__global__ __launch_bounds__(64 * WAVES) void block_matvec_kernel(const BlockMatvecParams p) {
    __shared__ f32x4 s_sum[RT * WAVES * 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r16 = lane & 15, q = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * (16 * RT);
    const int blocks = (int)(p.kp >> 7);
    const int b_begin = blockIdx.y * p.blocks_per_split, b_end = min(b_begin + p.blocks_per_split, blocks);
    static_assert(kBlock % (16 * RT) == 0, "a workgroup's rows of W lie in one block");
    // rows past the last repeat it: what they give is not stored
    const uint8_t* w_row[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) w_row[t] = p.values + min(n0 + 16 * t + r16, p.n - 1) * p.kp + 16 * q;
    const uint8_t* const w_exp = p.exps + (n0 >> 7) * blocks;
    const int xr0 = (int)blockIdx.z * 16 + r16;
    const int64_t xr = min(xr0, p.m - 1);
    const char* const x_row = (const char*)p.X + xr * p.ldx * XBlock<TYPE, ODD>::kBytes;
    const uint8_t* const x_exp = TYPE == KQ_T_E4M3 ? p.x_exps + xr * blocks : nullptr;
    f32x4 y[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) y[t] = f32x4{0, 0, 0, 0};

    struct Block {
        u32x4 w[RT][2];
        unsigned ew;
        XBlock<TYPE, ODD> x;
    };
    auto fetch = [&](Block& f, int b) {
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            f.w[t][0] = *(const u32x4*)(w_row[t] + (int64_t)b * kBlock);
            f.w[t][1] = *(const u32x4*)(w_row[t] + (int64_t)b * kBlock + 64);
        }
        f.ew = w_exp[b];
        f.x.load(x_row, b, q, p.k);
        if constexpr (TYPE == KQ_T_E4M3) f.x.e = x_exp[b];
    };
    Block next;
    if (b_begin + wave < b_end) fetch(next, b_begin + wave);
    for (int b = b_begin + wave; b < b_end; b += WAVES) {  // the next block's loads are on their way
        const Block now = next;
        if (b + WAVES < b_end) fetch(next, b + WAVES);
        u32x4 x[2], xd[4];
        const unsigned ex = now.x.quantize(x);
#pragma unroll
        for (int i = 0; i < 4; ++i) xd[i] = decode8(x[i >> 1][2 * (i & 1)], x[i >> 1][2 * (i & 1) + 1], 1.0f);
        const int shift = (int)(now.ew + ex) - 254;
        const float one = now.ew == 255u || ex == 255u ? __builtin_bit_cast(float, 0x7fc00000u) : 1.0f;
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            f32x4 acc = {0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < 4; ++i) acc = Act<true>::mfma(decode8(now.w[t][i >> 1][2 * (i & 1)], now.w[t][i >> 1][2 * (i & 1) + 1], 1.0f), xd[i], acc);
#pragma unroll
            for (int r = 0; r < 4; ++r) y[t][r] = __builtin_fmaf(__builtin_ldexpf(acc[r], shift), one, y[t][r]);
        }
    }

    // lane holds Y[r16][n0 + 16 t + 4 q + r]: the waves' sums in order
#pragma unroll
    for (int t = 0; t < RT; ++t) s_sum[(t * WAVES + wave) * 64 + lane] = y[t];
    __syncthreads();
    if (wave < RT && xr0 < p.m) {
        f32x4 v = s_sum[wave * WAVES * 64 + lane];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v += s_sum[(wave * WAVES + w) * 64 + lane];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int64_t n = n0 + 16 * wave + 4 * q + r;
            if (n >= p.n) break;
            if (p.part) {
                p.part[((int64_t)blockIdx.y * p.m + xr0) * p.n + n] = v[r];
                continue;
            }
            const float o = v[r] + (p.bias ? p.bias[n] : 0.0f);
            const int64_t at = (int64_t)xr0 * p.ldy + n;
            if (p.y_type == KQ_T_F32) ((float*)p.Y)[at] = o;
            else ((uint16_t*)p.Y)[at] = p.y_type == KQ_T_BF16 ? Act<true>::one(o) : Act<false>::one(o);
        }
    }
}

// Row tiles a workgroup takes, splits of the columns and waves.  A wave's work on X (quantizing it, reading it from L2) is
// shared by its row tiles, so there are several where W is long or has more row tiles than the chip has room for; the
// columns are split where the workgroups would not fill the chip and are long enough for the joining launch (2 to 3 us).
// Measured (us, rows of bf16 X / n x k; row tiles x splits w waves):
//    1 / 4096 x 25088: 1x1w16 29.9, 2x2w8 23.1, 2x4w4 23.0, 4x4w4 23.6     16 / 4096 x 25088: 1x1w16 38.8, 2x2w8 29.3, 4x4w4 25.2
//    1 / 4096 x 4096:  1x1w8 6.7, 2x2w8 8.0, 4x4w4 8.5                     16 / 4096 x 4096:  4x4w8 9.0, 1x1w8 9.0
//    1 / 1000 x 25088: 2x8w8 9.5, 1x4w8 9.9, 4x8w4 above 11.7             16 / 1000 x 25088: 2x8w8 11.8, 1x4w8 13.7
//   16 / 8192 x 8192:  1x1 above 22, 2x1w8 19.3, 4x4w4 19.4                1 / 1000 x 512:   1x1w4 3.3, 2x1w4 3.6
BlockMatvecPlan block_matvec_plan(int m, int64_t n, int64_t k) {
    BlockMatvecPlan v = {};
    const int64_t blocks = block_pitch(k) / kBlock, tiles = ceil_div64(n, 16);
    v.row_tiles = blocks >= 96 ? (m > 4 && tiles > 128 ? 4 : 2) : tiles >= 512 ? 2 : 1;
    const int64_t groups = ceil_div64(tiles, v.row_tiles), room = groups < 256 ? 256 / groups : 1;
    const int64_t long_enough = blocks >= 16 ? blocks / 8 : 1;
    const int64_t splits = room < long_enough ? room : long_enough;
    v.blocks_per_split = (int)ceil_div64(blocks, splits);
    v.splits = (int)ceil_div64(blocks, v.blocks_per_split);
    v.waves = v.row_tiles == 4 || v.blocks_per_split <= 12 ? 4 : v.row_tiles == 2 || v.blocks_per_split <= 64 ? 8 : 16;
    v.ws_bytes = v.splits > 1 ? (size_t)v.splits * (size_t)m * (size_t)n * sizeof(float) : 0;
    return v;
}

// More than 16 rows: sixteens of them in the grid's third dimension.  Every workgroup quantizes its rows of X again, so this is
// for products that are small: nothing is launched before it, and its workgroups are smaller than the product's.  A
// workgroup's block takes `x` us for X and 0.054 us for each row tile, and workgroups of one CU share it; a split
// contraction pays the joining launch.  Fitted to (us, rows / n x k; here and quantizer and product): 64 / 1000 x 512
// bf16 4.4 and 8.5, fp32 4.8 and 9.7, 8-bit X 3.9 and 5.8; 64 / 1000 x 4096 bf16 8.6 (4x4w4) and 12.4; 32 / 4096 x 4096
// 10.9 (2x1w4) and 12.9, 64 / 4096 x 4096 14.2 and 13.9; 512 / 1000 x 512 6.9 (4x1w4) and 8.7.
BlockMatvecPlan block_matvec_plan(int x_type, int m, int64_t n, int64_t k) {
    const int64_t blocks = block_pitch(k) / kBlock;
    const float x = x_type == KQ_T_E4M3 ? 0.06f : x_type == KQ_T_F32 ? 0.215f : 0.109f;
    const float value_us = (float)m * (float)n * 8.0f / 6e6f;
    BlockMatvecPlan v = {};
    for (int rt = 1; rt <= 4; rt *= 2) {
        const int64_t groups = ceil_div64(n, 16 * rt) * ceil_div64(m, 16);
        for (int splits = 1; splits <= 8 && splits <= (blocks + 3) / 4; splits *= 2) {
            const int64_t per = ceil_div64(blocks, splits), workgroups = groups * ceil_div64(blocks, per);
            const float share = workgroups > 256 ? (float)workgroups / 256.0f : 1.0f;
            const float us = 3.8f + share * (float)per * (x + 0.054f * (float)rt) + (splits > 1 ? 2.0f + (float)splits * value_us : 0.0f);
            if (v.row_tiles && us >= v.us) continue;
            v = {rt, 4, (int)ceil_div64(blocks, per), (int)per, 0, us};
        }
    }
    v.ws_bytes = v.splits > 1 ? (size_t)v.splits * (size_t)m * (size_t)n * sizeof(float) : 0;
    return v;
}

template <int TYPE, bool ODD = false>
static void launch_matvec_type(const BlockMatvecPlan& v, const BlockMatvecParams& p, hipStream_t s) {
    const dim3 grid((unsigned)ceil_div64(p.n, 16 * v.row_tiles), (unsigned)p.splits, (unsigned)ceil_div64(p.m, 16)), block(64 * v.waves);
    if (v.row_tiles == 4) {
        block_matvec_kernel<TYPE, 4, 4, ODD><<<grid, block, 0, s>>>(p);
    } else if (v.row_tiles == 2) {
        if (v.waves == 8) block_matvec_kernel<TYPE, 8, 2, ODD><<<grid, block, 0, s>>>(p);
        else block_matvec_kernel<TYPE, 4, 2, ODD><<<grid, block, 0, s>>>(p);
    } else {
        if (v.waves == 16) block_matvec_kernel<TYPE, 16, 1, ODD><<<grid, block, 0, s>>>(p);
        else if (v.waves == 8) block_matvec_kernel<TYPE, 8, 1, ODD><<<grid, block, 0, s>>>(p);
        else block_matvec_kernel<TYPE, 4, 1, ODD><<<grid, block, 0, s>>>(p);
    }
}

hipError_t launch_block_matvec(const BlockMatvecPlan& plan, BlockMatvecParams p, hipStream_t s) {
    p.splits = plan.splits;
    p.blocks_per_split = plan.blocks_per_split;
    const bool odd = ((uintptr_t)p.X & 2) || (p.m > 1 && (p.ldx & 1));
    if (p.splits == 1) p.part = nullptr;
    if (p.x_type == KQ_T_E4M3) launch_matvec_type<KQ_T_E4M3>(plan, p, s);
    else if (p.x_type == KQ_T_F32) launch_matvec_type<KQ_T_F32>(plan, p, s);
    else if (p.x_type == KQ_T_BF16 && odd) launch_matvec_type<KQ_T_BF16, true>(plan, p, s);
    else if (p.x_type == KQ_T_BF16) launch_matvec_type<KQ_T_BF16>(plan, p, s);
    else if (odd) launch_matvec_type<KQ_T_F16, true>(plan, p, s);
    else launch_matvec_type<KQ_T_F16>(plan, p, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.splits == 1) return e;
    const JoinParams j = {p.part, p.splits, p.m, p.n, p.bias, p.Y, p.ldy, p.y_type};
    return launch_join(j, s);
}

}  // namespace kq
