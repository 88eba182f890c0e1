// Y = X W^T for few rows of X (one token, a small batch): a stream of the packed codes past the matrix
// cores.
//
// A wave multiplies 16 rows of W by 16 rows of X, 128 columns at a time: 16 bytes of codes a lane are one
// contiguous kilobyte and four operands of the 16 x 16 x 32 matrix instruction, so the codes go from memory
// to the matrix cores through registers alone.  A code q becomes 1 + q / 16 in one shift and one masked OR a pair
// (the four bits are the top of the mantissa of 1); a product of X with the constant -1.5 is added, and so the sum
// is that of x (q - 8) / 16.  (Products and sums stay below 2 |x|: with 16 + q and -24 they overflowed for finite X.)
// Its fp32 rounding is that of terms of up to 31 |x| where the direct sum's are of up to 8 |x|.  Tables of levels
// are looked up with byte permutes.  Every product is exact (in fp16 a table's levels are brought into its range by a
// power of two, which the scales take off); a group's fp32 sum takes the group's scale in fp32, and without a table
// the row's sum the factor 16 at the end.
// The waves of a workgroup take the 128-column blocks of its rows in turn and add their sums through LDS in
// order.  Where there are few rows of W the columns are also split over workgroups, joined by a second kernel.
//
// Measured: one token through 4096 x 25088, 128 columns a group, 10.8 to 11.1 us a call (4.8 to 4.9 TB/s: memory, at the
// rate of a large copy; the streaming passes reach 6 TB/s, which would be 9 us).  Without a table a kilobyte of codes takes about 60 vector instructions, a fifth of the
// time that memory leaves; with a table about 140.  One token through 1000 x 512: 4.5 to 4.9 us a call, kernel 3.0: the
// launch.  13 rows of fp16 through 4096 x 4096 with a table, 32 columns a group: 7.2 us; X's fragments from L2 (four
// loads beside each load of codes) and the load latency of four dependent rounds.
#include "kq_group.h"

namespace kq {

// ---- codes to 16-bit values -------------------------------------------------------------------------------

// the 8 columns of a dword of codes, in order: levels, or 1 + q / 16 without a table
template <bool BF, bool LUT>
__device__ __forceinline__ u32x4 decode(unsigned d, const LevelTable& t) {
    u32x4 o;
    if constexpr (LUT) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {  // nibbles 0 2 4 6 are columns 0 4 1 5, nibbles 1 3 5 7 columns 2 6 3 7
            const unsigned idx = (h ? d >> 4 : d) & 0x0f0f0f0fu;
            const unsigned low3 = idx & 0x07070707u, pick = ((idx >> 1) & 0x04040404u) | 0x03020100u;
            const unsigned lo = look_up(t.lo, low3, pick), hi = look_up(t.hi, low3, pick);
            o[h] = __builtin_amdgcn_perm(hi, lo, 0x06020400u);
            o[2 + h] = __builtin_amdgcn_perm(hi, lo, 0x07030501u);
        }
    } else if constexpr (BF) {
        o[0] = ((d << 3) & 0x00780078u) | 0x3f803f80u;
        o[1] = ((d >> 1) & 0x00780078u) | 0x3f803f80u;
        o[2] = ((d >> 5) & 0x00780078u) | 0x3f803f80u;
        o[3] = ((d >> 9) & 0x00780078u) | 0x3f803f80u;
    } else {
        o[0] = ((d << 6) & 0x03c003c0u) | 0x3c003c00u;
        o[1] = ((d << 2) & 0x03c003c0u) | 0x3c003c00u;
        o[2] = ((d >> 2) & 0x03c003c0u) | 0x3c003c00u;
        o[3] = ((d >> 6) & 0x03c003c0u) | 0x3c003c00u;
    }
    return o;
}

// 8 neighbours of a row of X from column c, zeros from `limit` on
__device__ __forceinline__ u32x4 load_x(const uint16_t* row, int c, int limit, bool full) {
    u32x4 v;
    if (full || c + 8 <= limit) {
        __builtin_memcpy(&v, row + c, 16);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const unsigned lo = c + 2 * e < limit ? row[c + 2 * e] : 0u;
            const unsigned hi = c + 2 * e + 1 < limit ? row[c + 2 * e + 1] : 0u;
            v[e] = lo | (hi << 16);
        }
    }
    return v;
}

// GPB: groups a block (1, 2 or 4).  RT: 16-row tiles of W a workgroup takes.  XLDS: X (at most
// kMatvecLdsRows rows) is staged through LDS in chunks of p.chunk blocks; otherwise its fragments come from
// the caches with the codes.  A wave loads its next block while it multiplies the one before.
template <bool BF, bool LUT, int GPB, int WAVES, int RT, bool XLDS>
__global__ __launch_bounds__(64 * WAVES) void group_matvec_kernel(const MatvecParams p) {
    constexpr int kSumBytes = WAVES * RT * 64 * 16;
    constexpr int kXBytes = XLDS ? kMatvecLdsBytes : 0;
    constexpr int kPieces = 4 / GPB;  // 32-column pieces a group
    __shared__ u32x4 s_buf[(kSumBytes > kXBytes ? kSumBytes : kXBytes) / 16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r16 = lane & 15, q = lane >> 4;
    const int nt0 = blockIdx.x * RT;
    const int k_begin = blockIdx.y * p.blocks_per_split;
    const int k_end = min(k_begin + p.blocks_per_split, p.w.ktiles);
    // row tiles and rows past the last repeat it: what they give is not stored
    const uint8_t* codes[RT];
    const uint16_t* scales[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        codes[t] = p.w.codes + (int64_t)min(nt0 + t, p.w.ntiles - 1) * p.w.ktiles * kTileBytes;
        scales[t] = p.w.scales + (int64_t)min((nt0 + t) * kTileRows + r16, p.w.n - 1) * p.w.groups;
    }
    const unsigned code_off = r16 * 64 + q * 16;
    const uint16_t* xrow = (const uint16_t*)p.X + (int64_t)min(r16, p.m - 1) * p.ldx;

    const unsigned offset_bits = BF ? 0xbfc0bfc0u : 0xbe00be00u;  // a pair of -1.5
    const u32x4 offset = {offset_bits, offset_bits, offset_bits, offset_bits};
    LevelTable table;
    f32x4 y[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) y[t] = f32x4{0, 0, 0, 0};

    const int chunk = XLDS ? p.chunk : k_end - k_begin;
    const int pitch = chunk * 16 + 4;  // 16-byte pieces of a staged row: rows 64 bytes apart in the banks
    struct Block {
        u32x4 codes[RT], x[XLDS ? 1 : 4];
        unsigned short s[RT][GPB];
    };
    auto fetch = [&](Block& f, int kb) {  // past the end, the last block again
        const int b = min(kb, p.w.ktiles - 1);
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            f.codes[t] = *(const u32x4*)(codes[t] + (int64_t)b * kTileBytes + code_off);
            if (GPB == 1 || (b + 1) * GPB <= p.w.groups) {
                __builtin_memcpy(f.s[t], scales[t] + b * GPB, 2 * GPB);
            } else {
#pragma unroll
                for (int g = 0; g < GPB; ++g) f.s[t][g] = scales[t][min(b * GPB + g, p.w.groups - 1)];
            }
        }
        if constexpr (!XLDS) {
            const bool full = (b + 1) * kTileCols <= p.w.k;
#pragma unroll
            for (int i = 0; i < 4; ++i) f.x[i] = load_x(xrow, b * kTileCols + 32 * i + 8 * q, p.w.k, full);
        }
    };
    for (int c0 = k_begin; c0 < k_end; c0 += chunk) {
        const int c1 = min(c0 + chunk, k_end);
        Block next;
        fetch(next, c0 + wave);
        if constexpr (LUT) table = load_levels<BF>(p.w.levels);  // (after the loads that take longest)
        if constexpr (XLDS) {
            __syncthreads();  // the previous chunk is read
            const int pieces = (c1 - c0) * 16;
            for (int r = 0; r < p.m; ++r)
                for (int ch = threadIdx.x; ch < pieces; ch += 64 * WAVES)
                    s_buf[r * pitch + ch] = load_x((const uint16_t*)p.X + (int64_t)r * p.ldx, c0 * kTileCols + ch * 8, p.w.k, false);
            __syncthreads();
        }
        for (int b = c0 + wave; b < c1; b += WAVES) {
            const Block cur = next;
            if (b + WAVES < c1) fetch(next, b + WAVES);
            f32x4 acc[RT], base;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                u32x4 x;
                if constexpr (XLDS) x = s_buf[min(r16, p.m - 1) * pitch + (b - c0) * 16 + 4 * i + q];
                else x = cur.x[i];
                if (i % kPieces == 0) base = f32x4{0, 0, 0, 0};
                if constexpr (!LUT) base = Act<BF>::mfma(x, offset, base);  // once for all row tiles
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    const u32x4 w = decode<BF, LUT>(cur.codes[t][i], table);
                    if (i % kPieces == 0) acc[t] = f32x4{0, 0, 0, 0};
                    acc[t] = Act<BF>::mfma(x, w, acc[t]);
                    if ((i + 1) % kPieces == 0) {  // the group's last piece
                        if constexpr (!LUT) acc[t] += base;
                        float s = bf16_bits_to_f32(cur.s[t][i / kPieces]);
                        if constexpr (LUT && !BF) s = __builtin_ldexpf(s, -table.shift);
#pragma unroll
                        for (int r = 0; r < 4; ++r) y[t][r] = __builtin_fmaf(s, acc[t][r], y[t][r]);
                    }
                }
            }
        }
    }

    // lane holds Y[4 q + r][16 (nt0 + t) + r16]: the waves' sums in order
    if constexpr (XLDS) __syncthreads();
    f32x4* s_sum = (f32x4*)s_buf;
#pragma unroll
    for (int t = 0; t < RT; ++t) s_sum[(t * WAVES + wave) * 64 + lane] = LUT ? y[t] : y[t] * 16.0f;
    __syncthreads();
    if (wave < RT) {
        f32x4 v = s_sum[wave * WAVES * 64 + lane];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v += s_sum[(wave * WAVES + w) * 64 + lane];
        const int n = (nt0 + wave) * kTileRows + r16;
        if (n < p.w.n) {
            const float bias = p.bias && !p.part ? p.bias[n] : 0.0f;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int m = 4 * q + r;
                if (m < p.m) {
                    if (p.part) p.part[((int64_t)blockIdx.y * p.m + m) * p.w.n + n] = v[r];
                    else ((uint16_t*)p.Y)[(int64_t)m * p.ldy + n] = Act<BF>::one(v[r] + bias);
                }
            }
        }
    }
}

// Row tiles a workgroup takes, splits of the columns and waves.  A workgroup's time grows with the bytes of X
// it reads beside its codes, so several row tiles share a workgroup's X where X is long or there are more row
// tiles than the chip has room for; the columns are split where the workgroups would not fill the chip and
// are long enough to pay for the joining launch (about 3 us).  Measured (us, rows of X / n x k, group 128;
// row tiles x splits):
//   16 / 4096 x 25088: 1x1 27.9, 2x2 20.1, 4x4 17.5    8 / 4096 x 12288: 1x1 13.1, 2x2 12.4, 4x4 12.4
//   16 / 4096 x 8192:  1x1 12.2, 2x2 11.2, 4x4 11.4    16 / 8192 x 8192: 1x1 22.0, 2x1 15.2, 4x2 15.2
//   16 / 1000 x 8192:  1x1 11.9, 1x2 9.5, 1x4 7.7      16 / 1000 x 25088: 1x1 27.5, 1x4 11.8, 4x8 12.8
//    1 / 1000 x 4096:  1x1 4.9, 1x2 7.7                 1 / 1000 x 25088: 1x1 10.5, 1x2 9.7, 1x4 8.0
// and of waves: 1 / 4096 x 25088, 8 waves 13.1, 16 waves 11.4; 1 / 4096 x 4096, 4 waves 5.2, 8 4.4, 16 4.4;
// 1 / 1000 x 512 (kernel alone), 4 waves 3.2, 8 3.8, 16 4.7.
MatvecPlan matvec_plan(int m, int64_t n, int64_t k) {
    MatvecPlan v = {};
    const int64_t blocks = ceil_div64(k, kTileCols), tiles = ceil_div64(n, kTileRows);
    const bool lds = m <= kMatvecLdsRows;
    v.row_tiles = lds ? 1 : tiles >= 1024 || (blocks >= 96 && tiles > 128) ? 4 : tiles >= 512 ? 2 : 1;
    const int64_t groups = ceil_div64(tiles, v.row_tiles), room = groups < 256 ? 256 / groups : 1;
    const int64_t long_enough = lds ? (blocks >= 128 ? blocks / 48 : 1) : (blocks >= 64 ? blocks / 16 : 1);
    const int64_t splits = room < long_enough ? room : long_enough;
    v.blocks_per_split = (int)ceil_div64(blocks, splits);
    v.splits = (int)ceil_div64(blocks, v.blocks_per_split);
    v.waves = v.blocks_per_split < 16 ? 4 : v.blocks_per_split < 96 || !lds ? 8 : 16;
    if (v.row_tiles == 4) v.waves = 8;
    v.ws_bytes = v.splits > 1 ? (size_t)v.splits * (size_t)m * (size_t)n * sizeof(float) : 0;
    return v;
}

template <bool BF, bool LUT, int GPB>
static void launch_matvec_groups(const MatvecPlan& v, const MatvecParams& p, hipStream_t s) {
    const dim3 grid((unsigned)ceil_div(p.w.ntiles, v.row_tiles), (unsigned)p.splits), block(64 * v.waves);
    if (p.m <= kMatvecLdsRows) {
        if (v.waves == 16) group_matvec_kernel<BF, LUT, GPB, 16, 1, true><<<grid, block, 0, s>>>(p);
        else if (v.waves == 8) group_matvec_kernel<BF, LUT, GPB, 8, 1, true><<<grid, block, 0, s>>>(p);
        else group_matvec_kernel<BF, LUT, GPB, 4, 1, true><<<grid, block, 0, s>>>(p);
    } else if (v.row_tiles == 1) {
        if (v.waves == 8) group_matvec_kernel<BF, LUT, GPB, 8, 1, false><<<grid, block, 0, s>>>(p);
        else group_matvec_kernel<BF, LUT, GPB, 4, 1, false><<<grid, block, 0, s>>>(p);
    } else if (v.row_tiles == 2) {
        if (v.waves == 8) group_matvec_kernel<BF, LUT, GPB, 8, 2, false><<<grid, block, 0, s>>>(p);
        else group_matvec_kernel<BF, LUT, GPB, 4, 2, false><<<grid, block, 0, s>>>(p);
    } else {
        group_matvec_kernel<BF, LUT, GPB, 8, 4, false><<<grid, block, 0, s>>>(p);
    }
}
template <bool BF, bool LUT>
static void launch_matvec_type(const MatvecPlan& v, const MatvecParams& p, hipStream_t s) {
    if (p.w.log_group == 7) launch_matvec_groups<BF, LUT, 1>(v, p, s);
    else if (p.w.log_group == 6) launch_matvec_groups<BF, LUT, 2>(v, p, s);
    else launch_matvec_groups<BF, LUT, 4>(v, p, s);
}

hipError_t launch_matvec(bool bf16, const MatvecPlan& plan, MatvecParams p, hipStream_t s) {
    p.splits = plan.splits;
    p.blocks_per_split = plan.blocks_per_split;
    if (p.splits == 1) p.part = nullptr;
    // blocks of X in LDS at a time: m rows of 16 pieces a block, and 4 pieces between rows
    p.chunk = (kMatvecLdsBytes / 16 / p.m - 4) / 16;
    const bool lut = p.w.levels != nullptr;
    if (bf16 && lut) launch_matvec_type<true, true>(plan, p, s);
    if (bf16 && !lut) launch_matvec_type<true, false>(plan, p, s);
    if (!bf16 && lut) launch_matvec_type<false, true>(plan, p, s);
    if (!bf16 && !lut) launch_matvec_type<false, false>(plan, p, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.splits == 1) return e;
    const JoinParams j = {p.part, p.splits, p.m, p.w.n, p.bias, p.Y, p.ldy, bf16 ? KQ_T_BF16 : KQ_T_F16};
    return launch_join(j, s);
}

}  // namespace kq
