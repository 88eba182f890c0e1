// Y = X W^T for few rows of X (one token, a small batch): a stream of the packed codes past the matrix
// cores.
//
// A wave multiplies 16 rows of W by 16 rows of X, 128 columns at a time: 16 bytes of codes a lane are one
// contiguous kilobyte and four operands of the 16 x 16 x 32 matrix instruction, so the codes go from memory
// to the matrix cores through registers alone.  A code q becomes 16 + q in one shift and one masked OR a pair
// (the four bits are the top of the mantissa of 16); a product of X with the constant -24 starts the
// accumulator, and so the sum is that of x (q - 8).  Tables of levels are looked up with byte permutes.
// Every product is exact; a group's fp32 sum takes the group's scale in fp32.
// The waves of a workgroup take the 128-column blocks of its rows in turn and add their sums through LDS in
// order.  Where there are few rows of W the columns are also split over workgroups, joined by a second kernel.
#include "kq_group.h"

namespace kq {

// ---- codes to 16-bit values -------------------------------------------------------------------------------

template <bool BF>
__device__ __forceinline__ LevelTable load_levels(const uint16_t* levels) {
    LevelTable t;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        unsigned a, b;  // levels 4 r .. 4 r + 3 in two registers
        if constexpr (BF) {
            a = (unsigned)levels[4 * r] | (unsigned)levels[4 * r + 1] << 16;
            b = (unsigned)levels[4 * r + 2] | (unsigned)levels[4 * r + 3] << 16;
        } else {  // fp16 holds a bf16 level exactly from 2^-14 on, and to 2^-25 below
            a = Act<false>::pack(bf16_bits_to_f32(levels[4 * r]), bf16_bits_to_f32(levels[4 * r + 1]));
            b = Act<false>::pack(bf16_bits_to_f32(levels[4 * r + 2]), bf16_bits_to_f32(levels[4 * r + 3]));
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

// the 8 columns of a dword of codes, in order: levels, or 16 + q without a table
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
        o[0] = ((d << 3) & 0x00780078u) | 0x41804180u;
        o[1] = ((d >> 1) & 0x00780078u) | 0x41804180u;
        o[2] = ((d >> 5) & 0x00780078u) | 0x41804180u;
        o[3] = ((d >> 9) & 0x00780078u) | 0x41804180u;
    } else {
        o[0] = ((d << 6) & 0x03c003c0u) | 0x4c004c00u;
        o[1] = ((d << 2) & 0x03c003c0u) | 0x4c004c00u;
        o[2] = ((d >> 2) & 0x03c003c0u) | 0x4c004c00u;
        o[3] = ((d >> 6) & 0x03c003c0u) | 0x4c004c00u;
    }
    return o;
}

// 8 neighbours of a row of X from column c, zeros from `limit` on
__device__ __forceinline__ u32x4 load_x(const uint16_t* row, int c, int limit) {
    u32x4 v;
    if (c + 8 <= limit) {
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

// MT: 16-row tiles of X.  XLDS: X (at most kMatvecLdsRows rows) is staged through LDS in chunks of
// p.chunk blocks; otherwise its fragments are loaded from the caches.
template <bool BF, bool LUT, int MT, int WAVES, int U, bool XLDS>
__global__ __launch_bounds__(64 * WAVES) void group_matvec_kernel(const MatvecParams p) {
    constexpr int kSumBytes = WAVES * MT * 64 * 16;
    constexpr int kXBytes = XLDS ? kMatvecLdsBytes : 0;
    __shared__ u32x4 s_buf[(kSumBytes > kXBytes ? kSumBytes : kXBytes) / 16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r16 = lane & 15, q = lane >> 4;
    const int nt = blockIdx.x;
    const int n = nt * kTileRows + r16;
    const int k_begin = blockIdx.y * p.blocks_per_split;
    const int k_end = min(k_begin + p.blocks_per_split, p.w.ktiles);
    const uint8_t* codes = p.w.codes + (int64_t)nt * p.w.ktiles * kTileBytes + r16 * 64 + q * 16;
    const uint16_t* scales = p.w.scales + (int64_t)min(n, p.w.n - 1) * p.w.groups;
    const int gpb = kTileCols >> p.w.log_group;  // groups a block: 1, 2 or 4

    LevelTable table;
    if constexpr (LUT) table = load_levels<BF>(p.w.levels);
    const unsigned offset_bits = BF ? 0xc1c0c1c0u : 0xce00ce00u;  // a pair of -24
    const u32x4 offset = {offset_bits, offset_bits, offset_bits, offset_bits};

    const uint16_t* xrow[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) xrow[t] = (const uint16_t*)p.X + (int64_t)min(16 * t + r16, p.m - 1) * p.ldx;

    f32x4 y[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) y[t] = f32x4{0, 0, 0, 0};

    const int chunk = XLDS ? p.chunk : k_end - k_begin;
    const int pitch = chunk * 16 + 4;  // 16-byte pieces of a staged row: rows 64 bytes apart in the banks
    for (int c0 = k_begin; c0 < k_end; c0 += chunk) {
        const int c1 = min(c0 + chunk, k_end);
        u32x4 next[U];
        unsigned short ns[U][4];
        auto fetch = [&](int kb) {  // blocks kb, kb + WAVES, ...
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int b = min(kb + u * WAVES, p.w.ktiles - 1);
                next[u] = *(const u32x4*)(codes + (int64_t)b * kTileBytes);
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    if (g < gpb) ns[u][g] = scales[min(b * gpb + g, p.w.groups - 1)];
            }
        };
        fetch(c0 + wave);
        if constexpr (XLDS) {
            __syncthreads();  // the previous chunk is read
            const int pieces = (c1 - c0) * 16;
            for (int id = threadIdx.x; id < p.m * pieces; id += 64 * WAVES) {
                const int r = id / pieces, ch = id - r * pieces;
                s_buf[r * pitch + ch] = load_x((const uint16_t*)p.X + (int64_t)r * p.ldx, c0 * kTileCols + ch * 8, p.w.k);
            }
            __syncthreads();
        }
        for (int kb = c0 + wave; kb < c1; kb += U * WAVES) {
            u32x4 cur[U];
            unsigned short cs[U][4];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                cur[u] = next[u];
#pragma unroll
                for (int g = 0; g < 4; ++g) cs[u][g] = ns[u][g];
            }
            if (kb + U * WAVES < c1) fetch(kb + U * WAVES);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int b = kb + u * WAVES;
                if (b < c1) {
                    f32x4 acc[MT];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const u32x4 w = decode<BF, LUT>(cur[u][i], table);
                        const int col = b * kTileCols + 32 * i + 8 * q;
                        const bool first = (i & ((1 << (p.w.log_group - 5)) - 1)) == 0;
#pragma unroll
                        for (int t = 0; t < MT; ++t) {
                            u32x4 x;
                            if constexpr (XLDS) x = s_buf[min(r16, p.m - 1) * pitch + (b - c0) * 16 + 4 * i + q];
                            else x = load_x(xrow[t], col, p.w.k);
                            if (first) acc[t] = f32x4{0, 0, 0, 0};
                            if constexpr (!LUT) acc[t] = Act<BF>::mfma(x, offset, acc[t]);
                            acc[t] = Act<BF>::mfma(x, w, acc[t]);
                        }
                        if (((i + 1) & ((1 << (p.w.log_group - 5)) - 1)) == 0) {
                            const int g = i >> (p.w.log_group - 5);
                            const float s = bf16_bits_to_f32(g == 0 ? cs[u][0] : g == 1 ? cs[u][1] : g == 2 ? cs[u][2] : cs[u][3]);
#pragma unroll
                            for (int t = 0; t < MT; ++t)
#pragma unroll
                                for (int r = 0; r < 4; ++r) y[t][r] = __builtin_fmaf(s, acc[t][r], y[t][r]);
                        }
                    }
                }
            }
        }
    }

    // lane holds Y[16 t + 4 q + r][n]: the waves' sums in order
    if constexpr (XLDS) __syncthreads();
    f32x4* s_sum = (f32x4*)s_buf;
#pragma unroll
    for (int t = 0; t < MT; ++t) s_sum[(t * WAVES + wave) * 64 + lane] = y[t];
    __syncthreads();
    for (int t = wave; t < MT; t += WAVES) {
        f32x4 v = s_sum[t * WAVES * 64 + lane];
        for (int w = 1; w < WAVES; ++w) v += s_sum[(t * WAVES + w) * 64 + lane];
        if (n < p.w.n) {
            const float bias = p.bias && !p.part ? p.bias[n] : 0.0f;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int m = 16 * t + 4 * q + r;
                if (m < p.m) {
                    if (p.part) p.part[((int64_t)blockIdx.y * p.m + m) * p.w.n + n] = v[r];
                    else ((uint16_t*)p.Y)[(int64_t)m * p.ldy + n] = Act<BF>::one(v[r] + bias);
                }
            }
        }
    }
}

MatvecPlan matvec_plan(int m, int64_t n, int64_t k) {
    MatvecPlan v = {};
    v.splits = 1;
    v.blocks_per_split = (int)ceil_div64(k, kTileCols);
    v.ws_bytes = 0;
    return v;
}

template <bool BF, bool LUT>
static void launch_matvec_type(const MatvecParams& p, hipStream_t s) {
    const dim3 grid((unsigned)p.w.ntiles, (unsigned)p.splits);
    if (p.m <= kMatvecLdsRows) group_matvec_kernel<BF, LUT, 1, 8, 4, true><<<grid, 512, 0, s>>>(p);
    else group_matvec_kernel<BF, LUT, 1, 8, 4, false><<<grid, 512, 0, s>>>(p);
}

hipError_t launch_matvec(bool bf16, const MatvecPlan& plan, MatvecParams p, hipStream_t s) {
    p.splits = plan.splits;
    p.blocks_per_split = plan.blocks_per_split;
    // blocks of X in LDS at a time: m rows of 16 pieces a block, and 4 pieces between rows
    p.chunk = (kMatvecLdsBytes / 16 / p.m - 4) / 16;
    const bool lut = p.w.levels != nullptr;
    if (bf16 && lut) launch_matvec_type<true, true>(p, s);
    if (bf16 && !lut) launch_matvec_type<true, false>(p, s);
    if (!bf16 && lut) launch_matvec_type<false, true>(p, s);
    if (!bf16 && !lut) launch_matvec_type<false, false>(p, s);
    return hipGetLastError();
}

}  // namespace kq
