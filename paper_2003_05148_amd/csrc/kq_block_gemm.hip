// The products of the 8-bit fully-connected layer on the matrix cores: out[j][i] = sum_c A[i][c] B[j][c], both operands
// rows of e4m3 bytes with one power of two for 128 of them.
//
// A workgroup holds a BI x BJ tile of the output in registers and walks the contraction block by block (128 deep).
// The operands' bytes go from memory to LDS directly, rows of 128 bytes in eight 16-byte chunks, chunk ch of row r
// at ch ^ (r & 7).  i is the contiguous dimension of the output, so that four accumulators of a lane are neighbours
// in memory.  The contraction is in any order that both operands share: lane l of the 32 x 32 x 64 instruction takes
// chunks 2 h' and 2 h' + 1 of its row's half, h' = l / 32.
//
// Two forms.  The scaled 8-bit instruction takes the bytes and both exponents as they are, at twice the 16-bit rate;
// it adds eight products at a time and cuts each off 13 bits below the largest of them.  That is 1.5e-5 of the
// result's norm on random operands, which an output of 16 bits hides (its own rounding is 1.7e-3 or 2.1e-4) and
// one of 32 does not: there the bytes are decoded to bf16 between LDS and the 16-bit instruction, which is exact.
#include "kq_block.h"

namespace kq {

using f32x16 = __attribute__((ext_vector_type(16))) float;
using i32x8 = __attribute__((ext_vector_type(8))) int;

// A step's rows from memory to LDS: a wave's instruction takes 64 chunks, eight rows.
template <int ROWS, int WAVES>
struct DirectRows {
    static constexpr int N = ROWS / 8 / WAVES;
    static_assert(N >= 1 && ROWS % (8 * WAVES) == 0, "pieces");
    unsigned off[N];  // bytes from the tile's first row (of 256 rows and a pitch up to 2^24: below 2^32)
    __device__ __forceinline__ void init(const BlockOperand& o, int64_t row0, int64_t rows, int lane, int wave) {
        const int last = (int)min(rows - 1 - row0, (int64_t)ROWS - 1);  // rows past the last repeat it: not stored
#pragma unroll
        for (int t = 0; t < N; ++t) {
            const int r = (t * WAVES + wave) * 8 + (lane >> 3);
            off[t] = (unsigned)min(r, last) * (unsigned)o.pitch + 16 * ((lane & 7) ^ (r & 7));
        }
    }
    __device__ __forceinline__ void load(const uint8_t* base, u32x4* lds, int wave) const {
#pragma unroll
        for (int t = 0; t < N; ++t)
            __builtin_amdgcn_global_load_lds((global_ptr)(base + off[t]), (lds_ptr)(lds + (t * WAVES + wave) * 64), 16, 0, 0);
    }
};

template <bool EXACT, bool AROWS, int BI, int BJ, int WI, int WJ>
__global__ __launch_bounds__(64 * WI * WJ) void block_gemm_kernel(const BlockGemmParams p) {
    constexpr int MI = BI / WI / 32, MJ = BJ / WJ / 32, WAVES = WI * WJ;
    __shared__ u32x4 s_a0[BI * 8];
    __shared__ u32x4 s_a1[BI * 8];
    __shared__ u32x4 s_b0[BJ * 8];
    __shared__ u32x4 s_b1[BJ * 8];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wi = wave % WI, wj = wave / WI, r32 = lane & 31, half = lane >> 5;
    const int tile = xcd_tile(blockIdx.x, p.itiles * p.jtiles);
    const int64_t i0 = (int64_t)(tile % p.itiles) * BI, j0 = (int64_t)(tile / p.itiles) * BJ;
    const int64_t iw = i0 + wi * MI * 32, jw = j0 + wj * MJ * 32;  // the wave's part

    f32x16 acc[MI][MJ];
#pragma unroll
    for (int a = 0; a < MI; ++a)
#pragma unroll
        for (int b = 0; b < MJ; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[a][b][r] = 0.0f;

    const int s_begin = blockIdx.y * p.steps_per_split, s_end = min(s_begin + p.steps_per_split, p.steps);
    DirectRows<BI, WAVES> la;
    DirectRows<BJ, WAVES> lb;
    la.init(p.A, i0, p.I, lane, wave);
    lb.init(p.B, j0, p.J, lane, wave);
    const uint8_t* const a_base = p.A.v + i0 * p.A.pitch;
    const uint8_t* const b_base = p.B.v + j0 * p.B.pitch;
    const uint8_t* ea[MI];
    const uint8_t* eb[MJ];
#pragma unroll
    for (int a = 0; a < MI; ++a) {
        const int64_t r = min(iw + 32 * a + (AROWS ? r32 : 0), p.I - 1);
        ea[a] = p.A.e + (AROWS ? r : r >> 7) * p.A.e_row;
    }
#pragma unroll
    for (int b = 0; b < MJ; ++b) eb[b] = p.B.e + min(jw + 32 * b + r32, p.J - 1) * p.B.e_row;

    auto step = [&](int s, const u32x4* a_now, u32x4* a_next, const u32x4* b_now, u32x4* b_next) {
        unsigned xa[MI], xb[MJ];
#pragma unroll
        for (int a = 0; a < MI; ++a) xa[a] = ea[a][s * p.A.e_col];
#pragma unroll
        for (int b = 0; b < MJ; ++b) xb[b] = eb[b][s * p.B.e_col];
        if (s + 1 < s_end) {
            la.load(a_base + (int64_t)(s + 1) * kBlock, a_next, wave);
            lb.load(b_base + (int64_t)(s + 1) * kBlock, b_next, wave);
        }
        const u32x4* a_rows = a_now + (wi * MI * 32 + r32) * 8;
        const u32x4* b_rows = b_now + (wj * MJ * 32 + r32) * 8;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int c0 = (4 * h + 2 * half) ^ (r32 & 7), c1 = (4 * h + 2 * half + 1) ^ (r32 & 7);
            if constexpr (!EXACT) {
                i32x8 af[MI], bf[MJ];
                auto fragment = [&](const u32x4* rows) {
                    const u32x4 lo = rows[c0], hi = rows[c1];
                    return i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
                };
#pragma unroll
                for (int a = 0; a < MI; ++a) af[a] = fragment(a_rows + a * 256);
#pragma unroll
                for (int b = 0; b < MJ; ++b) bf[b] = fragment(b_rows + b * 256);
#pragma unroll
                for (int a = 0; a < MI; ++a)
#pragma unroll
                    for (int b = 0; b < MJ; ++b)
                        acc[a][b] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(af[a], bf[b], acc[a][b], 0, 0, 0, (int)xa[a], 0, (int)xb[b]);
            } else {
#pragma unroll
                for (int q = 0; q < 2; ++q) {  // a chunk is two instructions' worth
                    u32x4 ac[MI], bc[MJ];
#pragma unroll
                    for (int a = 0; a < MI; ++a) ac[a] = a_rows[a * 256 + (q ? c1 : c0)];
#pragma unroll
                    for (int b = 0; b < MJ; ++b) bc[b] = b_rows[b * 256 + (q ? c1 : c0)];
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        bf16x8 ad[MI], bd[MJ];
#pragma unroll
                        for (int a = 0; a < MI; ++a) ad[a] = __builtin_bit_cast(bf16x8, decode8(ac[a][2 * u], ac[a][2 * u + 1], checkpoint_step(xa[a])));
#pragma unroll
                        for (int b = 0; b < MJ; ++b) bd[b] = __builtin_bit_cast(bf16x8, decode8(bc[b][2 * u], bc[b][2 * u + 1], checkpoint_step(xb[b])));
#pragma unroll
                        for (int a = 0; a < MI; ++a)
#pragma unroll
                            for (int b = 0; b < MJ; ++b) acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ad[a], bd[b], acc[a][b], 0, 0, 0);
                    }
                }
            }
        }
        __syncthreads();  // (waits for the direct loads too)
    };
    if (s_begin < s_end) {
        la.load(a_base + (int64_t)s_begin * kBlock, s_a0, wave);
        lb.load(b_base + (int64_t)s_begin * kBlock, s_b0, wave);
        __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
        __syncthreads();
        for (int s = s_begin; s < s_end; s += 2) {
            step(s, s_a0, s_a1, s_b0, s_b1);
            if (s + 1 < s_end) step(s + 1, s_a1, s_a0, s_b1, s_b0);
        }
    }

    // lane holds out[j][i .. i + 3] for j = its column, i = 8 g + 4 half of a 32 x 32 tile
#pragma unroll
    for (int b = 0; b < MJ; ++b) {
        const int64_t j = jw + 32 * b + r32;
        if (j >= p.J) continue;
#pragma unroll
        for (int a = 0; a < MI; ++a)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int64_t i = iw + 32 * a + 8 * g + 4 * half;
                if (i >= p.I) continue;
                float v[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] = acc[a][b][4 * g + r];
                const bool whole = i + 4 <= p.I;
                if (p.bias && !p.part) {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (i + r < p.I) v[r] += p.bias[i + r];
                }
                if (p.part || p.type == KQ_T_F32) {
                    float* o = p.part ? p.part + ((int64_t)blockIdx.y * p.J + j) * p.I + i : (float*)p.out + j * p.ldo + i;
                    if (whole) {
                        __builtin_memcpy(o, v, 16);
                    } else {
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (i + r < p.I) o[r] = v[r];
                    }
                } else {
                    uint16_t* o = (uint16_t*)p.out + j * p.ldo + i;
                    unsigned h[2];
                    if (p.type == KQ_T_BF16) {
                        h[0] = Act<true>::pack(v[0], v[1]);
                        h[1] = Act<true>::pack(v[2], v[3]);
                    } else {
                        h[0] = Act<false>::pack(v[0], v[1]);
                        h[1] = Act<false>::pack(v[2], v[3]);
                    }
                    if (whole) {
                        __builtin_memcpy(o, h, 8);
                    } else {
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (i + r < p.I) o[r] = (uint16_t)(h[r >> 1] >> (16 * (r & 1)));
                    }
                }
            }
    }
}

BlockGemmPlan block_gemm_plan(bool exact, int64_t I, int64_t J, int64_t C) {
    (void)exact;
    BlockGemmPlan g = {};
    const int64_t steps = block_pitch(C) / kBlock;
    g.bi = 128;
    g.bj = J <= 32 ? 32 : 128;
    const int64_t tiles = ceil_div64(I, g.bi) * ceil_div64(J, g.bj);
    int64_t splits = 1;
    while (tiles * splits < 256 && splits * 8 <= steps) splits *= 2;
    g.steps_per_split = (int)(steps ? ceil_div64(steps, splits) : 1);
    g.splits = steps ? (int)ceil_div64(steps, g.steps_per_split) : 1;
    g.part_bytes = g.splits > 1 ? ((size_t)g.splits * (size_t)(I * J) * sizeof(float) + 255) & ~size_t(255) : 0;
    return g;
}

template <bool EXACT, bool AROWS>
static hipError_t launch_tile(const BlockGemmPlan& g, const BlockGemmParams& p, hipStream_t s) {
    const dim3 grid((unsigned)((int64_t)p.itiles * p.jtiles), (unsigned)p.splits);
    const int tile = g.bi * 1000 + g.bj;
    if (tile == 128128) block_gemm_kernel<EXACT, AROWS, 128, 128, 2, 2><<<grid, dim3(256), 0, s>>>(p);
    else if (tile == 128032) block_gemm_kernel<EXACT, AROWS, 128, 32, 4, 1><<<grid, dim3(256), 0, s>>>(p);
    else return hipErrorInvalidValue;
    return hipGetLastError();
}

hipError_t launch_block_gemm(bool exact, bool a_rows, const BlockGemmPlan& plan, BlockGemmParams p, void* part, hipStream_t s) {
    p.itiles = (int)ceil_div64(p.I, plan.bi);
    p.jtiles = (int)ceil_div64(p.J, plan.bj);
    p.splits = plan.splits;
    p.steps_per_split = plan.steps_per_split;
    p.part = plan.splits > 1 ? (float*)part : nullptr;
    hipError_t e;
    if (exact) e = a_rows ? launch_tile<true, true>(plan, p, s) : launch_tile<true, false>(plan, p, s);
    else e = a_rows ? launch_tile<false, true>(plan, p, s) : launch_tile<false, false>(plan, p, s);
    if (e != hipSuccess || plan.splits == 1) return e;
    const JoinParams j = {p.part, p.splits, p.J, p.I, p.bias, p.out, p.ldo, p.type};
    return launch_join(j, s);
}

}  // namespace kq
