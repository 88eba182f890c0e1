// The products of a 4-bit fully-connected layer on the matrix cores.
//
// Every product is out[j][i] = sum_c A[i][c] B[j][c] with i the contiguous dimension of the output, so
// that a lane's four accumulators are neighbours in memory.  A workgroup holds a BI x BJ tile of the output
// in registers and walks the contraction in steps of 64; a step's operands are staged through LDS as
// 16-bit rows of 64 (128 bytes).  What differs between the products is how a step gets there:
//   Linear      A = W from its codes (a row's eight columns are one dword), B = X as it is
//   GradInput   A = W^T: eight rows' dwords of one thread are an 8 x 8 block, written transposed; B = dY
//   GradWeight  A = X^^T from the checkpoint (8 rows x 4 columns a thread), B = dY^T (8 x 4 a thread)
//   GradScales  the same product; the epilogue multiplies it by the levels and adds up each group
// Weights are s * level rounded once to the activation's type (bf16: s has 8 bits and -8..7 three, so
// about half of them are exact); checkpoints and activations are exact, sums are fp32.
#include "kq_group.h"

namespace kq {

constexpr int kStep = 64;  // contraction per step

// LDS rows of 128 bytes in eight 16-byte chunks; chunk ch of row r lies at ch ^ swizzle(r).  Eight
// consecutive rows of one chunk (fragment reads), rows 4 l + t (transposed writes of four columns) and rows
// 8 d + 2 t + par (transposed writes of a dword's even or odd columns) all fall on eight different chunks.
__device__ __forceinline__ int swizzle(int r) { return (r ^ (r >> 2)) & 7; }
__device__ __forceinline__ int lds_chunk(int r, int ch) { return r * 8 + (ch ^ swizzle(r)); }

// four level values (fp32) of the codes at nibbles 0..3 of w >> shift
template <bool BF, bool LUT, int MODE, int BI, int BJ, int WI, int WJ>
struct Gemm {
    static constexpr int NT = 64 * WI * WJ;
    static constexpr int MI = BI / WI / 16, MJ = BJ / WJ / 16;  // 16 x 16 tiles of a wave
    static constexpr bool kWeightRows = MODE == (int)Product::Linear;
    static constexpr bool kWeightCols = MODE == (int)Product::GradInput;
    static constexpr bool kCheckpoint = MODE >= (int)Product::GradWeight;

    using A_ = Act<BF>;

    // ---- A ----
    static constexpr int kATasks = kWeightRows ? BI * 4 : BI * 2;
    static constexpr int PA = kATasks / NT;
    static_assert(kATasks % NT == 0 && PA >= 1, "A tasks");
    struct StageA {
        unsigned w[PA][kWeightRows ? 2 : 8];
        unsigned short s[PA][kWeightRows ? 2 : 8];  // scales (bf16 bits) or checkpoint exponents
    };
    // ---- B ----
    static constexpr int kBTasks = kCheckpoint ? BJ * 2 : BJ * 8;
    static constexpr int PB = kBTasks / NT;
    static_assert(kBTasks % NT == 0 && PB >= 1, "B tasks");
    struct StageB {
        unsigned v[PB][kCheckpoint ? 16 : 4];
    };

    static __device__ __forceinline__ void load_a(const GemmParams& p, int i0, int c, int tid, StageA& st) {
#pragma unroll
        for (int t = 0; t < PA; ++t) {
            const int id = t * NT + tid;
            if constexpr (kWeightRows) {
                const int r = id >> 2, q = id & 3, n = i0 + r;
                const int i = (c & 127) >> 5;  // 0 or 2: the half of the tile
                const bool in = (n >> 4) < p.w.ntiles;
                const uint8_t* at = p.w.codes + ((int64_t)(n >> 4) * p.w.ktiles + (c >> 7)) * kTileBytes + (n & 15) * 64 + q * 16 + i * 4;
                u32x2 d = {0, 0};
                if (in) d = *(const u32x2*)at;
                st.w[t][0] = d.x;
                st.w[t][1] = d.y;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    int g = (c + 32 * h) >> p.w.log_group;
                    g = g < p.w.groups ? g : p.w.groups - 1;
                    st.s[t][h] = n < p.w.n ? p.w.scales[(int64_t)n * p.w.groups + g] : (unsigned short)0;
                }
            } else if constexpr (kWeightCols) {
                const int par = id & 1, d = (id >> 1) % (BI / 8), oct = (id >> 1) / (BI / 8);
                const int k = i0 + 8 * d, n = c + 8 * oct;
                const int kk = k & 127, dw = ((kk >> 3) & 3) * 4 + (kk >> 5);
                const bool in = (n >> 4) < p.w.ntiles && (k >> 7) < p.w.ktiles;
                const uint8_t* at = p.w.codes + ((int64_t)(n >> 4) * p.w.ktiles + (k >> 7)) * kTileBytes + (n & 15) * 64 + dw * 4;
                int g = k >> p.w.log_group;
                g = g < p.w.groups ? g : p.w.groups - 1;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    st.w[t][e] = in ? (*(const unsigned*)(at + e * 64)) >> (16 * par) : 0u;
                    st.s[t][e] = n + e < p.w.n ? p.w.scales[(int64_t)(n + e) * p.w.groups + g] : (unsigned short)0;
                }
            } else {
                const int kq4 = id % (BI / 4), oct = id / (BI / 4);
                const int k = i0 + 4 * kq4;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int64_t m = (int64_t)c + 8 * oct + e;
                    const bool in = m < p.C && k < p.kq;
                    st.w[t][e] = in ? *(const unsigned*)(p.q + m * p.kq + k) : 0u;
                    st.s[t][e] = in ? (unsigned short)p.exps[m * (p.kq >> 5) + (k >> 5)] : (unsigned short)0;
                }
            }
        }
    }

    static __device__ __forceinline__ float level(unsigned code, const float* s_level) {
        if constexpr (LUT) return s_level[code];
        else return (float)((int)code - 8);
    }

    static __device__ __forceinline__ void store_a(u32x4* lds, int tid, const StageA& st, const float* s_level) {
#pragma unroll
        for (int t = 0; t < PA; ++t) {
            const int id = t * NT + tid;
            if constexpr (kWeightRows) {
                const int r = id >> 2, q = id & 3;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float s = bf16_bits_to_f32(st.s[t][h]);
                    const unsigned w = st.w[t][h];
                    u32x4 o;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        o[j] = A_::pack(s * level((w >> (4 * j)) & 15u, s_level), s * level((w >> (16 + 4 * j)) & 15u, s_level));
                    lds[lds_chunk(r, 4 * h + q)] = o;
                }
            } else if constexpr (kWeightCols) {
                const int par = id & 1, d = (id >> 1) % (BI / 8), oct = (id >> 1) / (BI / 8);
                float s[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) s[e] = bf16_bits_to_f32(st.s[t][e]);
#pragma unroll
                for (int j = 0; j < 4; ++j) {  // column 8 d + 2 j + par
                    u32x4 o;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        o[e] = A_::pack(s[2 * e] * level((st.w[t][2 * e] >> (4 * j)) & 15u, s_level),
                                        s[2 * e + 1] * level((st.w[t][2 * e + 1] >> (4 * j)) & 15u, s_level));
                    lds[lds_chunk(8 * d + 2 * j + par, oct)] = o;
                }
            } else {
                const int kq4 = id % (BI / 4), oct = id / (BI / 4);
                float s[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) s[e] = __builtin_bit_cast(float, st.s[t][e] == 255 ? 0x7fc00000u : (unsigned)st.s[t][e] << 23);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    u32x4 o;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        o[e] = A_::pack_exact(s[2 * e] * (float)((int)(st.w[t][2 * e] << (24 - 8 * j)) >> 24),
                                              s[2 * e + 1] * (float)((int)(st.w[t][2 * e + 1] << (24 - 8 * j)) >> 24));
                    lds[lds_chunk(4 * kq4 + j, oct)] = o;
                }
            }
        }
    }

    static __device__ __forceinline__ void load_b(const GemmParams& p, int j0, int c, int tid, StageB& st) {
#pragma unroll
        for (int t = 0; t < PB; ++t) {
            const int id = t * NT + tid;
            if constexpr (!kCheckpoint) {  // rows j, 8 neighbours along c
                const int r = id >> 3, ch = id & 7, c0 = c + 8 * ch;
                const bool in = j0 + r < p.J;
                const uint16_t* at = (const uint16_t*)p.B + (in ? (int64_t)(j0 + r) * p.ldb : 0) + c0;
                if (in && c0 + 8 <= p.C) {
                    __builtin_memcpy(st.v[t], at, 16);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const unsigned lo = in && c0 + 2 * e < p.C ? at[2 * e] : 0u;
                        const unsigned hi = in && c0 + 2 * e + 1 < p.C ? at[2 * e + 1] : 0u;
                        st.v[t][e] = lo | (hi << 16);
                    }
                }
            } else {  // rows along c, four neighbours along j
                const int n4 = id % (BJ / 4), oct = id / (BJ / 4);
                const int n = j0 + 4 * n4;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int64_t m = (int64_t)c + 8 * oct + e;
                    const bool in = m < p.C;
                    const uint16_t* at = (const uint16_t*)p.B + (in ? m * p.ldb : 0) + n;
                    if (in && n + 4 <= p.J) {
                        __builtin_memcpy(&st.v[t][2 * e], at, 8);
                    } else {
                        unsigned h[4];
#pragma unroll
                        for (int f = 0; f < 4; ++f) h[f] = in && n + f < p.J ? at[f] : 0u;
                        st.v[t][2 * e] = h[0] | (h[1] << 16);
                        st.v[t][2 * e + 1] = h[2] | (h[3] << 16);
                    }
                }
            }
        }
    }

    static __device__ __forceinline__ void store_b(u32x4* lds, int tid, const StageB& st) {
#pragma unroll
        for (int t = 0; t < PB; ++t) {
            const int id = t * NT + tid;
            if constexpr (!kCheckpoint) {
                const int r = id >> 3, ch = id & 7;
                lds[lds_chunk(r, ch)] = u32x4{st.v[t][0], st.v[t][1], st.v[t][2], st.v[t][3]};
            } else {
                const int n4 = id % (BJ / 4), oct = id / (BJ / 4);
#pragma unroll
                for (int f = 0; f < 4; ++f) {
                    u32x4 o;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        o[e] = __builtin_amdgcn_perm(st.v[t][2 * (2 * e + 1) + (f >> 1)], st.v[t][2 * (2 * e) + (f >> 1)],
                                                     (f & 1) ? 0x07060302u : 0x05040100u);
                    lds[lds_chunk(4 * n4 + f, oct)] = o;
                }
            }
        }
    }
};

template <bool BF, bool LUT, int MODE, int BI, int BJ, int WI, int WJ>
__global__ __launch_bounds__(64 * WI * WJ) void group_gemm_kernel(const GemmParams p) {
    using G = Gemm<BF, LUT, MODE, BI, BJ, WI, WJ>;
    constexpr int MI = G::MI, MJ = G::MJ;
    __shared__ u32x4 s_a[BI * 8];
    __shared__ u32x4 s_b[BJ * 8];
    __shared__ float s_level[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wi = wave % WI, wj = wave / WI;
    const int it = blockIdx.x % p.itiles, jt = blockIdx.x / p.itiles;
    const int i0 = it * BI, j0 = jt * BJ;
    if (LUT && tid < 16) s_level[tid] = bf16_bits_to_f32(p.w.levels[tid]);
    __syncthreads();

    f32x4 acc[MI][MJ];
#pragma unroll
    for (int a = 0; a < MI; ++a)
#pragma unroll
        for (int b = 0; b < MJ; ++b) acc[a][b] = f32x4{0, 0, 0, 0};

    const int64_t c_begin = (int64_t)blockIdx.y * p.steps_per_split * kStep;
    int64_t c_end = c_begin + (int64_t)p.steps_per_split * kStep;
    if (c_end > p.C) c_end = p.C;
    typename G::StageA sa;
    typename G::StageB sb;
    for (int64_t c = c_begin; c < c_end; c += kStep) {
        G::load_a(p, i0, (int)c, tid, sa);
        G::load_b(p, j0, (int)c, tid, sb);
        __syncthreads();
        G::store_a(s_a, tid, sa, s_level);
        G::store_b(s_b, tid, sb);
        __syncthreads();
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            u32x4 af[MI], bf[MJ];
#pragma unroll
            for (int a = 0; a < MI; ++a) af[a] = s_a[lds_chunk((wi * MI + a) * 16 + (lane & 15), kk * 4 + (lane >> 4))];
#pragma unroll
            for (int b = 0; b < MJ; ++b) bf[b] = s_b[lds_chunk((wj * MJ + b) * 16 + (lane & 15), kk * 4 + (lane >> 4))];
#pragma unroll
            for (int a = 0; a < MI; ++a)
#pragma unroll
                for (int b = 0; b < MJ; ++b) acc[a][b] = Act<BF>::mfma(af[a], bf[b], acc[a][b]);
        }
    }

    // lane holds out[j][i .. i + 3], j = its column of the 16 x 16 tile
    const int jl = j0 + wj * MJ * 16 + (lane & 15), il = i0 + wi * MI * 16 + 4 * (lane >> 4);
    if constexpr (MODE == (int)Product::GradScales) {
        static_assert(BI / WI == 128, "a wave holds whole groups");
#pragma unroll
        for (int b = 0; b < MJ; ++b) {
            const int n = jl + 16 * b;
            const bool live = n < p.w.n;
            float sum[MI / 2];  // per 32 columns
#pragma unroll
            for (int a = 0; a < MI; ++a) {
                const int k = il + 16 * a, kk = k & 127;
                unsigned d = 0;
                if (live && (k >> 7) < p.w.ktiles)
                    d = *(const unsigned*)(p.w.codes + ((int64_t)(n >> 4) * p.w.ktiles + (k >> 7)) * kTileBytes + (n & 15) * 64 + ((kk >> 3) & 3) * 16 + (kk >> 5) * 4);
                const int half = (kk >> 2) & 1;
                float v = 0.0f;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const unsigned code = (d >> (4 * ((r & 1) * 4 + 2 * half + (r >> 1)))) & 15u;
                    // columns past the matrix: the checkpoint is zero there
                    v = __builtin_fmaf(G::level(code, s_level), acc[a][b][r], v);
                }
                if (a & 1) sum[a >> 1] += v;
                else sum[a >> 1] = v;
            }
            if (p.w.log_group >= 6) {
#pragma unroll
                for (int h = 0; h < MI / 2; h += 2) sum[h] += sum[h + 1];
            }
            if (p.w.log_group >= 7) {
#pragma unroll
                for (int h = 0; h < MI / 2; h += 4) sum[h] += sum[h + 2];
            }
            const int i_wave = i0 + wi * MI * 16;
            float* out = p.part ? p.part + (int64_t)blockIdx.y * p.w.n * p.w.groups : (float*)p.out;
#pragma unroll
            for (int h = 0; h < MI / 2; ++h) {
                float v = sum[h];
                v += __shfl_xor(v, 16);
                v += __shfl_xor(v, 32);
                const int k = i_wave + 32 * h;
                if (lane < 16 && live && k < p.w.k && (k & ((1 << p.w.log_group) - 1)) == 0)
                    out[(int64_t)n * p.w.groups + (k >> p.w.log_group)] = v;
            }
        }
    } else {
#pragma unroll
        for (int b = 0; b < MJ; ++b) {
            const int j = jl + 16 * b;
            if (j >= p.J) continue;
#pragma unroll
            for (int a = 0; a < MI; ++a) {
                const int i = il + 16 * a;
                if (i >= p.I) continue;
                f32x4 v = acc[a][b];
                const bool whole = i + 4 <= p.I;
                if (MODE == (int)Product::GradWeight || p.part != nullptr) {
                    float* o = p.part ? p.part + ((int64_t)blockIdx.y * p.J + j) * p.I + i : (float*)p.out + (int64_t)j * p.ldo + i;
                    if (whole) {
                        __builtin_memcpy(o, &v, 16);
                    } else {
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (i + r < p.I) o[r] = v[r];
                    }
                } else {
                    if (MODE == (int)Product::Linear && p.bias) {
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (i + r < p.I) v[r] += p.bias[i + r];
                    }
                    uint16_t* o = (uint16_t*)p.out + (int64_t)j * p.ldo + i;
                    unsigned h[2] = {Act<BF>::pack(v[0], v[1]), Act<BF>::pack(v[2], v[3])};
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
}

GemmPlan gemm_plan(Product mode, int64_t I, int64_t J, int64_t C, int groups) {
    GemmPlan g;
    g.bi = 128;
    g.bj = 128;
    g.splits = 1;
    g.steps_per_split = (int)ceil_div64(C, kStep);
    g.ws_bytes = 0;
    return g;
}

template <int MODE, int BI, int BJ, int WI, int WJ>
static hipError_t launch_tile(bool bf16, const GemmParams& p, hipStream_t s) {
    const dim3 grid((unsigned)((int64_t)p.itiles * p.jtiles), (unsigned)p.splits), block(64 * WI * WJ);
    const bool lut = MODE != (int)Product::GradWeight && p.w.levels != nullptr;
    if constexpr (MODE != (int)Product::GradWeight) {
        if (lut && bf16) group_gemm_kernel<true, true, MODE, BI, BJ, WI, WJ><<<grid, block, 0, s>>>(p);
        if (lut && !bf16) group_gemm_kernel<false, true, MODE, BI, BJ, WI, WJ><<<grid, block, 0, s>>>(p);
    }
    if (!lut && bf16) group_gemm_kernel<true, false, MODE, BI, BJ, WI, WJ><<<grid, block, 0, s>>>(p);
    if (!lut && !bf16) group_gemm_kernel<false, false, MODE, BI, BJ, WI, WJ><<<grid, block, 0, s>>>(p);
    return hipGetLastError();
}

hipError_t launch_gemm(Product mode, bool bf16, const GemmPlan& plan, GemmParams p, hipStream_t s) {
    p.itiles = (int)ceil_div64(p.I, plan.bi);
    p.jtiles = (int)ceil_div64(p.J, plan.bj);
    p.splits = plan.splits;
    p.steps_per_split = plan.steps_per_split;
    switch (mode) {
        case Product::Linear: return launch_tile<0, 128, 128, 2, 2>(bf16, p, s);
        case Product::GradInput: return launch_tile<1, 128, 128, 2, 2>(bf16, p, s);
        case Product::GradWeight: return launch_tile<2, 128, 128, 1, 4>(bf16, p, s);
        default: return launch_tile<3, 128, 128, 1, 4>(bf16, p, s);
    }
}

}  // namespace kq
