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

// The bytes of four codes, 0..15 each, as fp32 s * level.
template <bool LUT>
struct Levels;
template <>
struct Levels<false> {
    __device__ __forceinline__ void init(const uint16_t*) {}
    // levels -8 .. 7: s * (q - 8) = fma(q, s, -8 s), exact
    static __device__ __forceinline__ void scaled(const Levels&, unsigned b, const float (&s)[4], float (&v)[4]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = __builtin_fmaf((float)((b >> (8 * j)) & 255u), s[j], -8.0f * s[j]);
    }
    static __device__ __forceinline__ void plain(const Levels&, unsigned b, float (&v)[4]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = (float)((b >> (8 * j)) & 255u) - 8.0f;
    }
};
template <>
struct Levels<true> {
    LevelTable t;  // bf16 levels by bytes
    __device__ __forceinline__ void init(const uint16_t* levels) { t = load_levels<true>(levels); }
    static __device__ __forceinline__ void plain(const Levels& l, unsigned b, float (&v)[4]) {
        const unsigned low3 = b & 0x07070707u, pick = ((b >> 1) & 0x04040404u) | 0x03020100u;
        const unsigned lo = look_up(l.t.lo, low3, pick), hi = look_up(l.t.hi, low3, pick);
        // byte j of lo and hi to the top half of a register
        v[0] = __builtin_bit_cast(float, __builtin_amdgcn_perm(hi, lo, 0x04000c0cu));
        v[1] = __builtin_bit_cast(float, __builtin_amdgcn_perm(hi, lo, 0x05010c0cu));
        v[2] = __builtin_bit_cast(float, __builtin_amdgcn_perm(hi, lo, 0x06020c0cu));
        v[3] = __builtin_bit_cast(float, __builtin_amdgcn_perm(hi, lo, 0x07030c0cu));
    }
    static __device__ __forceinline__ void scaled(const Levels& l, unsigned b, const float (&s)[4], float (&v)[4]) {
        plain(l, b, v);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] *= s[j];
    }
};

template <bool BF, bool LUT, int MODE, int BI, int BJ, int WI, int WJ>
struct Gemm {
    static constexpr int NT = 64 * WI * WJ;
    static constexpr int MI = BI / WI / 16, MJ = BJ / WJ / 16;  // 16 x 16 tiles of a wave
    static constexpr bool kWeightRows = MODE == (int)Product::Linear;
    static constexpr bool kWeightCols = MODE == (int)Product::GradInput;
    static constexpr bool kCheckpoint = MODE >= (int)Product::GradWeight;
    using A_ = Act<BF>;
    using L = Levels<LUT>;

    // Pieces of a step that a thread stages: A and B tasks.  Rows past the output's edges repeat the last
    // one (what they give is not stored); the contraction's edge is zero on both sides.
    static constexpr int kATasks = kWeightRows ? BI * 4 : BI * 2;
    static constexpr int PA = kATasks / NT;
    static_assert(kATasks % NT == 0 && PA >= 1, "A tasks");
    static constexpr int kBTasks = kCheckpoint ? BJ * 2 : BJ * 8;
    static constexpr int PB = kBTasks / NT;
    static_assert(kBTasks % NT == 0 && PB >= 1, "B tasks");

    unsigned aw[PA][kWeightRows ? 2 : 8];
    unsigned short as[PA][kWeightRows ? 2 : 8];  // scales (bf16 bits) or checkpoint exponents
    unsigned bv[PB][kCheckpoint ? 16 : 4];

    // Which rows of the contraction a thread's transposed tasks take: octet t * kOctets + ...; with 256
    // rows of output a wave has one octet, and its row addresses are scalar.
    template <int B>
    static __device__ __forceinline__ int octet(int t, int tid, int wave) {
        if constexpr (B == 256) return t * (NT / 64) + wave;
        else return (t * NT + tid) / (B / 4);
    }
    template <class T>
    static __device__ __forceinline__ T at(const void* base, unsigned off) {
        return *(const T*)((const char*)base + off);
    }

    __device__ __forceinline__ void load_a(const GemmParams& p, int i0, int c, int tid, int wave) {
        const bool full = c + kStep <= p.C;
#pragma unroll
        for (int t = 0; t < PA; ++t) {
            const int id = t * NT + tid;
            if constexpr (kWeightRows) {  // row of W, 8 bytes: two runs of 8 columns, 32 apart
                const int r = min(id >> 2, p.w.n - 1 - i0), q = id & 3;
                const uint8_t* base = p.w.codes + ((int64_t)(i0 >> 4) * p.w.ktiles + (c >> 7)) * kTileBytes + ((c & 64) >> 3);
                const u32x2 d = at<u32x2>(base, (unsigned)(r >> 4) * (unsigned)p.w.ktiles * kTileBytes + (r & 15) * 64 + q * 16);
                aw[t][0] = d.x;
                aw[t][1] = d.y;
                const uint16_t* sc = p.w.scales + (int64_t)i0 * p.w.groups;
                const unsigned row = (unsigned)r * (unsigned)p.w.groups;
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    as[t][h] = at<unsigned short>(sc + min((c + 32 * h) >> p.w.log_group, p.w.groups - 1), 2 * row);
            } else if constexpr (kWeightCols) {  // 8 rows, one dword: the even or the odd half of 8 columns
                const int oct = octet<BI>(t, tid, wave), d = (id >> 1) % (BI / 8);
                const int k = min(i0 + 8 * d, p.w.k - 1), n = c + 8 * oct;
                const int kk = k & 127, dw = ((kk >> 3) & 3) * 4 + (kk >> 5);
                const uint8_t* base = p.w.codes + (int64_t)min(n >> 4, p.w.ntiles - 1) * p.w.ktiles * kTileBytes + (n & 15) * 64;
                const unsigned col = (unsigned)(k >> 7) * kTileBytes + dw * 4, g = 2 * (unsigned)(k >> p.w.log_group);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    aw[t][e] = at<unsigned>(base + e * 64, col);
                    as[t][e] = at<unsigned short>(p.w.scales + (int64_t)min(n + e, p.w.n - 1) * p.w.groups, g);
                    if (!full && n + e >= p.w.n) as[t][e] = 0;
                }
            } else {  // 8 rows of the checkpoint, 4 columns
                const int oct = octet<BI>(t, tid, wave), quad = id % (BI / 4);
                const unsigned k = min(i0 + 4 * quad, p.kq - 4);
                const int m = c + 8 * oct;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int64_t row = full ? m + e : min(m + e, (int)p.C - 1);
                    aw[t][e] = at<unsigned>(p.q + row * p.kq, k);
                    as[t][e] = at<uint8_t>(p.exps + row * (p.kq >> 5), k >> 5);
                    if (!full && m + e >= p.C) as[t][e] = 0;
                }
            }
        }
    }

    __device__ __forceinline__ void store_a(u32x4* lds, int tid, int wave, const L& lv) const {
#pragma unroll
        for (int t = 0; t < PA; ++t) {
            const int id = t * NT + tid;
            if constexpr (kWeightRows) {
                const int r = id >> 2, q = id & 3;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float s1 = bf16_bits_to_f32(as[t][h]);
                    const float s[4] = {s1, s1, s1, s1};
                    float e[4], o[4];  // nibbles 0 2 4 6 are columns 0 4 1 5, nibbles 1 3 5 7 columns 2 6 3 7
                    L::scaled(lv, aw[t][h] & 0x0f0f0f0fu, s, e);
                    L::scaled(lv, (aw[t][h] >> 4) & 0x0f0f0f0fu, s, o);
                    lds[lds_chunk(r, 4 * h + q)] = u32x4{A_::pack(e[0], e[2]), A_::pack(o[0], o[2]), A_::pack(e[1], e[3]), A_::pack(o[1], o[3])};
                }
            } else if constexpr (kWeightCols) {
                const int par = id & 1, d = (id >> 1) % (BI / 8), oct = octet<BI>(t, tid, wave);
                const unsigned half = par ? 0x07060302u : 0x05040100u;
                u32x4 out[4];  // column 8 d + 2 j + par, 8 rows each
#pragma unroll
                for (int e = 0; e < 4; ++e) {  // rows 2 e and 2 e + 1
                    const unsigned w = __builtin_amdgcn_perm(aw[t][2 * e + 1], aw[t][2 * e], half);
                    const float s0 = bf16_bits_to_f32(as[t][2 * e]), s1 = bf16_bits_to_f32(as[t][2 * e + 1]);
                    const float s[4] = {s0, s0, s1, s1};
                    float x[4], y[4];  // columns 0, 2 of both rows; columns 1, 3
                    L::scaled(lv, w & 0x0f0f0f0fu, s, x);
                    L::scaled(lv, (w >> 4) & 0x0f0f0f0fu, s, y);
                    out[0][e] = A_::pack(x[0], x[2]);
                    out[1][e] = A_::pack(y[0], y[2]);
                    out[2][e] = A_::pack(x[1], x[3]);
                    out[3][e] = A_::pack(y[1], y[3]);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) lds[lds_chunk(8 * d + 2 * j + par, oct)] = out[j];
            } else {
                const int quad = id % (BI / 4), oct = octet<BI>(t, tid, wave);
                u32x4 out[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float v[2][4];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const unsigned x = as[t][2 * e + h];
                        const float s = __builtin_bit_cast(float, x == 255u ? 0x7fc00000u : x << 23);
                        const unsigned u = aw[t][2 * e + h] ^ 0x80808080u;  // q + 128
#pragma unroll
                        for (int j = 0; j < 4; ++j) v[h][j] = __builtin_fmaf((float)((u >> (8 * j)) & 255u), s, -128.0f * s);
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) out[j][e] = A_::pack_exact(v[0][j], v[1][j]);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) lds[lds_chunk(4 * quad + j, oct)] = out[j];
            }
        }
    }

    __device__ __forceinline__ void load_b(const GemmParams& p, int64_t j0, int c, int tid, int wave) {
        const bool full = c + kStep <= p.C;
#pragma unroll
        for (int t = 0; t < PB; ++t) {
            const int id = t * NT + tid;
            if constexpr (!kCheckpoint) {  // rows j, 8 neighbours along c
                const int r = id >> 3, ch = id & 7, c0 = c + 8 * ch;
                const uint16_t* row = (const uint16_t*)p.B + c + (min(j0 + r, p.J - 1) * p.ldb + 8 * ch);
                if (full) {
                    __builtin_memcpy(bv[t], row, 16);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const unsigned lo = c0 + 2 * e < p.C ? row[2 * e] : 0u;
                        const unsigned hi = c0 + 2 * e + 1 < p.C ? row[2 * e + 1] : 0u;
                        bv[t][e] = lo | (hi << 16);
                    }
                }
            } else {  // 8 rows along c, four neighbours along j
                const int oct = octet<BJ>(t, tid, wave), quad = id % (BJ / 4), m = c + 8 * oct;
                const int n = (int)j0 + 4 * quad, J = (int)p.J;
                if (J >= 4) {  // four that lie inside, moved down to column n
                    const int n1 = min(n, J - 4), shift = 16 * min(n - n1, 3);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int64_t row = full ? m + e : min(m + e, (int)p.C - 1);
                        uint64_t v;
                        __builtin_memcpy(&v, (const char*)((const uint16_t*)p.B + row * p.ldb) + 2u * (unsigned)n1, 8);
                        if (j0 + BJ > J) v >>= shift;
                        if (!full && m + e >= p.C) v = 0;
                        bv[t][2 * e] = (unsigned)v;
                        bv[t][2 * e + 1] = (unsigned)(v >> 32);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const uint16_t* row = (const uint16_t*)p.B + (int64_t)min(m + e, (int)p.C - 1) * p.ldb;
                        unsigned h[4];
#pragma unroll
                        for (int f = 0; f < 4; ++f) h[f] = m + e < p.C ? row[min(n + f, J - 1)] : 0u;
                        bv[t][2 * e] = h[0] | (h[1] << 16);
                        bv[t][2 * e + 1] = h[2] | (h[3] << 16);
                    }
                }
            }
        }
    }

    __device__ __forceinline__ void store_b(u32x4* lds, int tid, int wave) const {
#pragma unroll
        for (int t = 0; t < PB; ++t) {
            const int id = t * NT + tid;
            if constexpr (!kCheckpoint) {
                const int r = id >> 3, ch = id & 7;
                lds[lds_chunk(r, ch)] = u32x4{bv[t][0], bv[t][1], bv[t][2], bv[t][3]};
            } else {
                const int quad = id % (BJ / 4), oct = octet<BJ>(t, tid, wave);
#pragma unroll
                for (int f = 0; f < 4; ++f) {
                    u32x4 o;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        o[e] = __builtin_amdgcn_perm(bv[t][2 * (2 * e + 1) + (f >> 1)], bv[t][2 * (2 * e) + (f >> 1)],
                                                     (f & 1) ? 0x07060302u : 0x05040100u);
                    lds[lds_chunk(4 * quad + f, oct)] = o;
                }
            }
        }
    }
};

// Workgroups are dealt to the eight XCDs in turn; tile numbers are dealt so that an XCD's workgroups take
// neighbouring tiles (their operands meet in its L2).  A bijection for any count.
__device__ __forceinline__ int xcd_tile(int b, int count) {
    const int per = count >> 3, rest = count & 7, x = b & 7;
    return x * per + min(x, rest) + (b >> 3);
}

template <bool BF, bool LUT, int MODE, int BI, int BJ, int WI, int WJ>
__global__ __launch_bounds__(64 * WI * WJ) void group_gemm_kernel(const GemmParams p) {
    using G = Gemm<BF, LUT, MODE, BI, BJ, WI, WJ>;
    constexpr int MI = G::MI, MJ = G::MJ;
    __shared__ u32x4 s_buf[2][(BI + BJ) * 8];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wi = wave % WI, wj = wave / WI;
    const int tile = xcd_tile(blockIdx.x, p.itiles * p.jtiles);
    const int i0 = tile % p.itiles * BI, j0 = tile / p.itiles * BJ;
    typename G::L levels;
    if constexpr (LUT) levels.init(p.w.levels);

    f32x4 acc[MI][MJ];
#pragma unroll
    for (int a = 0; a < MI; ++a)
#pragma unroll
        for (int b = 0; b < MJ; ++b) acc[a][b] = f32x4{0, 0, 0, 0};

    const int s_begin = blockIdx.y * p.steps_per_split;
    const int s_end = min(s_begin + p.steps_per_split, (int)((p.C + kStep - 1) / kStep));
    G st;
    auto load = [&](int s) {
        st.load_a(p, i0, s * kStep, tid, wave);
        st.load_b(p, j0, s * kStep, tid, wave);
    };
    auto store = [&](int buf) {
        st.store_a(s_buf[buf], tid, wave, levels);
        st.store_b(s_buf[buf] + BI * 8, tid, wave);
    };
    auto compute = [&](int buf) {
        const u32x4* s_a = s_buf[buf];
        const u32x4* s_b = s_buf[buf] + BI * 8;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            u32x4 af[MI], bf[MJ];
#pragma unroll
            for (int b = 0; b < MJ; ++b) bf[b] = s_b[lds_chunk((wj * MJ + b) * 16 + (lane & 15), kk * 4 + (lane >> 4))];
#pragma unroll
            for (int a = 0; a < MI; ++a) af[a] = s_a[lds_chunk((wi * MI + a) * 16 + (lane & 15), kk * 4 + (lane >> 4))];
#pragma unroll
            for (int a = 0; a < MI; ++a)
#pragma unroll
                for (int b = 0; b < MJ; ++b) acc[a][b] = Act<BF>::mfma(af[a], bf[b], acc[a][b]);
        }
    };
    if (s_begin < s_end) {
        load(s_begin);
        store(0);
        if (s_begin + 1 < s_end) load(s_begin + 1);
        __syncthreads();
        // Two waves share a SIMD: one stages the next step while the other computes, then they change places.
        const bool stage_first = wave < WI * WJ / 2;
        for (int s = s_begin; s < s_end; ++s) {
            const int buf = (s - s_begin) & 1;
            if (!stage_first) compute(buf);
            if (s + 1 < s_end) store(buf ^ 1);
            if (s + 2 < s_end) load(s + 2);
            if (stage_first) compute(buf);
            __syncthreads();
        }
    }

    // lane holds out[j][i .. i + 3], j = its column of the 16 x 16 tile
    const int64_t jl = (int64_t)j0 + wj * MJ * 16 + (lane & 15);
    const int il = i0 + wi * MI * 16 + 4 * (lane >> 4);
    if constexpr (MODE == (int)Product::GradScales) {
        static_assert(BI / WI == 128, "a wave holds whole groups");
#pragma unroll
        for (int b = 0; b < MJ; ++b) {
            const int n = (int)jl + 16 * b;
            const bool live = n < p.w.n;
            float sum[MI / 2];  // per 32 columns
#pragma unroll
            for (int a = 0; a < MI; ++a) {
                // columns past the matrix repeat codes of the last tile: the checkpoint is zero there, or the group is not stored
                const int k = il + 16 * a, kk = k & 127;
                const unsigned d = *(const unsigned*)(p.w.codes + ((int64_t)(min(n, p.w.n - 1) >> 4) * p.w.ktiles + min(k >> 7, p.w.ktiles - 1)) * kTileBytes +
                                                      (n & 15) * 64 + ((kk >> 3) & 3) * 16 + (kk >> 5) * 4);
                // columns 4 h .. 4 h + 3 of the dword: nibbles 2 h, 2 h + 4, 2 h + 1, 2 h + 5
                const unsigned w = d >> (8 * ((kk >> 2) & 1));
                const unsigned b4 = (w & 15u) | (w & 0xf0000u) >> 8 | (w & 0xf0u) << 12 | (w & 0xf00000u) << 4;
                float lv[4];
                G::L::plain(levels, b4, lv);
                float v = 0.0f;
#pragma unroll
                for (int r = 0; r < 4; ++r) v = __builtin_fmaf(lv[r], acc[a][b][r], v);
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
            const int64_t j = jl + 16 * b;
            if (j >= p.J) continue;
#pragma unroll
            for (int a = 0; a < MI; ++a) {
                const int i = il + 16 * a;
                if (i >= p.I) continue;
                f32x4 v = acc[a][b];
                const bool whole = i + 4 <= p.I;
                if (MODE == (int)Product::GradWeight || p.part != nullptr) {
                    float* o = p.part ? p.part + ((int64_t)blockIdx.y * p.J + j) * p.I + i : (float*)p.out + j * p.ldo + i;
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
                    uint16_t* o = (uint16_t*)p.out + j * p.ldo + i;
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
    const int64_t steps = ceil_div64(C, kStep);
    auto tiles = [&](int bi, int bj) { return ceil_div64(I, bi) * ceil_div64(J, bj); };
    const bool rows = mode == Product::Linear || mode == Product::GradInput;
    if (tiles(256, 256) >= 192) g.bi = g.bj = 256;
    else if (rows && J <= 32) g.bi = 128, g.bj = 32;
    else if (rows && J <= 64) g.bi = 128, g.bj = 64;
    else if (rows && tiles(256, 128) >= 192) g.bi = 256, g.bj = 128;
    else g.bi = g.bj = 128;
    int64_t splits = 1;
    const int64_t t = tiles(g.bi, g.bj);
    if (t < 256) splits = 512 / t < steps / 4 ? 512 / t : steps / 4;
    if (splits < 1) splits = 1;
    g.steps_per_split = (int)ceil_div64(steps, splits);
    if (g.steps_per_split < 1) g.steps_per_split = 1;
    g.splits = steps ? (int)ceil_div64(steps, g.steps_per_split) : 1;
    const int64_t values = mode == Product::GradScales ? J * groups : I * J;
    g.ws_bytes = g.splits > 1 ? (size_t)g.splits * (size_t)values * sizeof(float) : 0;
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

template <int MODE>
static hipError_t launch_mode(bool bf16, const GemmPlan& g, const GemmParams& p, hipStream_t s) {
    if constexpr (MODE == (int)Product::Linear || MODE == (int)Product::GradInput) {
        if (g.bj == 32) return launch_tile<MODE, 128, 32, 4, 1>(bf16, p, s);
        if (g.bj == 64) return launch_tile<MODE, 128, 64, 2, 2>(bf16, p, s);
        if (g.bi == 256 && g.bj == 128) return launch_tile<MODE, 256, 128, 4, 2>(bf16, p, s);
    }
    if (g.bi == 256) return launch_tile<MODE, 256, 256, 2, 4>(bf16, p, s);
    // (a wave of the scales' gradient holds whole groups)
    return launch_tile<MODE, 128, 128, MODE == (int)Product::GradScales ? 1 : 2, MODE == (int)Product::GradScales ? 4 : 2>(bf16, p, s);
}

hipError_t launch_gemm(Product mode, bool bf16, const GemmPlan& plan, GemmParams p, hipStream_t s) {
    p.itiles = (int)ceil_div64(p.I, plan.bi);
    p.jtiles = (int)ceil_div64(p.J, plan.bj);
    p.splits = plan.splits;
    p.steps_per_split = plan.steps_per_split;
    if (plan.splits == 1) p.part = nullptr;
    hipError_t e;
    switch (mode) {
        case Product::Linear: e = launch_mode<0>(bf16, plan, p, s); break;
        case Product::GradInput: e = launch_mode<1>(bf16, plan, p, s); break;
        case Product::GradWeight: e = launch_mode<2>(bf16, plan, p, s); break;
        default: e = launch_mode<3>(bf16, plan, p, s);
    }
    if (e != hipSuccess || plan.splits == 1) return e;
    const bool rows = mode == Product::Linear || mode == Product::GradInput;
    const JoinParams j = {p.part, p.splits, p.J, mode == Product::GradScales ? p.w.groups : p.I, p.bias, p.out, p.ldo,
                          rows ? (bf16 ? KQ_T_BF16 : KQ_T_F16) : KQ_T_F32};
    return launch_join(j, s);
}

}  // namespace kq
