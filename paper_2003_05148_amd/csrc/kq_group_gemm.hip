// The products of a 4-bit fully-connected layer on the matrix cores.
//
// Every product is out[j][i] = sum_c A[i][c] B[j][c] with i the contiguous dimension of the output, so
// that a lane's four accumulators are neighbours in memory.  A workgroup holds a BI x BJ tile of the output
// in registers and walks the contraction in steps of 64; a step's operands lie in LDS as 16-bit rows of 64
// (128 bytes), two steps' worth of them.
//   Linear      A = W from its codes (a row's eight columns are one dword), B = X
//   GradInput   A = W^T: eight rows' dwords of one thread are an 8 x 8 block, written transposed; B = dY
//   GradWeight  A = X^^T from the checkpoint (8 rows x 4 columns a thread), B = dY^T
//   GradScales  the same product; the epilogue multiplies it by the levels and adds up each group
// A goes through registers, where it becomes 16-bit values; B goes from memory to LDS directly, so it has to
// lie in 16-byte aligned rows along c: dY is transposed into the workspace first (its column sums, the bias
// gradient, are taken on the way), and an X or dY whose rows are not aligned is copied there.
// Weights are s * level rounded once to the activation's type (bf16: s has 8 bits and -8..7 three, so
// about half of them are exact; fp16 holds all of these in its range): applying the scale to a group's fp32 sum
// instead, as the few-row kernel does, would take as many accumulators again, and the tile would halve.  Equal
// codes of a group round alike, so where X has one sign their errors add up: of the result's norm 0.0022 for random
// X and up to 0.0041 for positive X with a level table, where rounding the result alone gives 0.0017 (fp16: 2.1e-4
// with -8 .. 7, 2.9e-4 and 4.3e-4 with a table, and 2.1e-4).  Checkpoints and activations are exact, sums are fp32.
//
// Measured, bf16: Linear 2048 x 4096 x 4096 82 us (837 TFLOP/s; 80 to 86 on several machines), GradInput 4096 x 4096 x
// 4096 131 us (1050; 127 to 140), GradScales 2048 x 4096 x 25088 463 us (909), with dY's transpose (11 us) and the bias gradient.  What
// bounds them: no pipe alone.  Of an earlier GradInput (143 us in that run) the products by themselves take 103 us
// (MFMA issue and fragment reads), decoding by itself 50, loads by themselves 88; two waves a SIMD cover part
// of each other.  At a split contraction the partial sums count too (the weight's gradient of 2047 x 1000 x
// 4095: 5 transpose + 33 product + 14 joining of 51 us).
#include "kq_group.h"

namespace kq {

constexpr int kStep = 64;  // contraction per step

// LDS rows of 128 bytes in eight 16-byte chunks; chunk ch of row r lies at ch ^ swizzle(r).  Eight
// consecutive rows of one chunk (fragment reads), rows 4 l + t (transposed writes of four columns) and rows
// 8 d + 2 t + par (transposed writes of a dword's even or odd columns) all fall on eight different chunks.  Linear's
// writes do not: eight lanes write chunks 4 h + 0 .. 3 of two neighbouring rows, two to a bank (8 more cycles a
// write, a quarter of the kernel's LDS cycles).
__device__ __forceinline__ int swizzle(int r) { return (r ^ (r >> 2)) & 7; }
__device__ __forceinline__ int lds_chunk(int r, int ch) { return r * 8 + (ch ^ swizzle(r)); }

// A 16-byte store to LDS.  The compiler cannot always tell an ordinary one from the target of a direct load in
// flight, and then waits for every load first; the step's end waits for both.
__device__ __forceinline__ void write_lds(u32x4* at, u32x4 v) {
    asm volatile("ds_write_b128 %0, %1" ::"v"((unsigned)(uintptr_t)(__attribute__((address_space(3))) u32x4*)at), "v"(v) : "memory");
}

// Four codes as fp32 s * level (scaled: the even or the odd nibbles of w) or as levels (plain: the bytes of b, 0..15).
template <bool LUT>
struct Levels;
template <>
struct Levels<false> {
    __device__ __forceinline__ void init(const uint16_t*) {}
    // levels -8 .. 7: a nibble with its top bit turned, in the upper half of a byte, is 16 (q - 8) as a signed byte.
    // (fma(q, s, -8 s) would overflow for scales from 2^125 on, of which the largest weights have some.)
    template <int ODD>
    static __device__ __forceinline__ void scaled(const Levels&, unsigned w, const float (&s)[4], float (&v)[4]) {
        const unsigned b = ((ODD ? w : w << 4) & 0xf0f0f0f0u) ^ 0x80808080u;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = (float)((int)(b << (24 - 8 * j)) >> 24) * (0.0625f * s[j]);
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
    template <int ODD>
    static __device__ __forceinline__ void scaled(const Levels& l, unsigned w, const float (&s)[4], float (&v)[4]) {
        plain(l, (ODD ? w >> 4 : w) & 0x0f0f0f0fu, v);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] *= s[j];
    }
};

template <bool BF, bool LUT, int MODE, int BI, int BJ, int WI, int WJ>
struct StageA {
    static constexpr int NT = 64 * WI * WJ;
    static constexpr int MI = BI / WI / 16, MJ = BJ / WJ / 16;  // 16 x 16 tiles of a wave
    static constexpr bool kWeightRows = MODE == (int)Product::Linear;
    static constexpr bool kWeightCols = MODE == (int)Product::GradInput;
    static constexpr bool kCheckpoint = MODE >= (int)Product::GradWeight;
    using A_ = Act<BF>;
    using L = Levels<LUT>;

    // A thread's pieces of a step.  Rows past the output's edge repeat the last ones (what they give is not
    // stored, or cleared before a group's sum); past the contraction's edge both A and B are zero.
    static constexpr int kATasks = kWeightRows ? BI * 4 : BI * 2;
    static constexpr int PA = kATasks / NT;
    static_assert(kATasks % NT == 0 && PA >= 1, "A tasks");
    unsigned w[PA][kWeightRows ? 2 : 8];
    unsigned short x[PA][kWeightRows ? 2 : 8];  // scales (bf16 bits) or checkpoint exponents

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

    __device__ __forceinline__ void load(const GemmParams& p, int i0, int c, int tid, int wave) {
        const bool full = c + kStep <= p.C;
#pragma unroll
        for (int t = 0; t < PA; ++t) {
            const int id = t * NT + tid;
            if constexpr (kWeightRows) {  // row of W, 8 bytes: two runs of 8 columns, 32 apart
                const int r = min(id >> 2, p.w.n - 1 - i0), q = id & 3;
                const uint8_t* base = p.w.codes + ((int64_t)(i0 >> 4) * p.w.ktiles + (c >> 7)) * kTileBytes + ((c & 64) >> 3);
                const u32x2 d = at<u32x2>(base, (unsigned)(r >> 4) * (unsigned)p.w.ktiles * kTileBytes + (r & 15) * 64 + q * 16);
                w[t][0] = d.x;
                w[t][1] = d.y;
                const uint16_t* sc = p.w.scales + (int64_t)i0 * p.w.groups;
                const unsigned row = (unsigned)r * (unsigned)p.w.groups;
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    x[t][h] = at<unsigned short>(sc + min((c + 32 * h) >> p.w.log_group, p.w.groups - 1), 2 * row);
            } else if constexpr (kWeightCols) {  // 8 rows, one dword: the even or the odd half of 8 columns
                const int oct = octet<BI>(t, tid, wave), d = (id >> 1) % (BI / 8);
                const int k = min(i0 + 8 * d, p.w.k - 1), n = c + 8 * oct;
                const int kk = k & 127, dw = ((kk >> 3) & 3) * 4 + (kk >> 5);
                const uint8_t* base = p.w.codes + (int64_t)min(n >> 4, p.w.ntiles - 1) * p.w.ktiles * kTileBytes + (n & 15) * 64;
                const unsigned col = (unsigned)(k >> 7) * kTileBytes + dw * 4, g = 2 * (unsigned)(k >> p.w.log_group);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    w[t][e] = at<unsigned>(base + e * 64, col);
                    x[t][e] = at<unsigned short>(p.w.scales + (int64_t)min(n + e, p.w.n - 1) * p.w.groups, g);
                }
            } else {  // 8 rows of the checkpoint, 4 columns
                const int oct = octet<BI>(t, tid, wave), quad = id % (BI / 4);
                const unsigned k = min(i0 + 4 * quad, p.kq - 4);
                const int m = c + 8 * oct;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int64_t row = full ? m + e : min(m + e, (int)p.C - 1);
                    w[t][e] = at<unsigned>(p.q + row * p.kq, k);
                    x[t][e] = at<uint8_t>(p.exps + row * (p.kq >> 5), k >> 5);
                }
            }
        }
    }

    // c: the step's place in the contraction of C.  (What lies past its end was loaded from the last row; it
    // is taken off here, where the loads have arrived.)
    __device__ __forceinline__ void store(u32x4* lds, int64_t C, int c, int tid, int wave, const L& lv) const {
        if (kWeightRows || c + kStep <= C) store_step<false>(lds, C, c, tid, wave, lv);
        else store_step<true>(lds, C, c, tid, wave, lv);
    }
    // Linear's last step, after its store: columns of code 0 past the matrix.  Their weight may be infinite in the
    // activation's type although none of the matrix is, and infinity times B's zero is NaN.  (A thread clears what it
    // wrote itself: LDS keeps a wave's order.  In a branch that was there, Linear 2048 x 4096 x 4096 takes 81.8 us, 81.6
    // without it; selects in the store took 1.7 % more.)
    __device__ __forceinline__ void clear_past(u32x4* lds, int64_t C, int c, int tid) const {
#pragma unroll
        for (int t = 0; t < PA; ++t) {
            const int id = t * NT + tid, r = id >> 2, q = id & 3;
            for (int h = 0; h < 2; ++h)
                for (int j = max((int)min(C - c - 32 * h - 8 * q, (int64_t)8), 0); j < 8; ++j)
                    ((uint16_t*)(lds + lds_chunk(r, 4 * h + q)))[j] = 0;
        }
    }
    template <bool EDGE>
    __device__ __forceinline__ void store_step(u32x4* lds, int64_t C, int c, int tid, int wave, const L& lv) const {
#pragma unroll
        for (int t = 0; t < PA; ++t) {
            const int id = t * NT + tid;
            const int left = !EDGE ? 8 : (int)min(C - c - 8 * octet<BI>(t, tid, wave), (int64_t)8);  // rows of the octet
            if constexpr (kWeightRows) {
                const int r = id >> 2, q = id & 3;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float s1 = bf16_bits_to_f32(x[t][h]);
                    const float s[4] = {s1, s1, s1, s1};
                    float e[4], o[4];  // nibbles 0 2 4 6 are columns 0 4 1 5, nibbles 1 3 5 7 columns 2 6 3 7
                    L::template scaled<0>(lv, w[t][h], s, e);
                    L::template scaled<1>(lv, w[t][h], s, o);
                    write_lds(lds + lds_chunk(r, 4 * h + q), u32x4{A_::pack(e[0], e[2]), A_::pack(o[0], o[2]), A_::pack(e[1], e[3]), A_::pack(o[1], o[3])});
                }
            } else if constexpr (kWeightCols) {
                const int par = id & 1, d = (id >> 1) % (BI / 8), oct = octet<BI>(t, tid, wave);
                const unsigned half = par ? 0x07060302u : 0x05040100u;
                u32x4 out[4];  // column 8 d + 2 j + par, 8 rows each
#pragma unroll
                for (int e = 0; e < 4; ++e) {  // rows 2 e and 2 e + 1
                    const unsigned pairw = __builtin_amdgcn_perm(w[t][2 * e + 1], w[t][2 * e], half);
                    const float s0 = bf16_bits_to_f32(2 * e < left ? x[t][2 * e] : 0), s1 = bf16_bits_to_f32(2 * e + 1 < left ? x[t][2 * e + 1] : 0);
                    const float s[4] = {s0, s0, s1, s1};
                    float ev[4], od[4];  // columns 0, 2 of both rows; columns 1, 3
                    L::template scaled<0>(lv, pairw, s, ev);
                    L::template scaled<1>(lv, pairw, s, od);
                    out[0][e] = A_::pack(ev[0], ev[2]);
                    out[1][e] = A_::pack(od[0], od[2]);
                    out[2][e] = A_::pack(ev[1], ev[3]);
                    out[3][e] = A_::pack(od[1], od[3]);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) write_lds(lds + lds_chunk(8 * d + 2 * j + par, oct), out[j]);
            } else {
                const int quad = id % (BI / 4), oct = octet<BI>(t, tid, wave);
                u32x4 out[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float v[2][4];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const unsigned ex = 2 * e + h < left ? x[t][2 * e + h] : 0;
                        const float s = checkpoint_step(ex);
#pragma unroll
                        for (int j = 0; j < 4; ++j) v[h][j] = (float)((int)(w[t][2 * e + h] << (24 - 8 * j)) >> 24) * s;
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) out[j][e] = A_::pack_bf16_value(v[0][j], v[1][j]);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) write_lds(lds + lds_chunk(4 * quad + j, oct), out[j]);
            }
        }
    }
};

// A step of B from memory to LDS: a wave's instruction takes 64 chunks of 16 bytes, eight rows; lane l writes
// chunk l of them, so it reads the chunk that belongs there.
using lds_ptr = __attribute__((address_space(3))) void*;
using global_ptr = const __attribute__((address_space(1))) void*;
template <int BJ, int WAVES>
struct DirectB {
    static constexpr int N = BJ / 8 / WAVES;
    static_assert(N >= 1 && BJ % (8 * WAVES) == 0, "B pieces");
    unsigned off[N];  // bytes from the tile's first row
    int col;          // the lane's first column
    __device__ __forceinline__ void init(const GemmParams& p, int64_t j0, int lane, int wave) {
        const int last = (int)min(p.J - 1 - j0, (int64_t)BJ - 1);
#pragma unroll
        for (int t = 0; t < N; ++t) {
            const int r = (t * WAVES + wave) * 8 + (lane >> 3), ch = (lane & 7) ^ swizzle(r);
            off[t] = (unsigned)min(r, last) * (unsigned)(2 * p.ldb) + 16 * ch;
        }
        col = 8 * ((lane & 7) ^ swizzle(wave * 8 + (lane >> 3)));  // (rows 64 apart have the same)
        static_assert(N == 1 || WAVES % 4 == 0, "the rows of a lane agree in their swizzle");
    }
    __device__ __forceinline__ void load(const GemmParams& p, int64_t j0, int c, u32x4* lds, int lane, int wave) const {
        const char* base = (const char*)p.B + (j0 * p.ldb + c) * 2;
#pragma unroll
        for (int t = 0; t < N; ++t) {
            u32x4* to = lds + (t * WAVES + wave) * 64;
            if (c + col < p.C) __builtin_amdgcn_global_load_lds((global_ptr)(base + off[t]), (lds_ptr)to, 16, 0, 0);
            else to[lane] = u32x4{0, 0, 0, 0};
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
    using G = StageA<BF, LUT, MODE, BI, BJ, WI, WJ>;
    constexpr int MI = G::MI, MJ = G::MJ, WAVES = WI * WJ;
    // (arrays of their own, so that the compiler can tell the direct loads' target from what is read and written beside them)
    __shared__ u32x4 s_a0[BI * 8];
    __shared__ u32x4 s_a1[BI * 8];
    __shared__ u32x4 s_b0[BJ * 8];
    __shared__ u32x4 s_b1[BJ * 8];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wi = wave % WI, wj = wave / WI;
    const int tile = xcd_tile(blockIdx.x, p.itiles * p.jtiles);
    const int i0 = tile % p.itiles * BI;
    const int64_t j0 = (int64_t)(tile / p.itiles) * BJ;
    typename G::L levels;
    if constexpr (LUT) levels.init(p.w.levels);

    f32x4 acc[MI][MJ];
#pragma unroll
    for (int a = 0; a < MI; ++a)
#pragma unroll
        for (int b = 0; b < MJ; ++b) acc[a][b] = f32x4{0, 0, 0, 0};

    const int s_begin = blockIdx.y * p.steps_per_split;
    const int s_end = min(s_begin + p.steps_per_split, (int)((p.C + kStep - 1) / kStep));
    // fragment (tile a, half kk) starts at chunk frag[(kk ^ a) & 1] + 128 a of the wave's rows: 16 rows further
    // the swizzle differs in the bit that kk sets
    const int r16 = lane & 15, sw = swizzle(r16);
    const int frag0 = r16 * 8 + ((lane >> 4) ^ sw), frag1 = r16 * 8 + ((4 + (lane >> 4)) ^ sw);
    static_assert(MI % 2 == 0 && MJ % 2 == 0, "a wave's rows start at a multiple of 32");
    auto compute = [&](const u32x4* a_rows, const u32x4* b_rows) {
        a_rows += wi * MI * 128;
        b_rows += wj * MJ * 128;
        // Two rows of tiles at a time, their fragments read two turns ahead: left alone, the compiler reads each
        // one just before its use and waits for LDS every time.
        constexpr int kTurns = MI;
        u32x4 af[3][2], bf[2][MJ];
        auto read = [&](int t) {
            const int kk = t / (MI / 2), a0 = t % (MI / 2) * 2;
            if (a0 == 0) {
#pragma unroll
                for (int b = 0; b < MJ; ++b) bf[kk][b] = b_rows[b * 128 + (((kk ^ b) & 1) ? frag1 : frag0)];
            }
#pragma unroll
            for (int a = 0; a < 2; ++a) af[t % 3][a] = a_rows[(a0 + a) * 128 + (((kk ^ a) & 1) ? frag1 : frag0)];
        };
        read(0);
        read(1);
#pragma unroll
        for (int t = 0; t < kTurns; ++t) {
            const int kk = t / (MI / 2), a0 = t % (MI / 2) * 2;
            if (t + 2 < kTurns) read(t + 2);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int a = 0; a < 2; ++a)
#pragma unroll
                for (int b = 0; b < MJ; ++b) acc[a0 + a][b] = Act<BF>::mfma(af[t % 3][a], bf[kk][b], acc[a0 + a][b]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // Step s is multiplied while B of step s + 1 is on its way to LDS, A of step s + 1 is turned into LDS, and
    // A of step s + 2 is on its way to registers.  Two waves share a SIMD: where A is transposed, one stages while
    // the other multiplies, then they change places (GradInput 4096 x 4096 x 4096: 143 us, 158 with all staging
    // first); Linear's shorter staging is better done first by all (4096 x 4096 x 4096: 131 and 139 us).
    const bool stage_first = MODE == (int)Product::Linear || wave < WAVES / 2;
    DirectB<BJ, WAVES> db;
    G st;
    auto step = [&](int s, const u32x4* a_now, u32x4* a_next, const u32x4* b_now, u32x4* b_next) {
        auto stage = [&]() {
            if (s + 1 < s_end) st.store(a_next, p.C, (s + 1) * kStep, tid, wave, levels);
            if (s + 2 < s_end) st.load(p, i0, (s + 2) * kStep, tid, wave);
            else if (MODE == (int)Product::Linear && s + 1 < s_end && (s + 2) * kStep > p.C) st.clear_past(a_next, p.C, (s + 1) * kStep, tid);
        };
        if (stage_first) stage();
        if (s + 1 < s_end) db.load(p, j0, (s + 1) * kStep, b_next, lane, wave);
        __builtin_amdgcn_sched_barrier(0);
        compute(a_now, b_now);
        __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): the direct loads (A's come after them, or were waited for)
        __builtin_amdgcn_sched_barrier(0);
        if (!stage_first) stage();
        __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
        // (__syncthreads() would wait for the loads of A too)
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    if (s_begin < s_end) {
        db.init(p, j0, lane, wave);
        db.load(p, j0, s_begin * kStep, s_b0, lane, wave);
        st.load(p, i0, s_begin * kStep, tid, wave);
        st.store(s_a0, p.C, s_begin * kStep, tid, wave, levels);
        if (MODE == (int)Product::Linear && (s_begin + 1) * kStep > p.C) st.clear_past(s_a0, p.C, s_begin * kStep, tid);
        if (s_begin + 1 < s_end) st.load(p, i0, (s_begin + 1) * kStep, tid, wave);
        __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0) lgkmcnt(0)
        __syncthreads();
        for (int s = s_begin; s < s_end; s += 2) {
            step(s, s_a0, s_a1, s_b0, s_b1);
            if (s + 1 < s_end) step(s + 1, s_a1, s_a0, s_b1, s_b0);
        }
    }

    // lane holds out[j][i .. i + 3], j = its column of the 16 x 16 tile
    const int64_t jl = j0 + wj * MJ * 16 + (lane & 15);
    const int il = i0 + wi * MI * 16 + 4 * (lane >> 4);
    if constexpr (MODE >= (int)Product::GradWeight) {  // the partial column sums of dY, once
        if (p.dbias && i0 == 0 && blockIdx.y == 0) {
            for (int64_t j = j0 + tid; j < min(j0 + BJ, p.J); j += 64 * WAVES) {
                float v = 0.0f;
                for (int t = 0; t < p.bias_parts; ++t) v += p.bias_part[(int64_t)t * p.J + j];
                p.dbias[j] = v;
            }
        }
    }
    if constexpr (MODE == (int)Product::GradScales) {
        static_assert(BI / WI == 128, "a wave holds whole groups");
        // A matrix may end inside a group.  Past it the accumulators hold repeated columns, or 0 * inf where dY is not
        // finite, and the codes' level need not be zero: they are cleared.  (In a branch of the edge's workgroups:
        // a select beside each product took 25 of 459 us at 2048 x 4096 x 25088.)
        if (i0 + BI > p.w.k) {
#pragma unroll
            for (int a = 0; a < MI; ++a)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const bool past = il + 16 * a + r >= p.w.k;
#pragma unroll
                    for (int b = 0; b < MJ; ++b) acc[a][b][r] = past ? 0.0f : acc[a][b][r];
                }
        }
#pragma unroll
        for (int b = 0; b < MJ; ++b) {
            const int n = (int)jl + 16 * b;
            const bool live = n < p.w.n;
            float sum[MI / 2];  // per 32 columns
#pragma unroll
            for (int a = 0; a < MI; ++a) {
                // (past the last tile its codes again: their accumulators are zero)
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

// ---- B in aligned rows along the contraction -------------------------------------------------------------
// out[j][c], rows of p.pitch values (a multiple of 64, zeros from the contraction's end).
// Transposed (dY): a workgroup takes 32 columns of 256 rows, through LDS; column sums of its rows on the way.
__global__ __launch_bounds__(256) void transpose_grad_kernel(const StageBParams p, bool bf16) {
    constexpr int kPitch = 264;  // 16-bit values of an LDS row: 16 bytes over 512
    __shared__ __attribute__((aligned(16))) uint16_t s_t[32 * kPitch];
    __shared__ float s_sum[4][32];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, cl = tid & 3, rl = tid >> 2;
    const int64_t m0 = (int64_t)blockIdx.y * 256;
    const int n0 = blockIdx.x * 32 + 8 * cl;
    unsigned v[4][4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const int64_t m = m0 + 64 * t + rl;
        const uint16_t* at = (const uint16_t*)p.in + (m < p.C ? m * p.ld : 0) + n0;
        if (m < p.C && n0 + 8 <= p.J) {
            __builtin_memcpy(v[t], at, 16);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned lo = m < p.C && n0 + 2 * e < p.J ? at[2 * e] : 0u;
                const unsigned hi = m < p.C && n0 + 2 * e + 1 < p.J ? at[2 * e + 1] : 0u;
                v[t][e] = lo | (hi << 16);
            }
        }
    }
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int t = 0; t < 4; ++t) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int r = 64 * t + rl;
            s_t[(8 * cl + 2 * e) * kPitch + r] = (uint16_t)v[t][e];
            s_t[(8 * cl + 2 * e + 1) * kPitch + r] = (uint16_t)(v[t][e] >> 16);
            sum[2 * e] += bf16 ? Act<true>::lo(v[t][e]) : Act<false>::lo(v[t][e]);
            sum[2 * e + 1] += bf16 ? Act<true>::hi(v[t][e]) : Act<false>::hi(v[t][e]);
        }
    }
    if (p.bias_part) {
#pragma unroll
        for (int t = 0; t < 8; ++t) {
#pragma unroll
            for (int off = 4; off < 64; off <<= 1) sum[t] += __shfl_xor(sum[t], off);
            if (lane < 4) s_sum[wave][8 * lane + t] = sum[t];
        }
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < 4; ++t) {  // 32 rows of 512 bytes
        const int id = t * 256 + tid, r = id >> 5, ch = id & 31;
        const int64_t j = (int64_t)blockIdx.x * 32 + r, c = m0 + 8 * ch;
        if (j < p.J && c < p.pitch) *(u32x4*)((uint16_t*)p.out + j * p.pitch + c) = *(const u32x4*)(s_t + r * kPitch + 8 * ch);
    }
    const int64_t j = (int64_t)blockIdx.x * 32 + tid;
    if (p.bias_part && tid < 32 && j < p.J)
        p.bias_part[blockIdx.y * p.J + j] = ((s_sum[0][tid] + s_sum[1][tid]) + s_sum[2][tid]) + s_sum[3][tid];
}

// Copied: eight neighbours a thread.
__global__ __launch_bounds__(256) void align_rows_kernel(const StageBParams p) {
    const unsigned per_row = (unsigned)(p.pitch >> 3), id = blockIdx.x * 256u + threadIdx.x;  // (fewer than 2^32 threads)
    const int64_t j = id / per_row, c = (int64_t)(id - (unsigned)j * per_row) * 8;
    if (j >= p.J) return;
    const uint16_t* at = (const uint16_t*)p.in + j * p.ld + c;
    u32x4 v;
    if (c + 8 <= p.C) {
        __builtin_memcpy(&v, at, 16);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const unsigned lo = c + 2 * e < p.C ? at[2 * e] : 0u;
            const unsigned hi = c + 2 * e + 1 < p.C ? at[2 * e + 1] : 0u;
            v[e] = lo | (hi << 16);
        }
    }
    *(u32x4*)((uint16_t*)p.out + j * p.pitch + c) = v;
}

static bool rows_are_aligned(const void* B, int64_t ldb, int64_t C) {
    return ((uintptr_t)B & 15) == 0 && (ldb & 7) == 0 && (C & 7) == 0 && ldb < (int64_t(1) << 22);
}

// DirectB's 32-bit byte offsets reach the last chunk of bj rows (a staged operand's pitch is the contraction
// itself, up to KQ_GROUP_MAX_FEATURES: 256 rows reach to 8.42 million columns, 128 rows to all).
static bool row_offsets_fit(int bj, int64_t pitch) {
    return (int64_t)(bj - 1) * 2 * pitch + 2 * kStep <= int64_t(UINT32_MAX);
}
static_assert(127 * 2 * (int64_t)KQ_GROUP_MAX_FEATURES + 2 * kStep <= int64_t(UINT32_MAX), "every pitch has a tile");

// The tile and the splits with the shortest modelled time.  A workgroup's step takes `alone` us while it has a CU
// to itself, and a CU with n workgroups at hand takes n times `shared`; a split contraction pays the joining
// launch and its partial sums, written and read at about 6 MB a us.  The figures are fitted to sweeps of all
// tiles and 1 to 16 splits, and what is picked is within a twentieth of the sweeps' best (us for 1, 2, 4 and 8
// splits): X 512 x 4096 by W 4096 x 4096, 128x128 tiles 66 43 36 46, 256x128 73 48 35 47, 256x256 110 67 46 44,
// picked 36; 64 rows of X, 128x32 51 30 20 17, 128x128 63 37 24 19, picked 17; 1024 rows, 256x128 75 57 66 85,
// 256x256 111 71 55 73, picked 56; dX of 512 rows, 128x128 91 56 61 70, 256x128 99 60 40 50, picked 40; scales'
// gradient 2048 x 4096 x 1024, 128x128 61 46 49 56, 256x256 75 51 39 45, picked 40.
struct TileTime {
    int bi, bj;
    float alone[3], shared[3];  // Linear, GradInput, the gradients from a checkpoint
};
constexpr TileTime kTiles[] = {
    {128, 32, {0.62f, 1.10f, 0.0f}, {0.33f, 0.42f, 0.0f}},
    {128, 64, {0.70f, 1.00f, 0.0f}, {0.50f, 0.60f, 0.0f}},
    {128, 128, {0.92f, 1.30f, 1.50f}, {0.60f, 1.00f, 0.95f}},
    {256, 128, {1.15f, 1.37f, 0.0f}, {1.15f, 1.37f, 0.0f}},
    {256, 256, {1.75f, 1.80f, 2.00f}, {1.75f, 1.80f, 2.00f}},
};

GemmPlan gemm_plan(Product mode, const void* B, int64_t ldb, int64_t I, int64_t J, int64_t C, int groups) {
    GemmPlan g = {};
    const int64_t steps = ceil_div64(C, kStep);
    const bool rows = mode == Product::Linear || mode == Product::GradInput;
    const int column = mode == Product::Linear ? 0 : mode == Product::GradInput ? 1 : 2;
    const float value_us = (mode == Product::GradScales ? (float)J * groups : (float)I * J) * 8.0f / 6e6f;
    g.stage_b = !rows || !rows_are_aligned(B, ldb, C);
    g.pitch = ceil_div64(C, kStep) * kStep;
    float best = 0.0f;
    int64_t splits = 1;
    for (const TileTime& t : kTiles) {
        if (t.alone[column] == 0.0f) continue;
        if (!row_offsets_fit(t.bj, g.stage_b ? g.pitch : ldb)) continue;  // (of 128 rows and fewer all do)
        const int64_t tiles = ceil_div64(I, t.bi) * ceil_div64(J, t.bj);
        for (int s = 1; s <= 32 && (s == 1 || (s * 2 <= steps && s * tiles <= 1024)); s = s < 4 ? s + 1 : s * 3 / 2) {  // 1 2 3 4 6 9 13 ..
            const float n = (float)ceil_div64(tiles * s, 256), step = n * t.shared[column] > t.alone[column] ? n * t.shared[column] : t.alone[column];
            const float us = (float)ceil_div64(steps, s) * step + (s > 1 ? 2.5f + s * value_us : 0.0f);
            if (g.bi == 0 || us < best) {
                best = us;
                g.bi = t.bi;
                g.bj = t.bj;
                splits = s;
            }
        }
    }
    g.steps_per_split = (int)ceil_div64(steps, splits);
    if (g.steps_per_split < 1) g.steps_per_split = 1;
    g.splits = steps ? (int)ceil_div64(steps, g.steps_per_split) : 1;
    const int64_t values = mode == Product::GradScales ? J * groups : I * J;
    auto region = [](size_t bytes) { return (bytes + 255) & ~size_t(255); };
    g.part_bytes = g.splits > 1 ? region((size_t)g.splits * (size_t)values * sizeof(float)) : 0;
    g.b_bytes = g.stage_b ? region((size_t)J * (size_t)g.pitch * 2) : 0;
    g.bias_parts = rows ? 0 : (int)ceil_div64(C, 256);
    g.ws_bytes = g.part_bytes + g.b_bytes + (rows ? 0 : region((size_t)g.bias_parts * (size_t)J * sizeof(float)));
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

// (a tile that a product has no kernel for is refused: a kernel must have the plan's tile)
template <int MODE>
static hipError_t launch_mode(bool bf16, const GemmPlan& g, const GemmParams& p, hipStream_t s) {
    const int tile = g.bi * 1000 + g.bj;
    if constexpr (MODE == (int)Product::Linear || MODE == (int)Product::GradInput) {
        if (tile == 128032) return launch_tile<MODE, 128, 32, 4, 1>(bf16, p, s);
        if (tile == 128064) return launch_tile<MODE, 128, 64, 2, 2>(bf16, p, s);
        if (tile == 256128) return launch_tile<MODE, 256, 128, 4, 2>(bf16, p, s);
    }
    if (tile == 256256) return launch_tile<MODE, 256, 256, 2, 4>(bf16, p, s);
    // (a wave of the scales' gradient holds whole groups)
    if (tile == 128128)
        return launch_tile<MODE, 128, 128, MODE == (int)Product::GradScales ? 1 : 2, MODE == (int)Product::GradScales ? 4 : 2>(bf16, p, s);
    return hipErrorInvalidValue;
}

hipError_t launch_gemm(Product mode, bool bf16, const GemmPlan& plan, GemmParams p, void* ws, hipStream_t s) {
    const bool rows = mode == Product::Linear || mode == Product::GradInput;
    p.itiles = (int)ceil_div64(p.I, plan.bi);
    p.jtiles = (int)ceil_div64(p.J, plan.bj);
    p.splits = plan.splits;
    p.steps_per_split = plan.steps_per_split;
    p.part = plan.splits > 1 ? (float*)ws : nullptr;
    p.bias_parts = plan.bias_parts;
    p.bias_part = p.dbias ? (float*)((char*)ws + plan.part_bytes + plan.b_bytes) : nullptr;
    if (plan.stage_b && p.C > 0) {
        const StageBParams b = {p.B, p.ldb, p.J, p.C, (char*)ws + plan.part_bytes, plan.pitch, p.bias_part};
        if (rows) align_rows_kernel<<<dim3((unsigned)ceil_div64(p.J * (plan.pitch >> 3), 256)), dim3(256), 0, s>>>(b);
        else transpose_grad_kernel<<<dim3((unsigned)ceil_div64(p.J, 32), (unsigned)plan.bias_parts), dim3(256), 0, s>>>(b, bf16);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        p.B = b.out;
        p.ldb = plan.pitch;
    }
    hipError_t e;
    switch (mode) {
        case Product::Linear: e = launch_mode<0>(bf16, plan, p, s); break;
        case Product::GradInput: e = launch_mode<1>(bf16, plan, p, s); break;
        case Product::GradWeight: e = launch_mode<2>(bf16, plan, p, s); break;
        default: e = launch_mode<3>(bf16, plan, p, s);
    }
    if (e != hipSuccess || plan.splits == 1) return e;
    const JoinParams j = {p.part, p.splits, p.J, mode == Product::GradScales ? p.w.groups : p.I, p.bias, p.out, p.ldo,
                          rows ? (bf16 ? KQ_T_BF16 : KQ_T_F16) : KQ_T_F32};
    return launch_join(j, s);
}

}  // namespace kq
