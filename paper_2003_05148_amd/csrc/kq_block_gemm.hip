// The products of the 8-bit fully-connected layer on the matrix cores: out[j][i] = sum_c A[i][c] B[j][c], both operands
// rows of e4m3 bytes with one power of two for 128 of them.
//
// A workgroup holds a BI x BJ tile of the output in registers and walks the contraction block by block (128 deep).
// The operands' bytes go from memory to LDS directly, rows of 128 bytes in eight 16-byte chunks, chunk ch of row r at an
// exclusive or of ch and three bits of r (block_swizzle).  i is the contiguous dimension of the output, so that four
// accumulators of a lane are neighbours in memory.  The contraction is in any order that both operands share: lane l
// of the 32 x 32 x 64 instruction takes chunks 2 h' and 2 h' + 1 of its row's half, h' = l / 32.
//
// The input gradient's A is W^T: W's rows of BI bytes go to LDS as they lie, and the transposing LDS read gives a lane its column
// (a pass over W that wrote it transposed cost 6 of 71 us at 4096 x 4096 x 4096, and half of a call with few rows; this
// read costs the product 1 to 5 %).
//
// Two forms.  The scaled 8-bit instruction takes the bytes and both exponents as they are, at twice the 16-bit rate;
// it adds eight products at a time and cuts each off 13 bits below the largest of them.  That is 1.1e-5 to 1.5e-5 of the
// result's norm on Gaussian operands and on activations after a ReLU, and 4.1e-5 in a weight's gradient from such activations
// with rows of very different size (4096 deep); an output of 16 bits hides it (its own rounding is 1.7e-3 or 2.1e-4: 1 to
// 2 % of 4096 x 4096 bf16 results are the neighbour of what exact sums round to) and one of 32 does not: there the bytes are
// decoded to bf16 between LDS and the 16-bit instruction, which is exact.
//
// What bounds it.  4096 x 4096 x 25088 in 8 bits takes 310 to 335 us (2.5 to 2.7 PFLOP/s; torch's 8-bit product with one scale
// for all reaches 2.9 at 8192^3, where this takes 415 to 425 us, 2.6): the clock falls to 1.86 GHz under it, the matrix
// cores are busy 61 % of the cycles, LDS 18 %.  Without the direct loads it would take 267, without the reads from LDS 274: a
// single wave a SIMD issues them between its matrix instructions.  Loads spread over both halves of a block (1 to 3 %
// faster) would take 160 KB of LDS in five turns; eight waves a workgroup, two a SIMD, were 3 to 6 % slower.  4096^3
// takes 58.5: about 50 for its blocks and 9 for the first loads and the stores at the end, which nothing overlaps.
// The exact form is bound by the same and by decoding (4096^3 110 us, 1.25 PFLOP/s, where torch's bf16 product takes 94;
// 25088 x 4096 x 4096 640), small products by the latency of their blocks.
#include <type_traits>

#include "kq_block.h"

namespace kq {

using f32x16 = __attribute__((ext_vector_type(16))) float;
using i32x8 = __attribute__((ext_vector_type(8))) int;
using i32x2 = __attribute__((ext_vector_type(2))) int;
using i32x2_lds = __attribute__((address_space(3))) i32x2*;

// Chunk ch (16 bytes) of row r of a block, rows of 128 bytes.  A fragment's read is free of bank conflicts where the chunks
// c and c + 2 of eight neighbouring rows, and one chunk of sixteen, fall on sixteen different 16-byte columns of the 64 banks.
__device__ __forceinline__ int block_swizzle(int r) { return (r >> 1 & 1) | (r >> 3 & 1) << 1 | (r >> 2 & 1) << 2; }
__device__ __forceinline__ int block_chunk(int r, int ch) { return r * 8 + (ch ^ block_swizzle(r)); }

// A block's rows from memory to LDS: a wave's instruction takes 64 chunks, eight whole cache lines.
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
            off[t] = (unsigned)min(r, last) * (unsigned)o.pitch + 16 * ((lane & 7) ^ block_swizzle(r));
        }
    }
    __device__ __forceinline__ void load(const uint8_t* base, u32x4* lds, int wave) const {
#pragma unroll
        for (int t = 0; t < N; ++t)
            __builtin_amdgcn_global_load_lds((global_ptr)(base + off[t]), (lds_ptr)(lds + (t * WAVES + wave) * 64), 16, 0, 0);
    }
};

// The same of an operand that lies transposed, BI neighbouring columns of its 128 rows of a block: the contraction's rows past
// the last repeat it (the other operand has zeros there, and a NaN makes the whole block of its columns NaN).
// Chunk ch of contraction row r lies at ch ^ column_swizzle(r): eight neighbouring rows of two chunks are on all banks.
template <int BI>
__device__ __forceinline__ int column_swizzle(int r) { return BI == 256 ? (r & 7) * 2 : (r >> 1 & 3) * 2; }
template <int BI, int WAVES>
struct DirectColumns {
    static constexpr int N = BI / 8 / WAVES, kChunks = BI / 16, kRows = 64 / kChunks;  // chunks of a row, rows of an instruction
    static_assert((kRows * WAVES) % 8 == 0, "a lane's rows have one swizzle, so one column");
    unsigned off[N], column;  // (of 128 rows and a pitch up to 2^24: below 2^32)
    unsigned pitch;
    int64_t depth;
    __device__ __forceinline__ void init(const BlockOperand& o, int64_t i0, int64_t cols, int64_t depth_, int lane, int wave) {
        pitch = (unsigned)o.pitch;
        depth = depth_;
        const int r = wave * kRows + lane / kChunks;
        column = (unsigned)min(i0 + 16 * ((lane % kChunks) ^ column_swizzle<BI>(r)), cols - 16);  // (columns past the last: not stored)
#pragma unroll
        for (int t = 0; t < N; ++t) off[t] = (unsigned)(r + t * WAVES * kRows) * pitch + column;
    }
    __device__ __forceinline__ void load(const uint8_t* values, int b, u32x4* lds, int wave) const {
        const uint8_t* base = values + (int64_t)b * kBlock * pitch;
        const unsigned last = (unsigned)min(depth - 1 - (int64_t)b * kBlock, (int64_t)kBlock - 1) * pitch + column;
#pragma unroll
        for (int t = 0; t < N; ++t)
            __builtin_amdgcn_global_load_lds((global_ptr)(base + min(off[t], last)), (lds_ptr)(lds + (t * WAVES + wave) * 64), 16, 0, 0);
    }
};

// The exponents of a lane's rows, one a row and block: eight blocks at a time, the lowest byte the current block's.
template <int N>
struct RowExponents {
    u32x2 now[N], next[N];
    unsigned off[N];
    const uint8_t* base;
    int steps, end;
    __device__ __forceinline__ void init(const BlockOperand& o, int64_t row0, int64_t rows, int lane, int steps_, int end_) {
        const int64_t first = min(row0, rows - 1);
        base = o.e + first * o.e_row;
        steps = steps_;
        end = end_;
#pragma unroll
        for (int t = 0; t < N; ++t) off[t] = (unsigned)(min(row0 + 32 * t + lane, rows - 1) - first) * (unsigned)o.e_row;
    }
    // (steps of eight and more: bytes as they lie, nothing behind a row's end; take() moves them, so that the loads have
    // time until then)
    __device__ __forceinline__ void load(int b) {
        if (b >= end) return;
        if (steps >= 8) {
            const unsigned from = (unsigned)min(b, steps - 8);
#pragma unroll
            for (int t = 0; t < N; ++t) __builtin_memcpy(&next[t], base + (off[t] + from), 8);
        } else {
#pragma unroll
            for (int t = 0; t < N; ++t) {
                uint64_t v = 0;
                for (int i = b; i < end; ++i) v |= (uint64_t)base[off[t] + (unsigned)i] << (8 * (i - b));
                next[t] = u32x2{(unsigned)v, (unsigned)(v >> 32)};
            }
        }
    }
    __device__ __forceinline__ void take(int b) {
        const int skip = steps >= 8 ? b - min(b, steps - 8) : 0, left = min(end - b, 8);
        const uint64_t mask = ~uint64_t(0) >> (8 * (8 - left));
#pragma unroll
        for (int t = 0; t < N; ++t) {
            const uint64_t v = (((uint64_t)next[t].y << 32 | next[t].x) >> (8 * skip)) & mask;
            now[t] = u32x2{(unsigned)v, (unsigned)(v >> 32)};
        }
    }
    template <int BLOCKS>
    __device__ __forceinline__ void shift() {
#pragma unroll
        for (int t = 0; t < N; ++t) now[t] = BLOCKS == 4 ? u32x2{now[t].y, 0u} : u32x2{__builtin_amdgcn_alignbit(now[t].y, now[t].x, 16), now[t].y >> 16};
    }
};

// s_waitcnt's operand: at most `vm` vector memory and `lgkm` LDS operations left
constexpr int waitcnt(int vm, int lgkm) { return (vm & 15) | (vm >> 4) << 14 | 7 << 4 | lgkm << 8; }

// 32 rows of COLS fp32 values in LDS (pitch COLS + 4) to rows j0 .. of out, 16 bytes a lane.  `stream`: past the caches'
// normal ways.
template <int TYPE, int COLS>
__device__ __forceinline__ void store_rows(const float* rows, char* out, int64_t ld, int64_t j0, int64_t i0, int64_t J, int64_t I,
                                           const float* bias, bool stream, int lane) {
    using u32x4_any = __attribute__((ext_vector_type(4), aligned(2))) unsigned;
    constexpr int N = TYPE == KQ_T_F32 ? 4 : 8, kBytes = 16 / N, kLanes = COLS / N, kRows = 64 / kLanes;
    const int c = lane % kLanes * N;
    const int64_t i = i0 + c;
    if (i >= I) return;
    const bool whole = i + N <= I;
    float add[N];
#pragma unroll
    for (int t = 0; t < N; ++t) add[t] = bias && i + t < I ? bias[i + t] : 0.0f;
#pragma unroll 4
    for (int r = lane / kLanes; r < 32; r += kRows) {
        if (j0 + r >= J) break;
        float v[N];
#pragma unroll
        for (int t = 0; t < N; t += 4) {
            const f32x4 q = *(const f32x4*)(rows + r * (COLS + 4) + c + t);
#pragma unroll
            for (int u = 0; u < 4; ++u) v[t + u] = q[u] + add[t + u];
        }
        char* const o = out + ((j0 + r) * ld + i) * kBytes;
        unsigned w[4];
        if constexpr (TYPE == KQ_T_F32) {
            __builtin_memcpy(w, v, 16);
        } else {
#pragma unroll
            for (int t = 0; t < 4; ++t) w[t] = Act<TYPE == KQ_T_BF16>::pack(v[2 * t], v[2 * t + 1]);
        }
        if (whole && stream) {
            __builtin_nontemporal_store((u32x4_any){w[0], w[1], w[2], w[3]}, (u32x4_any*)o);
        } else if (whole) {
            __builtin_memcpy(o, w, 16);
        } else {
#pragma unroll
            for (int t = 0; t < N; ++t)
                if (i + t < I) {
                    if constexpr (TYPE == KQ_T_F32) ((float*)o)[t] = v[t];
                    else ((uint16_t*)o)[t] = (uint16_t)(w[t >> 1] >> (16 * (t & 1)));
                }
        }
    }
}

template <bool EXACT, int FORM, int BI, int BJ, int WI, int WJ, int RING>
__global__ __launch_bounds__(64 * WI * WJ, 1) void block_gemm_kernel(const BlockGemmParams p) {
    constexpr bool AROWS = FORM == kFormRows, COLUMNS = FORM == kFormColumns;
    constexpr int MI = BI / WI / 32, MJ = BJ / WJ / 32, WAVES = WI * WJ;
    static_assert(MI * 32 <= kBlock, "a wave's rows of A lie in one block");
    // (arrays of their own, so that the compiler can tell the direct loads' target from what is read beside them)
    __shared__ u32x4 s_0[(BI + BJ) * 8];
    __shared__ u32x4 s_1[(BI + BJ) * 8];
    __shared__ u32x4 s_2[RING > 2 ? (BI + BJ) * 8 : 1];
    __shared__ u32x4 s_3[RING > 2 ? (BI + BJ) * 8 : 1];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wi = wave % WI, wj = wave / WI, r32 = lane & 31, half = lane >> 5;
    const int tile = xcd_tile(blockIdx.x, p.itiles * p.jtiles);
    // An XCD's tiles are neighbours in both directions: columns of kGroup tiles, so that its 32 CUs read 8 + 4 tiles' rows.
    constexpr int kGroup = 4;
    const int column = tile / (p.itiles * kGroup), in = tile - column * p.itiles * kGroup;
    const int width = min(kGroup, p.jtiles - column * kGroup);
    const int64_t i0 = (int64_t)(in / width) * BI, j0 = (int64_t)(column * kGroup + in % width) * BJ;
    const int64_t iw = i0 + wi * MI * 32, jw = j0 + wj * MJ * 32;  // the wave's part

    f32x16 acc[MI][MJ];
#pragma unroll
    for (int a = 0; a < MI; ++a)
#pragma unroll
        for (int b = 0; b < MJ; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[a][b][r] = 0.0f;

    const int b_begin = blockIdx.y * p.steps_per_split, b_end = min(b_begin + p.steps_per_split, p.steps);
    std::conditional_t<COLUMNS, DirectColumns<BI, WAVES>, DirectRows<BI, WAVES>> la;
    DirectRows<BJ, WAVES> lb;
    if constexpr (COLUMNS) la.init(p.A, i0, p.a_cols, p.depth, lane, wave);
    else la.init(p.A, i0, p.I, lane, wave);
    lb.init(p.B, j0, p.J, lane, wave);
    const uint8_t* const a_base = COLUMNS ? p.A.v : p.A.v + i0 * p.A.pitch;
    const uint8_t* const b_base = p.B.v + j0 * p.B.pitch;
    // Exponents.  Of an operand with one a row a lane holds eight blocks' at a time, and loads the next eight four blocks
    // before they are needed (a byte for each of the next two blocks, two blocks before, each row's cache line comes back again
    // and again: 4096 x 4096 x 25088, of one operand 314 to 320 us instead of 303 to 308, of both, a weight's gradient,
    // 477 to 490 instead of 402).  Of the 128 x 128 form lane l holds block l's of 64.  Blocks behind the last have 0.
    RowExponents<AROWS ? MI : 1> ea;
    RowExponents<MJ> eb;
    if constexpr (AROWS) ea.init(p.A, iw, p.I, r32, p.steps, b_end);
    eb.init(p.B, jw, p.J, r32, p.steps, b_end);
    const uint8_t* const block_exps = p.A.e + (min(iw, p.I - 1) >> 7) * p.A.e_row;
    auto load_block_exps = [&](int first) {
        const int b = first + lane;
        return b < b_end ? (unsigned)block_exps[b * p.A.e_col] : 0u;
    };
    unsigned block_exp = 0;

    struct Fragments {
        u32x4 a[MI][2], b[MJ][2];
    };
    // Where a lane reads a block's first half, in rows and of columns.  (Opaque, so that an address is a step or two from its
    // array: of longer ones the compiler does not know the array, and waits for all direct loads.)
    unsigned rows_at[2] = {(unsigned)block_chunk(r32, 2 * half), (unsigned)block_chunk(r32, 2 * half + 1)};
    asm("" : "+v"(rows_at[0]), "+v"(rows_at[1]));
    unsigned columns_at = (32 * half + (r32 % 16 >> 1)) * BI + 8 * (lane & 1) + 16 * ((wi * MI * 2 + (r32 >> 4)) ^ column_swizzle<BI>(r32 % 16 >> 1));
    if constexpr (COLUMNS) asm("" : "+v"(columns_at));
    // (past the end the last block again: nobody reads it)
    auto load_block = [&](int b, u32x4* to) {
        const int block = min(b, b_end - 1);
        if constexpr (COLUMNS) la.load(a_base, block, to, wave);
        else la.load(a_base + (int64_t)block * kBlock, to, wave);
        lb.load(b_base + (int64_t)block * kBlock, to + BI * 8, wave);
    };
    auto read_fragments = [&](const u32x4* from, int h, Fragments& f) {
        // (32 rows on: the same swizzle)
        const unsigned c0 = rows_at[0] ^ 4 * h, c1 = rows_at[1] ^ 4 * h, a_first = wi * MI * 256, b_first = BI * 8 + wj * MJ * 256;
#pragma unroll
        for (int a = 0; a < MI; ++a) {
            if constexpr (COLUMNS) {
#pragma unroll
                for (int t = 0; t < 4; ++t) {  // 8 rows of 16 columns for 16 lanes: lane i gets column i
                    const i32x2 v = __builtin_amdgcn_ds_read_tr8_b64_v2i32((i32x2_lds)((const char*)from + ((columns_at ^ 32 * a) + (64 * h + 8 * t) * BI)));
                    f.a[a][t >> 1][2 * (t & 1)] = (unsigned)v[0];
                    f.a[a][t >> 1][2 * (t & 1) + 1] = (unsigned)v[1];
                }
            } else {
                f.a[a][0] = from[a_first + c0 + a * 256];
                f.a[a][1] = from[a_first + c1 + a * 256];
            }
        }
#pragma unroll
        for (int b = 0; b < MJ; ++b) {
            f.b[b][0] = from[b_first + c0 + b * 256];
            f.b[b][1] = from[b_first + c1 + b * 256];
        }
    };
    // BYTE: which of the lane's exponents; xa: A's in the 128 x 128 form
    auto multiply = [&](const Fragments& f, unsigned xa, auto byte) {
        constexpr int BYTE = decltype(byte)::value;
        if constexpr (!EXACT) {
            auto join = [](const u32x4 (&c)[2]) {
                return i32x8{(int)c[0][0], (int)c[0][1], (int)c[0][2], (int)c[0][3], (int)c[1][0], (int)c[1][1], (int)c[1][2], (int)c[1][3]};
            };
#pragma unroll
            for (int a = 0; a < MI; ++a)
#pragma unroll
                for (int b = 0; b < MJ; ++b)
                    acc[a][b] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
                        join(f.a[a]), join(f.b[b]), acc[a][b], 0, 0, AROWS ? BYTE : 0, AROWS ? (int)ea.now[AROWS ? a : 0].x : (int)xa, BYTE, (int)eb.now[b].x);
        } else {
            float sa[MI], sb[MJ];
#pragma unroll
            for (int a = 0; a < MI; ++a) sa[a] = checkpoint_step(AROWS ? ea.now[AROWS ? a : 0].x >> (8 * BYTE) & 255u : xa);
#pragma unroll
            for (int b = 0; b < MJ; ++b) sb[b] = checkpoint_step(eb.now[b].x >> (8 * BYTE) & 255u);
#pragma unroll
            for (int u = 0; u < 4; ++u) {  // 16 of the contraction
                bf16x8 ad[MI], bd[MJ];
#pragma unroll
                for (int a = 0; a < MI; ++a)
                    ad[a] = __builtin_bit_cast(bf16x8, decode8(f.a[a][u >> 1][2 * (u & 1)], f.a[a][u >> 1][2 * (u & 1) + 1], sa[a]));
#pragma unroll
                for (int b = 0; b < MJ; ++b)
                    bd[b] = __builtin_bit_cast(bf16x8, decode8(f.b[b][u >> 1][2 * (u & 1)], f.b[b][u >> 1][2 * (u & 1) + 1], sb[b]));
#pragma unroll
                for (int a = 0; a < MI; ++a)
#pragma unroll
                    for (int b = 0; b < MJ; ++b) acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ad[a], bd[b], acc[a][b], 0, 0, 0);
            }
        }
    };
    // Half a block is multiplied from registers while the next half's fragments are read from LDS.  Between a block's halves
    // every wave has read the second one's fragments, and the next block has to be there: one barrier a block.  After it the
    // block's place takes the one RING blocks on, which has until then.  Four places instead of two where a CU has one workgroup
    // all the same and the loads come from memory (4096 x 128 x 25088, 64 workgroups: 79 us, 112 with two; 4096 x 512 x 4096,
    // 256 workgroups: 18.0 and 23.1; of 64 workgroups with the operands in the L2s 13.7 and 14.5).
    constexpr int PER = DirectRows<BI, WAVES>::N + DirectRows<BJ, WAVES>::N;
    // A matrix instruction, then its share of the reads and loads: they issue while it runs.  The reads go with the first half
    // of the instructions, so that LDS has answered at the end; the loads with all of them, since they hold up the wave
    // where they come faster than one a matrix instruction (4096 x 4096 x 25088: 310 us, 320 at two, 318 with the reads
    // spread too).
    auto in_turn = [&](auto loads) {
        constexpr int kMatrix = MI * MJ * (EXACT ? 4 : 1), kReads = (COLUMNS ? 4 : 2) * MI + 2 * MJ, kLoads = decltype(loads)::value ? PER : 0;
        int reads = 0, sent = 0;
#pragma unroll
        for (int t = 0; t < kMatrix; ++t) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            const int r = min(kReads, (2 * (t + 1) * kReads + kMatrix - 1) / kMatrix), l = (t + 1) * kLoads / kMatrix;
            for (; reads < r; ++reads) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            for (; sent < l; ++sent) __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);
        }
    };
    Fragments f0, f1;
    auto block = [&](int b, unsigned xa, auto byte, u32x4* now, u32x4* next) {
        __builtin_amdgcn_sched_barrier(0);
        read_fragments(now, 1, f1);
        multiply(f0, xa, byte);
        in_turn(std::false_type{});
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(waitcnt((RING - 2) * PER, 0));
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        load_block(b + RING, now);
        read_fragments(next, 0, f0);
        multiply(f1, xa, byte);
        in_turn(std::true_type{});
        __builtin_amdgcn_sched_barrier(0);
    };
    if (b_begin < b_end) {
        if constexpr (AROWS) ea.load(b_begin);
        eb.load(b_begin);
        if constexpr (!AROWS) block_exp = load_block_exps(b_begin);
        load_block(b_begin, s_0);
        load_block(b_begin + 1, s_1);
        if constexpr (RING > 2) {
            load_block(b_begin + 2, s_2);
            load_block(b_begin + 3, s_3);
        }
        __builtin_amdgcn_s_waitcnt(waitcnt((RING - 1) * PER, 15));
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        read_fragments(s_0, 0, f0);
        // RING blocks a turn.  Behind an odd last one comes the same block again, with exponents of zero on both sides: its
        // products are below 2^-220, nothing in fp32.  (A branch there made the compiler move the accumulators about.)
        constexpr int kTurns = 8 / RING;
        auto block_byte = [&](int t, int i) { return AROWS ? 0u : (unsigned)__builtin_amdgcn_readlane(block_exp, (RING * t + i) & 63); };
        for (int b = b_begin, t = 0; b < b_end; b += RING, ++t) {
            if (t % kTurns == 0) {
                if constexpr (AROWS) ea.take(b);
                eb.take(b);
                if (!AROWS && t % (8 * kTurns) == 0 && t > 0) block_exp = load_block_exps(b);
            }
            if (t % kTurns == kTurns / 2) {
                if constexpr (AROWS) ea.load(b + 4);
                eb.load(b + 4);
            }
            if constexpr (RING == 2) {
                const unsigned xa0 = block_byte(t, 0), xa1 = block_byte(t, 1);
                block(b, xa0, std::integral_constant<int, 0>{}, s_0, s_1);
                block(b + 1, xa1, std::integral_constant<int, 1>{}, s_1, s_0);
            } else {
                const unsigned xa0 = block_byte(t, 0), xa1 = block_byte(t, 1), xa2 = block_byte(t, 2), xa3 = block_byte(t, 3);
                block(b, xa0, std::integral_constant<int, 0>{}, s_0, s_1);
                block(b + 1, xa1, std::integral_constant<int, 1>{}, s_1, s_2);
                if (b + 2 >= b_end) break;
                block(b + 2, xa2, std::integral_constant<int, 2>{}, s_2, s_3);
                block(b + 3, xa3, std::integral_constant<int, 3>{}, s_3, s_0);
            }
            if constexpr (AROWS) ea.template shift<RING>();
            eb.template shift<RING>();
        }
        __builtin_amdgcn_s_waitcnt(waitcnt(0, 0));  // (no load may arrive in LDS after the workgroup's end)
    }

    if constexpr (AROWS) {  // the bias' gradient from its partial sums, once
        if (p.dbias && i0 == 0 && blockIdx.y == 0) {
            for (int64_t j = j0 + tid; j < min(j0 + BJ, p.J); j += 64 * WAVES) {
                float v = 0.0f;
#pragma unroll 16
                for (int t = 0; t < p.bias_parts; ++t) v += p.bias_part[(int64_t)t * p.J + j];
                p.dbias[j] = v;
            }
        }
    }

    // Lane holds out[j][i .. i + 3] for j = its column, i = 8 g + 4 half of a 32 x 32 tile: neighbours by fours, rows apart.
    // They go through LDS, 32 rows of the wave at a time in a part of its own, and leave as whole rows (of 4096 x 4096
    // bf16, stored by fours: 11 us).
    __syncthreads();  // (every wave has read its last fragments)
    constexpr int kCols = MI * 32, kPitch = kCols + 4;
    constexpr int kPart = (BI + BJ) * 64;  // bytes, half a block
    static_assert(kPart >= 32 * kPitch * 4 && WAVES <= 4, "a part for each wave");
    float* const rows = (float*)((char*)(wave < 2 ? s_0 : s_1) + (wave & 1) * kPart);
    const bool f32 = p.part || p.type == KQ_T_F32;
    char* const base = p.part ? (char*)(p.part + (int64_t)blockIdx.y * p.J * p.I) : (char*)p.out;
    const int64_t ld = p.part ? p.I : p.ldo;
    // (results that the L2s do not hold: 4096 x 4096 x 4096 bf16 60.6 us, 58.8 streamed; 25088 x 4096 fp32 667 and 637)
    const bool stream = !p.part && p.J * p.I >= (f32 ? 1 << 22 : 1 << 23);
#pragma unroll
    for (int b = 0; b < MJ; ++b) {
#pragma unroll
        for (int a = 0; a < MI; ++a)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *(f32x4*)(rows + r32 * kPitch + 32 * a + 8 * g + 4 * half) =
                    f32x4{acc[a][b][4 * g], acc[a][b][4 * g + 1], acc[a][b][4 * g + 2], acc[a][b][4 * g + 3]};
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (f32) store_rows<KQ_T_F32, kCols>(rows, base, ld, jw + 32 * b, iw, p.J, p.I, p.part ? nullptr : p.bias, stream, lane);
        else if (p.type == KQ_T_BF16) store_rows<KQ_T_BF16, kCols>(rows, base, ld, jw + 32 * b, iw, p.J, p.I, p.bias, stream, lane);
        else store_rows<KQ_T_F16, kCols>(rows, base, ld, jw + 32 * b, iw, p.J, p.I, p.bias, stream, lane);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// The tile and the splits with the shortest modelled time.  A workgroup's block of the contraction takes `few` us where few
// CUs have one, `full` where all 256 have (the clock and the caches give way), and a CU with n of them n times `shared`; a
// split contraction pays the joining launch and its partial sums, written and read at about 6 MB a us.  Where the tiles of
// 256 x 256 are a little over a number of full rounds, the columns of the last one are a product of their own (98 x 16 tiles
// of 4096 deep: six rounds and 128 small tiles instead of seven).  What a whole contraction's results take to store is in the
// fixed part, once however many rounds there are; so large results of one to four blocks take longer than it says (exact,
// 25088 x 4096 of two blocks 115 us for 50, of four 177 for 90; 4096 x 4096 21 to 29 for 12, 28 for 19), and which tile is
// the fastest there has not been measured.  Fitted to sweeps, all 4096 deep, us for one output size, 8-bit / exact:
//   4096 x 256:  128x64 14.8 / 20.8, 128x128 18.1 / 21.5 (four splits), 256x256 28 / 33
//   4096 x 1024: 128x64 25.5 / 38.3, 128x128 25.1 / 39.3, 256x256 40 / 51
//   4096 x 2048: 128x64 50.6 / 71.0, 128x128 35.4 / 61.6, 256x256 52.7 / 75.8
//   4096 x 4096: 128x64 95, 128x128 78 / 132, 256x256 59.8 / 110
struct BlockTileTime {
    int bi, bj;
    float fixed;
    float few[2], full[2], shared[2];  // 8-bit, exact
};
constexpr BlockTileTime kTiles[] = {
    {128, 64, 4.0f, {0.30f, 0.33f}, {0.44f, 0.74f}, {0.365f, 0.53f}},
    {128, 128, 5.0f, {0.33f, 0.50f}, {0.63f, 1.10f}, {0.53f, 0.90f}},
    {256, 256, 9.0f, {0.55f, 1.00f}, {1.59f, 3.15f}, {1.59f, 3.10f}},
};

static float block_time(const BlockTileTime& t, bool exact, int64_t workgroups) {
    if (workgroups <= 256) return t.few[exact] + (t.full[exact] - t.few[exact]) * (float)workgroups / 256.0f;
    const float shared = (float)ceil_div64(workgroups, 256) * t.shared[exact];
    return shared > t.full[exact] ? shared : t.full[exact];
}

static BlockGemmPlan one_plan(bool exact, int64_t I, int64_t J, int64_t steps, bool may_split, float& best) {
    BlockGemmPlan g = {};
    const float value_us = (float)I * (float)J * 8.0f / 6e6f;
    best = 0.0f;
    int64_t splits = 1;
    for (const BlockTileTime& t : kTiles) {
        const int64_t tiles = ceil_div64(I, t.bi) * ceil_div64(J, t.bj);
        for (int s = 1; s <= 32 && (s == 1 || (may_split && s * 4 <= steps && s * tiles <= 1024)); s = s < 4 ? s + 1 : s * 3 / 2) {
            const float us = t.fixed + (float)ceil_div64(steps, s) * block_time(t, exact, tiles * s) + (s > 1 ? 2.5f + (float)s * value_us : 0.0f);
            if (g.bi == 0 || us < best) {
                best = us;
                g.bi = t.bi;
                g.bj = t.bj;
                splits = s;
            }
        }
    }
    // (an even number of blocks a split: the kernel takes two at a time)
    const int64_t per = splits > 1 ? ceil_div64(ceil_div64(steps, splits), 2) * 2 : steps;
    g.steps_per_split = (int)(per ? per : 1);
    g.splits = steps ? (int)ceil_div64(steps, g.steps_per_split) : 1;
    return g;
}

BlockGemmPlan block_gemm_plan(bool exact, int64_t I, int64_t J, int64_t C) {
    const int64_t steps = block_pitch(C) / kBlock;
    float best;
    BlockGemmPlan g = one_plan(exact, I, J, steps, true, best);
    g.us = best;
    g.part_bytes = g.splits > 1 ? ((size_t)g.splits * (size_t)(I * J) * sizeof(float) + 255) & ~size_t(255) : 0;
    const int64_t jtiles = ceil_div64(J, 256), rounds = ceil_div64(I, 256) * jtiles / 256;
    const int64_t itiles = rounds * 256 / jtiles, rest = I - itiles * 256;
    if (rounds > 0 && rest > 0) {
        float rest_us;
        const BlockGemmPlan r = one_plan(exact, rest, J, steps, false, rest_us);
        const float us = 9.0f + (float)rounds * kTiles[2].shared[exact] * (float)steps + rest_us;
        if (us < best) {
            g = {256, 256, 1, (int)(steps ? steps : 1), 0, itiles * 256, r.bi, r.bj, us};
        }
    }
    return g;
}

template <bool EXACT, int FORM>
static hipError_t launch_tile(int bi, int bj, BlockGemmParams p, hipStream_t s) {
    p.itiles = (int)ceil_div64(p.I, bi);
    p.jtiles = (int)ceil_div64(p.J, bj);
    const dim3 grid((unsigned)((int64_t)p.itiles * p.jtiles), (unsigned)p.splits);
    const int tile = bi * 1000 + bj;
    // (four places for the decoding form only where that paid: 25088 x 64 x 4096 28.1 us, 33.9 with two, but 4096 x 256 x 4096
    // 23.9 and 22.2; of 128 x 128 tiles 25.1 and 28.4 with 256 workgroups, 19.4 and 18.5 with 64)
    const int64_t workgroups = (int64_t)grid.x * grid.y;
    const bool alone = workgroups <= 256, many = workgroups > 128;
    if (tile == 256256) {
        block_gemm_kernel<EXACT, FORM, 256, 256, 2, 2, 2><<<grid, dim3(256), 0, s>>>(p);
    } else if (tile == 128128) {
        if constexpr (!EXACT) {
            if (alone && many) {
                block_gemm_kernel<EXACT, FORM, 128, 128, 2, 2, 4><<<grid, dim3(256), 0, s>>>(p);
                return hipGetLastError();
            }
        }
        block_gemm_kernel<EXACT, FORM, 128, 128, 2, 2, 2><<<grid, dim3(256), 0, s>>>(p);
    } else if (tile == 128064) {
        if (alone && (!EXACT || many || p.steps_per_split > 128)) block_gemm_kernel<EXACT, FORM, 128, 64, 2, 2, 4><<<grid, dim3(256), 0, s>>>(p);
        else block_gemm_kernel<EXACT, FORM, 128, 64, 2, 2, 2><<<grid, dim3(256), 0, s>>>(p);
    } else {
        return hipErrorInvalidValue;
    }
    return hipGetLastError();
}
template <bool EXACT>
static hipError_t launch_as(int form, int bi, int bj, const BlockGemmParams& p, hipStream_t s) {
    if (form == kFormRows) return launch_tile<EXACT, kFormRows>(bi, bj, p, s);
    if (form == kFormColumns) return launch_tile<EXACT, kFormColumns>(bi, bj, p, s);
    return launch_tile<EXACT, kFormBlocks>(bi, bj, p, s);
}
static hipError_t launch_form(bool exact, int form, int bi, int bj, const BlockGemmParams& p, hipStream_t s) {
    return exact ? launch_as<true>(form, bi, bj, p, s) : launch_as<false>(form, bi, bj, p, s);
}

hipError_t launch_block_gemm(bool exact, int form, const BlockGemmPlan& plan, BlockGemmParams p, void* part, hipStream_t s) {
    p.splits = plan.splits;
    p.steps_per_split = plan.steps_per_split;
    p.part = plan.splits > 1 ? (float*)part : nullptr;
    if (plan.rest_from > 0) {  // (a multiple of 256: whole blocks of A's exponents)
        BlockGemmParams r = p;
        r.I = p.I - plan.rest_from;
        r.A.v += form == kFormColumns ? plan.rest_from : plan.rest_from * p.A.pitch;
        r.a_cols = p.a_cols - plan.rest_from;
        r.A.e += (form == kFormRows ? plan.rest_from : plan.rest_from >> 7) * p.A.e_row;
        r.out = (char*)p.out + plan.rest_from * (p.type == KQ_T_F32 ? 4 : 2);
        if (p.bias) r.bias = p.bias + plan.rest_from;
        r.dbias = nullptr;
        p.I = plan.rest_from;
        const hipError_t e = launch_form(exact, form, plan.bi, plan.bj, p, s);
        return e != hipSuccess ? e : launch_form(exact, form, plan.rest_bi, plan.rest_bj, r, s);
    }
    const hipError_t e = launch_form(exact, form, plan.bi, plan.bj, p, s);
    if (e != hipSuccess || plan.splits == 1) return e;
    const JoinParams j = {p.part, p.splits, p.J, p.I, p.bias, p.out, p.ldo, p.type};
    return launch_join(j, s);
}

}  // namespace kq
