// The 4-bit group quantizer, the weights it stands for, 8-bit activation checkpoints and the sums of
// split products: passes over memory.
#include "kq_group.h"

namespace kq {

// ---- element access by type --------------------------------------------------------------------------

// N consecutive values at any alignment of their type, as fp32
template <int TYPE, int N>
__device__ __forceinline__ void load_values(const void* base, int64_t at, float (&v)[N]) {
    if constexpr (TYPE == KQ_T_F32) {
        __builtin_memcpy(v, (const float*)base + at, 4 * N);
    } else {
        unsigned h[N / 2];
        __builtin_memcpy(h, (const uint16_t*)base + at, 2 * N);
#pragma unroll
        for (int t = 0; t < N / 2; ++t) {
            v[2 * t] = Act<TYPE == KQ_T_BF16>::lo(h[t]);
            v[2 * t + 1] = Act<TYPE == KQ_T_BF16>::hi(h[t]);
        }
    }
}
template <int TYPE>
__device__ __forceinline__ float load_value_as(const void* base, int64_t at) {
    if constexpr (TYPE == KQ_T_F32) return ((const float*)base)[at];
    else return Act<TYPE == KQ_T_BF16>::lo(((const uint16_t*)base)[at]);
}
// 4-byte aligned pieces of a stream that is written once and not read soon: past the caches' normal ways
// (fp32 weights of 4096 x 25088 rebuilt: 75 us, 131 us with ordinary stores).
__device__ __forceinline__ void stream_store(void* at, const unsigned* v, int words) {
    if (words == 4) {
        using u32x4_a4 = __attribute__((ext_vector_type(4), aligned(4))) unsigned;
        __builtin_nontemporal_store((u32x4_a4){v[0], v[1], v[2], v[3]}, (u32x4_a4*)at);
    } else {
        using u32x2_a4 = __attribute__((ext_vector_type(2), aligned(4))) unsigned;
        __builtin_nontemporal_store((u32x2_a4){v[0], v[1]}, (u32x2_a4*)at);
    }
}

template <int TYPE, int N>
__device__ __forceinline__ void store_values(void* base, int64_t at, const float (&v)[N], int count) {
    if constexpr (TYPE == KQ_T_F32) {
        float* o = (float*)base + at;
        if (count >= N) {
            unsigned h[N];
            __builtin_memcpy(h, v, 4 * N);
#pragma unroll
            for (int t = 0; t < N; t += 4) stream_store(o + t, h + t, 4);
        } else {
#pragma unroll
            for (int t = 0; t < N; ++t)
                if (t < count) o[t] = v[t];
        }
    } else {
        uint16_t* o = (uint16_t*)base + at;
        if (count >= N) {
            unsigned h[N / 2];
#pragma unroll
            for (int t = 0; t < N / 2; ++t) h[t] = Act<TYPE == KQ_T_BF16>::pack(v[2 * t], v[2 * t + 1]);
            if (((uintptr_t)o & 3) == 0) stream_store(o, h, N / 2);
            else __builtin_memcpy(o, h, 2 * N);
        } else {
#pragma unroll
            for (int t = 0; t < N; ++t)
                if (t < count) o[t] = Act<TYPE == KQ_T_BF16>::one(v[t]);
        }
    }
}

// 8 columns at c0 of a row, zeros past the row's `limit`
template <int TYPE>
__device__ __forceinline__ void load_columns(const void* base, int64_t row_at, int c0, int limit, float (&v)[8]) {
    if (c0 + 8 <= limit) {
        load_values<TYPE, 8>(base, row_at + c0, v);
    } else {
#pragma unroll
        for (int t = 0; t < 8; ++t) v[t] = c0 + t < limit ? load_value_as<TYPE>(base, row_at + c0 + t) : 0.0f;
    }
}

// max |v| as fp32 bits without the sign: an infinity or NaN is larger than every finite value
__device__ __forceinline__ unsigned max_bits(const float (&v)[8]) {
    unsigned a = 0;
#pragma unroll
    for (int t = 0; t < 8; ++t) {
        const unsigned b = __builtin_bit_cast(unsigned, v[t]) & 0x7fffffffu;
        a = b > a ? b : a;
    }
    return a;
}

// ---- quantizer -----------------------------------------------------------------------------------------
// A workgroup a 16 x 128 tile, sixteen lanes a row, 8 neighbouring columns and one dword of codes a lane, four rows a
// wave: a row's lanes read contiguous memory, and a group's columns lie in 4, 8 or 16 neighbouring lanes.
// Per group: a = max |w| (a non-finite value is larger than every other), s = bf16(a / top) with top = 7 or
// the largest |level| (zero below the normal range, NaN where a is not finite), and per weight t = w / s in
// fp32 and the nearest level to t, the lower one of two that are as near: for -8 .. 7 by rounding, for a
// table by a binary search of the midpoints of neighbouring levels for the number below t.
// A true division takes about ten instructions, so t is first w times the reciprocal, whose error is below
// 2^-21 |t|; only where that is too near a midpoint (or the scale is outside 2^-100 .. 2^100) is the weight
// divided, in a branch that a few waves in a hundred take.
__device__ __forceinline__ unsigned nearest_integer_code(float t) {
    float r = __builtin_rintf(t);       // ties to even
    if (r - t == 0.5f) r -= 1.0f;       // a tie that went up
    r = __builtin_fminf(__builtin_fmaxf(r, -8.0f), 7.0f);
    return (unsigned)((int)r + 8);
}
// mid[1 .. 15]: the midpoints of neighbouring levels
__device__ __forceinline__ unsigned nearest_level_code(float t, const float* mid) {
    unsigned code = 0;
#pragma unroll
    for (int step = 8; step >= 1; step >>= 1) code += t > mid[code + step] ? step : 0;
    return code;
}

// Measured: 4096 x 25088 fp32 weights 86 to 99 us (463 MB, 4.7 to 5.4 TB/s: memory), 1000 x 1023 bf16 with a table
// 5.5 us (latency of one round of loads, a division and the table's search).
template <int TYPE, bool LUT>
__global__ __launch_bounds__(256) void quantize_groups_kernel(const QuantizeParams p) {
    const int lane = threadIdx.x & 63, l16 = lane & 15;
    const unsigned tile = blockIdx.x;
    const int64_t id = (int64_t)tile * 16 + (threadIdx.x >> 4);  // row of a tile
    __shared__ float s_mid[17];
    float top = 7.0f;
    if constexpr (LUT) {
        if (threadIdx.x < 17)
            s_mid[threadIdx.x] = threadIdx.x == 0 ? -__builtin_inff() : threadIdx.x == 16 ? __builtin_inff() :
                                 0.5f * (bf16_bits_to_f32(p.levels[threadIdx.x - 1]) + bf16_bits_to_f32(p.levels[threadIdx.x]));
        top = 0.0f;
#pragma unroll
        for (int j = 0; j < 16; ++j) top = __builtin_fmaxf(top, __builtin_fabsf(bf16_bits_to_f32(p.levels[j])));
        __syncthreads();
    }
    const int nt = (int)(tile / (unsigned)p.ktiles), kt = (int)(tile - (unsigned)nt * p.ktiles);
    const int row = nt * kTileRows + (int)(id & 15);
    const bool live = row < p.n;
    const int limit = live ? p.k : 0;
    const int c0 = kt * kTileCols + 8 * l16;
    float v[8];
    load_columns<TYPE>(p.W, (int64_t)row * p.ldw, c0, limit, v);
    unsigned a = max_bits(v);
    for (int off = 1; off < 1 << (p.log_group - 3); off <<= 1) {
        const unsigned o = __shfl_xor(a, off);
        a = o > a ? o : a;
    }
    float s;
    if (a >= 0x7f800000u) {
        s = __builtin_bit_cast(float, 0x7fc00000u);
    } else {
        s = bf16_bits_to_f32(Act<true>::one(__builtin_bit_cast(float, a) / top));
        if (s < 0x1p-126f) s = 0.0f;
    }
    if (live && c0 < p.k && (c0 & ((1 << p.log_group) - 1)) == 0)
        p.scales[(int64_t)row * p.groups + (c0 >> p.log_group)] = (uint16_t)(__builtin_bit_cast(unsigned, s) >> 16);
    const float inv = __builtin_amdgcn_rcpf(s);
    bool near = !(s >= 0x1p-100f && s <= 0x1p100f);
    unsigned codes[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float t = v[j] * inv;
        if constexpr (LUT) {
            codes[j] = nearest_level_code(t, s_mid);
            const float slack = __builtin_fabsf(t) * 0x1p-20f;
            near |= t - s_mid[codes[j]] < slack || s_mid[codes[j] + 1] - t < slack;
        } else {
            codes[j] = nearest_integer_code(t);
            near |= __builtin_fabsf(t - __builtin_rintf(t)) > 0.5f - 0x1p-17f;
        }
    }
    if (near) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float t = s > 0.0f ? v[j] / s : 0.0f;
            codes[j] = LUT ? nearest_level_code(t, s_mid) : nearest_integer_code(t);
        }
    }
    unsigned d = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (c0 + j < limit) d |= codes[j] << (4 * ((j & 1) * 4 + (j >> 1)));
    // columns 8 l .. 8 l + 7 are dword 4 (l % 4) + l / 4 of the row
    *(unsigned*)(p.codes + id * 64 + ((l16 & 3) * 4 + (l16 >> 2)) * 4) = d;
}

hipError_t launch_quantize_groups(const QuantizeParams& p, hipStream_t s) {
    const int64_t tiles = (int64_t)ceil_div(p.n, kTileRows) * p.ktiles;
    const dim3 grid((unsigned)tiles), block(256);
    const bool lut = p.levels != nullptr;
#define KQ_LAUNCH(T)                                                        \
    if (lut) quantize_groups_kernel<T, true><<<grid, block, 0, s>>>(p);     \
    else quantize_groups_kernel<T, false><<<grid, block, 0, s>>>(p);
    if (p.type == KQ_T_F32) { KQ_LAUNCH(KQ_T_F32) }
    else if (p.type == KQ_T_BF16) { KQ_LAUNCH(KQ_T_BF16) }
    else { KQ_LAUNCH(KQ_T_F16) }
#undef KQ_LAUNCH
    return hipGetLastError();
}

// ---- reconstruction: W_hat[n][k] = scale * level -----------------------------------------------------------
// A workgroup a tile, 16 lanes a row.  A lane writes four neighbouring columns at a time, 4 l + 64 h, so a
// row's lanes write contiguous memory; two lanes share a dword of codes.  4096 x 25088 fp32: 71 to 80 us (463 MB,
// 5.8 to 6.5 TB/s: memory).
template <int TYPE, bool LUT>
__global__ __launch_bounds__(256) void reconstruct_groups_kernel(const ReconstructGroupsParams p) {
    const int l16 = threadIdx.x & 15;
    const unsigned tile = blockIdx.x;
    __shared__ float s_level[16];
    if constexpr (LUT) {
        if (threadIdx.x < 16) s_level[threadIdx.x] = bf16_bits_to_f32(p.w.levels[threadIdx.x]);
        __syncthreads();
    }
    const int nt = (int)(tile / (unsigned)p.w.ktiles), kt = (int)(tile - (unsigned)nt * p.w.ktiles);
    const int r = threadIdx.x >> 4, row = nt * kTileRows + r;
    if (row >= p.w.n) return;
    const unsigned* codes = (const unsigned*)(p.w.codes + (int64_t)tile * kTileBytes + r * 64);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int cc = 64 * h + 4 * l16, c0 = kt * kTileCols + cc;  // dword 4 q + i of columns 32 i + 8 q
        if (c0 >= p.w.k) break;
        const unsigned d = codes[((cc >> 3) & 3) * 4 + (cc >> 5)] >> (8 * (l16 & 1));
        const float s = bf16_bits_to_f32(p.w.scales[(int64_t)row * p.w.groups + (c0 >> p.w.log_group)]);
        float v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {  // the second four columns are the second nibble of each pair
            const unsigned code = (d >> (16 * (j & 1) + 4 * (j >> 1))) & 15u;
            v[j] = s * (LUT ? s_level[code] : (float)((int)code - 8));
        }
        store_values<TYPE, 4>(p.W_hat, (int64_t)row * p.ldw + c0, v, p.w.k - c0);
    }
}

hipError_t launch_reconstruct_groups(const ReconstructGroupsParams& p, hipStream_t s) {
    const int64_t tiles = (int64_t)p.w.ntiles * p.w.ktiles;
    const dim3 grid((unsigned)tiles), block(256);
    const bool lut = p.w.levels != nullptr;
#define KQ_LAUNCH(T)                                                           \
    if (lut) reconstruct_groups_kernel<T, true><<<grid, block, 0, s>>>(p);     \
    else reconstruct_groups_kernel<T, false><<<grid, block, 0, s>>>(p);
    if (p.type == KQ_T_F32) { KQ_LAUNCH(KQ_T_F32) }
    else if (p.type == KQ_T_BF16) { KQ_LAUNCH(KQ_T_BF16) }
    else { KQ_LAUNCH(KQ_T_F16) }
#undef KQ_LAUNCH
    return hipGetLastError();
}

// ---- 8-bit checkpoints ---------------------------------------------------------------------------------------
// Groups of 32 columns share a power of two: with E = floor(log2 max |x|) the step is 2^e, e = E - 6 (at least
// -126, and at least -24 for fp16 inputs: the resolution of their subnormals), and q = rint(x 2^-e) clipped to
// [-127, 127].  So |q| is at most 127 however large x is, q 2^e has seven significant bits (bf16 holds it
// exactly, and fp16 does for fp16 inputs), and the error is at most half a step, one step where rint gives 128.
// A group with an infinity or a NaN gets exponent 255: all of it is NaN when it is read.
// Four lanes a group, 8 columns a lane: 16-byte loads for 16-bit types.  8192 x 25088 bf16: pack 107 to 113 us, restore
// 100 to 105 us (623 MB each, 5.5 to 6.2 TB/s: memory).

template <int TYPE>
__global__ __launch_bounds__(256) void checkpoint_pack_kernel(const CheckpointParams p) {
    const int per_row = p.kq >> 3;  // 8-column pieces
    const unsigned id = blockIdx.x * 256u + threadIdx.x;  // (at most 2^34 values: fewer than 2^32 threads)
    const int64_t row = id / (unsigned)per_row;
    const bool live = row < p.m;     // (groups are whole: the four lanes of one agree)
    const int c0 = live ? (int)(id - (unsigned)row * per_row) * 8 : 0;
    float v[8];
    load_columns<TYPE>(p.X, live ? row * p.ldx : 0, c0, live ? p.k : 0, v);
    unsigned a = max_bits(v);
#pragma unroll
    for (int off = 1; off <= 2; off <<= 1) {
        const unsigned o = __shfl_xor(a, off);
        a = o > a ? o : a;
    }
    if (!live) return;
    constexpr int least = TYPE == KQ_T_F16 ? 127 - 24 : 1;
    int e = (int)(a >> 23) - 6;      // biased exponent of the step
    e = e < least ? least : e;
    const bool bad = a >= 0x7f800000u;
    // x * 2^-e: exact (a power of two, and |x| 2^-e < 128)
    const float inv = __builtin_bit_cast(float, (unsigned)(254 - e) << 23);
    unsigned w[2] = {0, 0};
#pragma unroll
    for (int t = 0; t < 8; ++t) {
        float r = __builtin_rintf(v[t] * inv);
        r = __builtin_fminf(__builtin_fmaxf(r, -127.0f), 127.0f);
        const int qi = bad ? 0 : (int)r;
        w[t >> 2] |= ((unsigned)qi & 255u) << (8 * (t & 3));
    }
    *(u32x2*)(p.q + row * p.kq + c0) = u32x2{w[0], w[1]};
    if ((threadIdx.x & 3) == 0) p.exps[row * (p.kq >> 5) + (c0 >> 5)] = (uint8_t)(bad ? 255 : e);
}

template <int TYPE>
__global__ __launch_bounds__(256) void checkpoint_restore_kernel(const CheckpointParams p) {
    const int per_row = p.kq >> 3;
    const unsigned id = blockIdx.x * 256u + threadIdx.x;
    const int64_t row = id / (unsigned)per_row;
    if (row >= p.m) return;
    const int c0 = (int)(id - (unsigned)row * per_row) * 8;
    if (c0 >= p.k) return;
    const u32x2 w = *(const u32x2*)(p.q + row * p.kq + c0);
    const float step = checkpoint_step(p.exps[row * (p.kq >> 5) + (c0 >> 5)]);
    float v[8];
#pragma unroll
    for (int t = 0; t < 8; ++t) v[t] = (float)((int)(w[t >> 2] << (24 - 8 * (t & 3))) >> 24) * step;
    store_values<TYPE, 8>(p.X, row * p.ldx + c0, v, p.k - c0);
}

#define KQ_BY_TYPE(KERNEL)                                                    \
    if (p.type == KQ_T_F32) KERNEL<KQ_T_F32><<<grid, block, 0, s>>>(p);       \
    else if (p.type == KQ_T_BF16) KERNEL<KQ_T_BF16><<<grid, block, 0, s>>>(p); \
    else KERNEL<KQ_T_F16><<<grid, block, 0, s>>>(p);

hipError_t launch_checkpoint_pack(const CheckpointParams& p, hipStream_t s) {
    const dim3 grid((unsigned)ceil_div64(p.m * (p.kq >> 3), 256)), block(256);
    KQ_BY_TYPE(checkpoint_pack_kernel)
    return hipGetLastError();
}
hipError_t launch_checkpoint_restore(const CheckpointParams& p, hipStream_t s) {
    const dim3 grid((unsigned)ceil_div64(p.m * (p.kq >> 3), 256)), block(256);
    KQ_BY_TYPE(checkpoint_restore_kernel)
    return hipGetLastError();
}
#undef KQ_BY_TYPE

// ---- partial sums of a split contraction -------------------------------------------------------------------------
template <int TYPE>
__global__ __launch_bounds__(256) void join_kernel(const JoinParams p) {
    const unsigned per_row = (unsigned)((p.cols + 3) >> 2), id = blockIdx.x * 256u + threadIdx.x;  // (fewer than 2^32 threads)
    const int64_t r = id / per_row, c = (int64_t)(id - (unsigned)r * per_row) * 4, total = p.rows * p.cols;
    if (r >= p.rows) return;
    float v[4] = {0, 0, 0, 0};
    const float* part = p.part + r * p.cols + c;
    const int count = (int)min((int64_t)4, p.cols - c);
    // (four splits' loads in flight at a time; the sums stay in order)
    if (count == 4) {
        int s = 0;
        for (; s + 4 <= p.splits; s += 4, part += 4 * total) {
            float x[4][4];
#pragma unroll
            for (int u = 0; u < 4; ++u) __builtin_memcpy(x[u], part + u * total, 16);
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int t = 0; t < 4; ++t) v[t] += x[u][t];
        }
#pragma unroll 3
        for (; s < p.splits; ++s, part += total) {
            float x[4];
            __builtin_memcpy(x, part, 16);
#pragma unroll
            for (int t = 0; t < 4; ++t) v[t] += x[t];
        }
    } else {
        for (int s = 0; s < p.splits; ++s, part += total)
#pragma unroll
            for (int t = 0; t < 4; ++t)
                if (t < count) v[t] += part[t];
    }
    if (p.bias) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
            if (t < count) v[t] += p.bias[c + t];
    }
    store_values<TYPE, 4>(p.out, r * p.ldo + c, v, count);
}

hipError_t launch_join(const JoinParams& p, hipStream_t s) {
    const dim3 grid((unsigned)ceil_div64(p.rows * ((p.cols + 3) >> 2), 256)), block(256);
    if (p.type == KQ_T_F32) join_kernel<KQ_T_F32><<<grid, block, 0, s>>>(p);
    else if (p.type == KQ_T_BF16) join_kernel<KQ_T_BF16><<<grid, block, 0, s>>>(p);
    else join_kernel<KQ_T_F16><<<grid, block, 0, s>>>(p);
    return hipGetLastError();
}

}  // namespace kq
