// The 4-bit group quantizer, the weights it stands for, 8-bit activation checkpoints and the bias
// gradient: passes over memory.
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
template <int TYPE, int N>
__device__ __forceinline__ void store_values(void* base, int64_t at, const float (&v)[N], int count) {
    if constexpr (TYPE == KQ_T_F32) {
        float* o = (float*)base + at;
        if (count >= N) {
            __builtin_memcpy(o, v, 4 * N);
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
            __builtin_memcpy(o, h, 2 * N);
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
// One wave per 16 x 128 tile of codes; lane (row r, quarter q) = (lane / 4, lane % 4) takes the four dwords
// of its 16 bytes: columns 32 i + 8 q + 0..7 for i = 0..3, so the lanes of a row read 32 consecutive columns
// at a time and a group's columns lie in the row's four lanes.  Per group: a = max |w| (a non-finite value is
// larger than every other), s = bf16(a / top) with top = 7 or the largest |level| (zero below the normal
// range, NaN where a is not finite), and per weight t = w / s in fp32 and the nearest level to t, the lower
// one of two that are as near: for -8 .. 7 by rounding, for a table by counting the midpoints of
// neighbouring levels below t.
__device__ __forceinline__ unsigned nearest_integer_code(float t) {
    float r = __builtin_rintf(t);       // ties to even
    if (r - t == 0.5f) r -= 1.0f;       // a tie that went up
    r = __builtin_fminf(__builtin_fmaxf(r, -8.0f), 7.0f);
    return (unsigned)((int)r + 8);
}

template <int TYPE, bool LUT>
__global__ __launch_bounds__(256) void quantize_groups_kernel(const QuantizeParams p) {
    const int lane = threadIdx.x & 63;
    const int64_t tile = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int64_t tiles = (int64_t)ceil_div(p.n, kTileRows) * p.ktiles;
    if (tile >= tiles) return;
    const int nt = (int)(tile / p.ktiles), kt = (int)(tile % p.ktiles);
    const int row = nt * kTileRows + (lane >> 2), q = lane & 3;
    const bool live = row < p.n;
    const int limit = live ? p.k : 0;
    const int64_t at = (int64_t)row * p.ldw;

    float mid[15];
    float top = 7.0f;
    if constexpr (LUT) {
        float prev = bf16_bits_to_f32(p.levels[0]);
        top = __builtin_fabsf(prev);
#pragma unroll
        for (int j = 1; j < 16; ++j) {
            const float l = bf16_bits_to_f32(p.levels[j]);
            mid[j - 1] = 0.5f * (prev + l);
            top = __builtin_fmaxf(top, __builtin_fabsf(l));
            prev = l;
        }
    }

    float v[4][8];
    unsigned a[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        load_columns<TYPE>(p.W, at, kt * kTileCols + 32 * i + 8 * q, limit, v[i]);
        a[i] = max_bits(v[i]);
    }
    // largest magnitude of each 32-column block over the row's four lanes, then over the group's blocks
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int off = 1; off <= 2; off <<= 1) {
            const unsigned o = __shfl_xor(a[i], off);
            a[i] = o > a[i] ? o : a[i];
        }
    }
    if (p.log_group >= 6) {
        a[0] = a[1] = a[0] > a[1] ? a[0] : a[1];
        a[2] = a[3] = a[2] > a[3] ? a[2] : a[3];
    }
    if (p.log_group >= 7) a[0] = a[1] = a[2] = a[3] = a[0] > a[2] ? a[0] : a[2];

    unsigned dw[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float s;
        if (a[i] >= 0x7f800000u) {
            s = __builtin_bit_cast(float, 0x7fc00000u);
        } else {
            s = bf16_bits_to_f32(Act<true>::one(__builtin_bit_cast(float, a[i]) / top));
            if (s < 0x1p-126f) s = 0.0f;
        }
        const int c0 = kt * kTileCols + 32 * i;
        const int g = c0 >> p.log_group;
        if (q == 0 && live && c0 < p.k && (c0 & ((1 << p.log_group) - 1)) == 0)
            p.scales[(int64_t)row * p.groups + g] = (uint16_t)(__builtin_bit_cast(unsigned, s) >> 16);
        unsigned d = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float t = s > 0.0f ? v[i][j] / s : 0.0f;
            unsigned code;
            if constexpr (LUT) {
                code = 0;
#pragma unroll
                for (int b = 0; b < 15; ++b) code += t > mid[b] ? 1u : 0u;
            } else {
                code = nearest_integer_code(t);
            }
            if (c0 + 8 * q + j >= limit) code = 0;
            d |= code << (4 * ((j & 1) * 4 + (j >> 1)));
        }
        dw[i] = d;
    }
    u32x4 o = {dw[0], dw[1], dw[2], dw[3]};
    *(u32x4*)(p.codes + tile * kTileBytes + lane * 16) = o;
}

hipError_t launch_quantize_groups(const QuantizeParams& p, hipStream_t s) {
    const int64_t tiles = (int64_t)ceil_div(p.n, kTileRows) * p.ktiles;
    const dim3 grid((unsigned)ceil_div64(tiles, 4)), block(256);
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
// The quantizer's layout backwards: one wave per tile, 16 bytes of codes a lane.
template <int TYPE, bool LUT>
__global__ __launch_bounds__(256) void reconstruct_groups_kernel(const ReconstructGroupsParams p) {
    const int lane = threadIdx.x & 63;
    const int64_t tile = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int64_t tiles = (int64_t)p.w.ntiles * p.w.ktiles;
    __shared__ float s_level[16];
    if (threadIdx.x < 16)
        s_level[threadIdx.x] = LUT ? bf16_bits_to_f32(p.w.levels[threadIdx.x]) : (float)((int)threadIdx.x - 8);
    __syncthreads();
    if (tile >= tiles) return;
    const int nt = (int)(tile / p.w.ktiles), kt = (int)(tile % p.w.ktiles);
    const int row = nt * kTileRows + (lane >> 2), q = lane & 3;
    if (row >= p.w.n) return;
    const u32x4 dw = *(const u32x4*)(p.w.codes + tile * kTileBytes + lane * 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c0 = kt * kTileCols + 32 * i + 8 * q;
        if (c0 >= p.w.k) break;
        const float s = bf16_bits_to_f32(p.w.scales[(int64_t)row * p.w.groups + (c0 >> p.w.log_group)]);
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const unsigned code = (dw[i] >> (4 * ((j & 1) * 4 + (j >> 1)))) & 15u;
            v[j] = s * (LUT ? s_level[code] : (float)((int)code - 8));
        }
        store_values<TYPE, 8>(p.W_hat, (int64_t)row * p.ldw + c0, v, p.w.k - c0);
    }
}

hipError_t launch_reconstruct_groups(const ReconstructGroupsParams& p, hipStream_t s) {
    const int64_t tiles = (int64_t)p.w.ntiles * p.w.ktiles;
    const dim3 grid((unsigned)ceil_div64(tiles, 4)), block(256);
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
// Four lanes a group, 8 columns a lane: 16-byte loads for 16-bit types.

template <int TYPE>
__global__ __launch_bounds__(256) void checkpoint_pack_kernel(const CheckpointParams p) {
    const int per_row = p.kq >> 3;  // 8-column pieces
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t row = id / per_row;
    const bool live = row < p.m;     // (groups are whole: the four lanes of one agree)
    const int c0 = live ? (int)(id - row * per_row) * 8 : 0;
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

__device__ __forceinline__ float checkpoint_step(unsigned e) {
    return __builtin_bit_cast(float, e == 255u ? 0x7fc00000u : e << 23);
}

template <int TYPE>
__global__ __launch_bounds__(256) void checkpoint_restore_kernel(const CheckpointParams p) {
    const int per_row = p.kq >> 3;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t row = id / per_row;
    if (row >= p.m) return;
    const int c0 = (int)(id - row * per_row) * 8;
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

// A launch has fewer than 2^32 threads: rows in pieces of at most 2^30 threads.
template <bool PACK>
static hipError_t launch_checkpoint(CheckpointParams p, hipStream_t s) {
    const int per_row = p.kq >> 3;
    const int64_t piece = (int64_t(1) << 30) / per_row, rows = p.m;
    for (int64_t r = 0; r < rows; r += piece) {
        p.m = rows - r < piece ? rows - r : piece;
        const dim3 grid((unsigned)ceil_div64(p.m * per_row, 256)), block(256);
        if constexpr (PACK) {
            KQ_BY_TYPE(checkpoint_pack_kernel)
        } else {
            KQ_BY_TYPE(checkpoint_restore_kernel)
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        p.X = (char*)p.X + piece * p.ldx * (p.type == KQ_T_F32 ? 4 : 2);
        p.q += piece * p.kq;
        p.exps += piece * (p.kq / kCkGroup);
    }
    return hipSuccess;
}
#undef KQ_BY_TYPE

hipError_t launch_checkpoint_pack(const CheckpointParams& p, hipStream_t s) { return launch_checkpoint<true>(p, s); }
hipError_t launch_checkpoint_restore(const CheckpointParams& p, hipStream_t s) { return launch_checkpoint<false>(p, s); }

// ---- bias gradient: dbias[n] = sum_m dY[m][n] ------------------------------------------------------------------
// A workgroup adds 32 columns: 4 lanes of 8 columns, 64 rows at a time, then the 64 partial sums in order.
template <bool BF>
__global__ __launch_bounds__(256) void bias_grad_kernel(const BiasGradParams p) {
    __shared__ float s_part[64][33];
    const int cl = threadIdx.x & 3, rl = threadIdx.x >> 2;
    const int c0 = blockIdx.x * 32 + cl * 8;
    float acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int64_t r = rl; r < p.m; r += 64) {
        float v[8];
        load_columns<BF ? KQ_T_BF16 : KQ_T_F16>(p.dY, r * p.ldy, c0, p.n, v);
#pragma unroll
        for (int t = 0; t < 8; ++t) acc[t] += v[t];
    }
#pragma unroll
    for (int t = 0; t < 8; ++t) s_part[rl][cl * 8 + t] = acc[t];
    __syncthreads();
    if (threadIdx.x < 32 && (int)(blockIdx.x * 32 + threadIdx.x) < p.n) {
        float v = 0.0f;
        for (int r = 0; r < 64; ++r) v += s_part[r][threadIdx.x];
        p.dbias[blockIdx.x * 32 + threadIdx.x] = v;
    }
}

hipError_t launch_bias_grad(const BiasGradParams& p, hipStream_t s) {
    const dim3 grid((unsigned)ceil_div(p.n, 32)), block(256);
    if (p.type == KQ_T_BF16) bias_grad_kernel<true><<<grid, block, 0, s>>>(p);
    else bias_grad_kernel<false><<<grid, block, 0, s>>>(p);
    return hipGetLastError();
}

}  // namespace kq
