// Element access by type (KQ_T_F32, KQ_T_BF16, KQ_T_F16) for the passes over memory.
#pragma once

#include "kq_group.h"

namespace kq {

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
// (fp32 weights of 4096 x 25088 rebuilt: 75 us, 131 us with ordinary stores).  Four values a thread only where they lie on
// their own size: pieces of lines are slow that way (rebuilt from 4 bits, ordinary and streamed: 4096 x 25087 fp32 133 and 181
// us, 4096 x 25090 bf16 56 and 128; rows that begin on their own size inside a line are as slow, 4096 x 25092 bf16 123).
// Eight 16-bit values on any dword (checkpoints of 4096 x 25090 bf16 restored: 46.7 us, 52.9 with ordinary stores; 4096 x 25087
// 47.3 and 54.6).
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
            for (int t = 0; t < N; t += 4) {
                if (((uintptr_t)o & 15) == 0) stream_store(o + t, h + t, 4);
                else __builtin_memcpy(o + t, h + t, 16);
            }
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
            if (((uintptr_t)o & (N == 8 ? 3 : 2 * N - 1)) == 0) stream_store(o, h, N / 2);
            else __builtin_memcpy(o, h, 2 * N);
        } else {
#pragma unroll
            for (int t = 0; t < N; ++t)
                if (t < count) o[t] = Act<TYPE == KQ_T_BF16>::one(v[t]);
        }
    }
}

// 8 columns at c0 of a row, zeros past the row's `limit`.  (A row's last few are loaded at clamped places, all at once: with a
// branch for each the next load waited for the one before.)
template <int TYPE>
__device__ __forceinline__ void load_columns(const void* base, int64_t row_at, int c0, int limit, float (&v)[8]) {
    if (c0 + 8 <= limit) {
        load_values<TYPE, 8>(base, row_at + c0, v);
    } else if (c0 < limit) {
#pragma unroll
        for (int t = 0; t < 8; ++t) v[t] = load_value_as<TYPE>(base, row_at + min(c0 + t, limit - 1));
#pragma unroll
        for (int t = 0; t < 8; ++t) v[t] = c0 + t < limit ? v[t] : 0.0f;
    } else {
#pragma unroll
        for (int t = 0; t < 8; ++t) v[t] = 0.0f;
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

}  // namespace kq
