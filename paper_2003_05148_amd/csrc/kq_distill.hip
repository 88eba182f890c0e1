// Distillation from a teacher's top logits: the loss of every row and the gradient of its logits.
//
//   p = softmax of the row's present teacher logits / T;  q = softmax of z / T;  s = softmax of z
//   loss = (1 - alpha) T^2 sum_j p_j (log p_j - log q_idx[j]) + alpha (-log s_label)
//   dz_c = d [ (1 - alpha) T (q_c - p_c) + alpha (s_c - [c = label]) ]
// With M the row's largest logit everything is taken from differences to it: q_c = exp((z_c - M) / T) / S_T, and p likewise
// with S_t.  Where p and q are close at a high temperature, the loss and the gradient at the teacher's classes are differences
// too small for that: Teacher::close_divergence.
// The gradient is dense in q and s and differs from that at the teacher's classes and the label: the dense part is
// written first, and once those stores have ended the few others are written over it.
//
// Memory bounds all of it (8 operations a logit), so a row is read once: it stays in registers, 16 bytes a chunk, between
// the largest logit, the sums and the gradient (distill_row_kernel: a wave a row while 8 chunks a lane hold it,
// then 256 or 1024 threads).  Rows of more chunks than that are read again.  Where there are few rows of many
// classes, a row is cut into segments: one kernel takes their largest logits and sums, the next joins them.
// 4096 x 50001 bf16: loss and gradient 161 to 170 us (822 MB, 4.8 to 5.1 TB/s, a copy's rate 5.2), the loss alone 85,
// the gradient alone 158.  With two temperatures (T other than 1 and labels) the exponentials bound it as well: 212, 122
// and 163 us.  Small calls are bound by a launch and the chain index, logit, sum (64 x 1000: 6.4 us; 64 x 100 fp32 of close rows
// at T = 20: 13).
#include "kq_values.h"

namespace kq {

struct DistillParams {
    const void* Z;
    int type;
    int64_t ldz, m;
    int v;
    const void* top_values;
    int top_type;
    const void* top_idx;
    int idx_bytes;
    int top;
    const void* labels;      // NULL where alpha is 0
    int label_bytes;
    float T, alpha;
    const float* dloss;
    float scale;
    float* loss;             // NULL where the loss is not asked for
    float* stats;            // out, or NULL
    void* dZ;                // NULL where the gradient is not asked for
    int64_t lddz;
    // rows in segments: what they gave, [m][segments][3] (of kq_distill_grad the stats, one segment), and the
    // logits at the teacher's classes and the label, [m][top + 1]
    float* part;
    float* at_top;
    int segments, chunks_per_segment;
    int workgroups;          // a row's, in a launch by segments
    float eT_hi, eT_lo, e1_hi, e1_lo;  // Exponential of T and of 1
};

__device__ __forceinline__ float load_any(const void* base, int type, int64_t at) {
    if (type == KQ_T_F32) return ((const float*)base)[at];
    const unsigned h = ((const uint16_t*)base)[at];
    return type == KQ_T_BF16 ? Act<true>::lo(h) : Act<false>::lo(h);
}
__device__ __forceinline__ int64_t load_index(const void* base, int bytes, int64_t at) {
    return bytes == 8 ? ((const int64_t*)base)[at] : ((const int32_t*)base)[at];
}
template <int TYPE>
__device__ __forceinline__ void store_one(char* row, int c, float v) {
    if constexpr (TYPE == KQ_T_F32) *(float*)(row + (unsigned)c * 4u) = v;
    else *(uint16_t*)(row + (unsigned)c * 2u) = Act<TYPE == KQ_T_BF16>::one(v);
}

// ---- rows as chunks of 16 bytes ---------------------------------------------------------------------------------
// A row is `head` values up to a 16-byte boundary, `chunks` chunks on such boundaries, and `tail` values.  (Rows of an odd
// number of classes begin anywhere: 4096 x 50001 bf16 took 211 us in unaligned chunks where 4096 x 50000 took 186.)  The at
// most 14 single values go to one thread each.
template <int TYPE>
struct Row {
    static constexpr int N = TYPE == KQ_T_F32 ? 4 : 8, kBytes = 16 / N;
    static constexpr unsigned kMasked = TYPE == KQ_T_F32 ? 0xff800000u : TYPE == KQ_T_BF16 ? 0xff80ff80u : 0xfc00fc00u;  // -infinity
    const char* z;   // the row
    int head, chunks, tail;
    __device__ __forceinline__ void init(const DistillParams& p, int64_t row) {
        z = (const char*)p.Z + row * p.ldz * kBytes;
        head = min((int)((16u - ((unsigned)(uintptr_t)z & 15u)) & 15u) / kBytes, p.v);
        chunks = (p.v - head) / N;
        tail = p.v - head - chunks * N;
    }
    // the c-th chunk, -infinity past the last
    __device__ __forceinline__ u32x4 load(int c) const {
        u32x4 w = {kMasked, kMasked, kMasked, kMasked};
        if (c < chunks) w = *(const u32x4*)(z + head * kBytes + (unsigned)c * 16u);
        return w;
    }
    // the class of the s-th single value, -1 past the last
    __device__ __forceinline__ int single(int s) const { return s < head ? s : s < head + tail ? chunks * N + s : -1; }
    __device__ __forceinline__ float at(int c) const {
        if constexpr (TYPE == KQ_T_F32) {
            return *(const float*)(z + (unsigned)c * 4u);
        } else {
            return Act<TYPE == KQ_T_BF16>::lo(*(const uint16_t*)(z + (unsigned)c * 2u));
        }
    }
    static __device__ __forceinline__ void unpack(u32x4 w, float (&x)[N]) {
        if constexpr (TYPE == KQ_T_F32) {
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const unsigned bits = w[t];  // (a bit cast of a vector's element takes the first one)
                x[t] = __builtin_bit_cast(float, bits);
            }
        } else {
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                x[2 * t] = Act<TYPE == KQ_T_BF16>::lo(w[t]);
                x[2 * t + 1] = Act<TYPE == KQ_T_BF16>::hi(w[t]);
            }
        }
    }
    static __device__ __forceinline__ u32x4 pack(const float (&x)[N]) {
        u32x4 w;
        if constexpr (TYPE == KQ_T_F32) {
#pragma unroll
            for (int t = 0; t < 4; ++t) w[t] = __builtin_bit_cast(unsigned, x[t]);
        } else {
#pragma unroll
            for (int t = 0; t < 4; ++t) w[t] = Act<TYPE == KQ_T_BF16>::pack(x[2 * t], x[2 * t + 1]);
        }
        return w;
    }
};

// Keeps a row packed between two passes over it: left alone, the compiler keeps the unpacked values of the first, twice or
// four times the registers.
template <int CH>
__device__ __forceinline__ void stay_packed(u32x4 (&w)[CH]) {
#pragma unroll
    for (int t = 0; t < CH; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            unsigned x = w[t][i];
            asm volatile("" : "+v"(x));
            w[t][i] = x;
        }
}

// One chunk after the other: a chunk has enough to overlap, and more of them at once take registers.
__device__ __forceinline__ void in_turn(float& v) {
    asm volatile("" : "+v"(v));
    __builtin_amdgcn_sched_barrier(0);
}

// exp(d / T) for d <= 0: log2(e) / T in two parts, so that its rounding does not grow with d.  The smaller part is above
// zero: minus infinity stays that.
struct Exponential {
    float hi, lo;
    static Exponential of(float T) {
        const double c = 1.4426950408889634 / (double)T;
        Exponential e;
        e.hi = (float)c;
        if ((double)e.hi >= c) e.hi = __builtin_bit_cast(float, __builtin_bit_cast(unsigned, e.hi) - 1u);
        e.lo = (float)(c - (double)e.hi);
        return e;
    }
    __device__ __forceinline__ float operator()(float d) const { return __builtin_amdgcn_exp2f(__builtin_fmaf(d, hi, d * lo)); }
    __device__ __forceinline__ float coarse(float d) const { return __builtin_amdgcn_exp2f(d * hi); }
};

// over N neighbouring lanes
template <int N = 64>
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int off = 1; off < N; off <<= 1) v = __builtin_fmaxf(v, __shfl_xor(v, off));
    return v;
}
template <int N = 64>
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int off = 1; off < N; off <<= 1) v += __shfl_xor(v, off);
    return v;
}

// The largest of some logits and sums of exponentials of the differences to it.
struct Sums {
    float M, sT, s1;
};
// `two`: s1 is wanted apart from sT
__device__ __forceinline__ void rebase(Sums& s, float M, bool two, const Exponential& eT, const Exponential& e1) {
    // (nothing but masked classes so far: no difference to take)
    const float d = s.M == M ? 0.0f : s.M - M;
    s.sT *= eT(d);
    if (two) s.s1 *= e1(d);
    s.M = M;
}
// over WAVES waves that share a row, the same value in every thread
template <int WAVES>
__device__ __forceinline__ Sums join_sums(Sums s, float (*s_red)[WAVES], int wave, bool two, const Exponential& eT, const Exponential& e1) {
    rebase(s, wave_max(s.M), two, eT, e1);
    s.sT = wave_sum(s.sT);
    if (two) s.s1 = wave_sum(s.s1);
    if constexpr (WAVES > 1) {
        if ((threadIdx.x & 63) == 0) {
            s_red[0][wave] = s.M;
            s_red[1][wave] = s.sT;
            s_red[2][wave] = s.s1;
        }
        __syncthreads();
        // (a wave's at each lane again: held in registers, 16 waves' would be 48)
        const int w = threadIdx.x & (WAVES - 1);
        s = {s_red[0][w], s_red[1][w], s_red[2][w]};
        rebase(s, wave_max<WAVES>(s.M), two, eT, e1);
        s.sT = wave_sum<WAVES>(s.sT);
        if (two) s.s1 = wave_sum<WAVES>(s.s1);
    }
    return s;
}

// ---- the teacher's entries of a row and its label, by one wave ------------------------------------------------------
struct __attribute__((aligned(16))) TopEntries {
    int idx[KQ_DISTILL_MAX_TOP];   // -1: absent (and behind the last, up to a multiple of 8)
    float t[KQ_DISTILL_MAX_TOP];   // teacher's logit less its largest; of a close row q - p from its divergence on
    float p[KQ_DISTILL_MAX_TOP];   // 0 for absent ones
    float z[KQ_DISTILL_MAX_TOP];   // the network's own logit there
    float row[8];                  // the row's sums and Teacher, where registers hold the row in between
};
__device__ __forceinline__ void wave_fence() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

// Above this temperature the divergence of p and q that are close is taken in a way of its own.  Up to it T^2 times the
// rounding of a plain sum is 10^-5 at most, and that way costs 0.4 to 1 us (64 x 1000 bf16 6.3 and 7.3 us, the loss alone of 4096
// x 32000 47.6 and 51.7).
constexpr float kCloseFrom = 4.0f;

struct Teacher {
    float St;         // sum of exp(t / T); 0 without a present entry
    int label;        // -1: absent
    float zy;         // the network's logit there
    __device__ __forceinline__ void keep(float* at) const {
        at[0] = St;
        at[1] = __builtin_bit_cast(float, label);
        at[2] = zy;
    }
    __device__ __forceinline__ void take(const float* at) {
        St = at[0];
        label = __builtin_bit_cast(int, at[1]);
        zy = at[2];
    }
    // reads z at the entries and the label
    template <int TYPE>
    __device__ __forceinline__ void init(const DistillParams& p, const Row<TYPE>& r, TopEntries& s, int64_t row, int lane, const Exponential& eT) {
        label = -1;
        zy = 0.0f;
        St = 0.0f;
        int64_t y = -1;
        if (p.alpha > 0.0f) y = load_index(p.labels, p.label_bytes, row);
        float tM = -__builtin_inff();
        if (p.alpha < 1.0f) {
            for (int j = lane; j < ((p.top + 7) & ~7); j += 64) {
                int64_t at = -1;
                float x = 0.0f;
                if (j < p.top) {
                    at = load_index(p.top_idx, p.idx_bytes, row * p.top + j);
                    x = load_any(p.top_values, p.top_type, row * p.top + j);
                }
                const bool here = at >= 0 && at < p.v && x != -__builtin_inff();
                x = here ? x : -__builtin_inff();
                s.idx[j] = here ? (int)at : -1;
                s.t[j] = x;
                s.z[j] = here ? r.at((int)at) : 0.0f;
                tM = __builtin_fmaxf(tM, x);
            }
        }
        if (y >= 0 && y < p.v) {
            label = (int)y;
            zy = r.at(label);
        }
        if (p.alpha >= 1.0f) return;
        tM = wave_max(tM);
        for (int j = lane; j < p.top; j += 64) {
            const float d = s.t[j] - tM, e = s.idx[j] >= 0 ? eT(d) : 0.0f;
            s.t[j] = d;
            s.p[j] = e;
            St += e;
        }
        St = wave_sum(St);
        const float inv = 1.0f / St;
        for (int j = lane; j < p.top; j += 64) s.p[j] = s.idx[j] >= 0 ? s.p[j] * inv : 0.0f;
        wave_fence();
    }
    // The divergence sum p (log p - log q) of p and q that are close (large temperatures, a network near its teacher), where
    // the sum of logarithms is a small difference of large terms and T^2 would multiply its rounding (100 classes, all of them
    // entries: 0.4442 for 0.4437 at T = 100, 0.84 for 0.45 at 1024; this way off by 3e-7 of itself).  With x_j = (t_j - z_j) / T less its mean under p,
    //   S_T / S_t e^mean = 1 + sum p_j (e^-x_j - 1 + x_j) + rest e^mean / S_t,
    // and the divergence is the logarithm of that: no term is below zero but for classes that stand twice, so nothing
    // cancels.  rest, of the classes that are no entries, is itself a difference of sums: below 2^-20 of S_T it may be
    // nothing but their rounding and counts as zero.  The gradient's q - p = p (e^-x S_t e^-mean / S_T - 1) is taken of the
    // same (100 classes: T q - T p is off by 8e-5 of its norm at T = 1024 and 8 % at 2^20, this by 3e-7).
    __device__ __forceinline__ float close_divergence(const DistillParams& p, TopEntries& s, int lane, const Sums& r, const Exponential& eT, float invT) const {
        float mean = 0.0f;
        for (int j = lane; j < p.top; j += 64)
            if (s.idx[j] >= 0 && s.p[j] != 0.0f) mean += s.p[j] * ((s.t[j] - (s.z[j] - r.M)) * invT);
        mean = wave_sum(mean);
        const float shift = Exponential{p.e1_hi, p.e1_lo}(mean) / St;
        float more = 0.0f, inside = 0.0f;
        for (int j = lane; j < p.top; j += 64) {
            const float pj = s.p[j];
            if (s.idx[j] < 0 || pj == 0.0f) continue;
            const float d = s.z[j] - r.M, e = eT(d), x = (s.t[j] - d) * invT - mean;
            inside += e;
            more += __builtin_fabsf(x) < 1.0f ? pj * above_tangent(x) : e * shift + pj * (x - 1.0f);
        }
        more = wave_sum(more);
        const float rest = r.sT - wave_sum(inside);
        if (__builtin_fabsf(rest) > 0x1p-20f * r.sT) more += rest * shift;
        for (int j = lane; j < p.top; j += 64) {
            const float pj = s.p[j], d = s.z[j] - r.M, x = (s.t[j] - d) * invT - mean;
            s.t[j] = pj != 0.0f && __builtin_fabsf(x) < 1.0f ? pj * (above_tangent(x) - x - more) / (1.0f + more) : eT(d) / r.sT - pj;
        }
        wave_fence();
        // log(1 + y) for |y| < 0.3 as 2 artanh(y / (2 + y))
        const float y = more / (2.0f + more), y2 = y * y;
        return 2.0f * y * (1.0f + y2 * (1.0f / 3 + y2 * (1.0f / 5 + y2 * (1.0f / 7 + y2 * (1.0f / 9)))));
    }
    // e^-x - 1 + x for |x| < 1, by its power series (the first term left out is below 2^-27 of it)
    static __device__ __forceinline__ float above_tangent(float x) {
        constexpr float c[] = {1.0f / 2, -1.0f / 6, 1.0f / 24, -1.0f / 120, 1.0f / 720, -1.0f / 5040, 1.0f / 40320, -1.0f / 362880, 1.0f / 3628800, -1.0f / 39916800};
        float y = c[9];
#pragma unroll
        for (int i = 8; i >= 0; --i) y = __builtin_fmaf(y, x, c[i]);
        return y * x * x;
    }
    // sum p (log p - log q), in every lane; 0 without a present entry.  close: the entries' t is q - p now.
    __device__ __forceinline__ float divergence(const DistillParams& p, TopEntries& s, int lane, const Sums& r, const Exponential& eT, bool& close) const {
        close = false;
        float sum = 0.0f;
        if (St != 0.0f) {  // (also where it is NaN)
            const float lse = logf(r.sT) - logf(St), invT = 1.0f / p.T;
            for (int j = lane; j < p.top; j += 64) {
                const float pj = s.p[j];
                if (s.idx[j] >= 0 && pj != 0.0f) sum += pj * ((s.t[j] - (s.z[j] - r.M)) * invT + lse);
            }
            sum = wave_sum(sum);
            close = p.T > kCloseFrom && __builtin_fabsf(sum) < 0.25f;
            if (close) sum = close_divergence(p, s, lane, r, eT, invT);
        }
        return sum;
    }
    // the row's loss, in every lane
    __device__ __forceinline__ float loss(const DistillParams& p, TopEntries& s, int lane, const Sums& r, const Exponential& eT, bool& close) const {
        const float sum = divergence(p, s, lane, r, eT, close) * ((1.0f - p.alpha) * p.T * p.T);
        return label >= 0 ? sum + p.alpha * (logf(r.s1) - (zy - r.M)) : sum;
    }
};

// Factors of a row's gradient: dz = fT exp((z - M) / T) + f1 exp(z - M), less wT p and w1 at the teacher's classes and the
// label.
struct Factors {
    float fT, f1, wT, w1;
    __device__ __forceinline__ void init(const DistillParams& p, int64_t row, float St, int label, const Sums& s) {
        const float d = p.dloss ? p.dloss[row] : p.scale;
        wT = St != 0.0f ? d * (1.0f - p.alpha) * p.T : 0.0f;
        w1 = label >= 0 ? d * p.alpha : 0.0f;
        // (0 times St: a NaN of the teacher's is one of the whole row's)
        fT = St != 0.0f ? wT / s.sT + 0.0f * St : 0.0f;
        f1 = label >= 0 ? w1 / s.s1 : 0.0f;
    }
};
// The dense part: of one logit, and of a chunk.  One exponential where T is 1 or a row has one term only.
struct Dense {
    Factors f;
    float M;
    bool one, none;   // none: a row without either term, whatever its logits are
    Exponential eT, e1;
    __device__ __forceinline__ void init(const DistillParams& p, int64_t row, float St, int label, const Sums& s, const Exponential& aT, const Exponential& a1) {
        f.init(p, row, St, label, s);
        M = s.M;
        one = p.T == 1.0f || f.f1 == 0.0f;
        none = f.fT == 0.0f && f.f1 == 0.0f;
        eT = aT;
        e1 = a1;
    }
    __device__ __forceinline__ float of(float z) const {
        const float d = z - M;
        if (none) return 0.0f;
        return one ? (f.fT + f.f1) * eT(d) : f.fT * eT(d) + f.f1 * e1(d);
    }
    template <int TYPE, bool ONE>
    __device__ __forceinline__ u32x4 chunk(u32x4 w) const {
        constexpr bool kFine = TYPE == KQ_T_F32;  // (16 bits hide the rounding of log2(e) / T)
        float x[Row<TYPE>::N];
        Row<TYPE>::unpack(w, x);
        if constexpr (ONE) {
            const float k = f.fT + f.f1;
#pragma unroll
            for (int t = 0; t < Row<TYPE>::N; ++t) x[t] = k * (kFine ? eT(x[t] - M) : eT.coarse(x[t] - M));
        } else {
#pragma unroll
            for (int t = 0; t < Row<TYPE>::N; ++t) {
                const float d = x[t] - M;
                x[t] = kFine ? f.fT * eT(d) + f.f1 * e1(d) : f.fT * eT.coarse(d) + f.f1 * e1.coarse(d);
            }
        }
        return Row<TYPE>::pack(x);
    }
    // Chunks c, c + step, ... below `end` to the row that begins at `first`.  STREAM: past the caches' normal ways, for rows of
    // more classes than a wave holds (1024 x 131072 fp32, loss and gradient: 267 us, 310 with ordinary stores; 4096 x 50001
    // bf16 170 and 174; but 8192 x 1000, where the exceptions come back to the same lines, 18.9 and 17.1).
    template <bool STREAM>
    static __device__ __forceinline__ void put(char* at, u32x4 g) {
        using u32x4_any = __attribute__((ext_vector_type(4), aligned(2))) unsigned;  // (dZ's rows may begin elsewhere than Z's)
        if constexpr (STREAM) __builtin_nontemporal_store((u32x4_any)g, (u32x4_any*)at);
        else *(u32x4_any*)at = (u32x4_any)g;
    }
    template <int TYPE, bool ONE, bool STREAM, int CH>
    __device__ __forceinline__ void store(char* first, int c, int step, int end, u32x4 (&w)[CH]) const {
        stay_packed(w);
#pragma unroll
        for (int t = 0; t < CH; ++t) {
            if (c + t * step < end) put<STREAM>(first + (unsigned)(c + t * step) * 16u, chunk<TYPE, ONE>(w[t]));
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    template <int TYPE, bool STREAM, int CH>
    __device__ __forceinline__ void chunks(char* first, int c, int step, int end, u32x4 (&w)[CH]) const {
        if (none) {
#pragma unroll
            for (int t = 0; t < CH; ++t)
                if (c + t * step < end) put<STREAM>(first + (unsigned)(c + t * step) * 16u, u32x4{0, 0, 0, 0});
        } else if (one) {
            store<TYPE, true, STREAM>(first, c, step, end, w);
        } else {
            store<TYPE, false, STREAM>(first, c, step, end, w);
        }
    }
};
// Its exceptions in classes [c_begin, c_end), by one wave; the dense stores there have ended.  An index that stands more
// than once is written by its first place, with all of its p, in order.
template <int TYPE>
__device__ __forceinline__ void write_exceptions(const DistillParams& p, const TopEntries& s, char* out, int lane, int label, float zy,
                                                 const Dense& d, bool close, int c_begin, int c_end) {
    bool hit = false;
    if (p.alpha < 1.0f) {
        for (int j0 = 0; j0 < p.top; j0 += 64) {
            const int j = j0 + lane, own = j < p.top ? s.idx[j] : -1;
            const bool here = own >= c_begin && own < c_end;
            hit |= here && own == label;
            if (__builtin_amdgcn_ballot_w64(here) == 0) continue;
            float sum = 0.0f;
            bool first = here;
            for (int o = 0; o < p.top; o += 8) {  // (eight at a time: their reads of LDS overlap)
                int oi[8];
                float op[8];
                __builtin_memcpy(oi, s.idx + o, 32);
                __builtin_memcpy(op, s.p + o, 32);
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const bool same = oi[u] == own;
                    sum += same ? op[u] : 0.0f;
                    first = first && !(same && o + u < j);
                }
            }
            if (!first) continue;
            const float g = close ? d.f.wT * (s.t[j] - (sum - s.p[j])) + d.f.f1 * d.e1(s.z[j] - d.M) : d.of(s.z[j]) - d.f.wT * sum;
            store_one<TYPE>(out, own, g - (own == label ? d.f.w1 : 0.0f));
        }
    }
    if (__builtin_amdgcn_ballot_w64(hit) == 0 && lane == 0 && label >= c_begin && label < c_end)
        store_one<TYPE>(out, label, d.of(zy) - d.f.w1);
}

// The sums of a chunk's logits, added to s; its largest is taken first.
template <int TYPE>
__device__ __forceinline__ float chunk_max(u32x4 w, float a) {
    float x[Row<TYPE>::N];
    Row<TYPE>::unpack(w, x);
#pragma unroll
    for (int t = 0; t < Row<TYPE>::N; ++t) a = __builtin_fmaxf(a, x[t]);
    return a;
}
template <int TYPE>
__device__ __forceinline__ float chunk_sum(u32x4 w, float base, const Exponential& e) {
    float x[Row<TYPE>::N], y[2] = {0.0f, 0.0f};
    Row<TYPE>::unpack(w, x);
#pragma unroll
    for (int t = 0; t < Row<TYPE>::N; ++t) y[t & 1] += e(x[t] - base);
    return y[0] + y[1];
}
// (Every pass over the chunks is a loop of its own that begins with packed ones: with a branch for each chunk the compiler
// carried all differences from one pass to the next.)
template <int TYPE, int CH>
__device__ __forceinline__ void add_chunks(Sums& s, u32x4 (&w)[CH], float base, bool two, const Exponential& eT, const Exponential& e1) {
    stay_packed(w);
#pragma unroll
    for (int t = 0; t < CH; ++t) {
        s.sT += chunk_sum<TYPE>(w[t], base, eT);
        in_turn(s.sT);
    }
    if (two) {
        stay_packed(w);
#pragma unroll
        for (int t = 0; t < CH; ++t) {
            s.s1 += chunk_sum<TYPE>(w[t], base, e1);
            in_turn(s.s1);
        }
    }
}
// a value that is among the sums' largest already
__device__ __forceinline__ void add_single(Sums& s, float x, bool two, const Exponential& eT, const Exponential& e1) {
    const float base = s.M == -__builtin_inff() ? 0.0f : s.M;
    s.sT += eT(x - base);
    if (two) s.s1 += e1(x - base);
}

// ---- a row in one workgroup or wave ------------------------------------------------------------------------------
// CH chunks a thread in registers, WAVES waves a row (1: four rows a workgroup).  CH = 0: the row is read again.
// LOSS, GRAD: what is asked for; the gradient alone takes a row's stats, and a wave (longer rows: distill_segment_kernel).
template <int TYPE, int CH, int WAVES, bool LOSS, bool GRAD>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES, WAVES == 16 ? (CH > 8 ? 4 : 8) : 1) void distill_row_kernel(const DistillParams p) {
    static_assert(LOSS || WAVES == 1, "the gradient alone");
    constexpr int NT = 64 * WAVES;
    constexpr int kHeld = CH ? CH : 1;
    // Of many chunks the loss comes after the dense stores, when no registers hold them and the stores are on their way (before
    // them it took up to 4 registers more than 8 waves a SIMD have); of few before (64 x 1000 bf16 0.1 us less).
    constexpr bool kLate = LOSS && GRAD && CH >= 8;
    __shared__ float s_red[3][WAVES];
    __shared__ float s_row[2];
    __shared__ TopEntries s_top[WAVES == 1 ? 4 : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tid = WAVES == 1 ? lane : threadIdx.x;
    const int64_t row = WAVES == 1 ? (int64_t)blockIdx.x * 4 + wave : blockIdx.x;
    if (WAVES == 1 && row >= p.m) return;
    const bool leader = WAVES == 1 || wave == 0;
    TopEntries& entries = s_top[WAVES == 1 ? wave : 0];
    const bool ce = p.alpha > 0.0f, two = ce && p.T != 1.0f;
    const Exponential eT = {p.eT_hi, p.eT_lo}, e1 = {p.e1_hi, p.e1_lo};
    Row<TYPE> r;
    r.init(p, row);

    u32x4 w[kHeld];
    if constexpr (CH > 0) {
#pragma unroll
        for (int t = 0; t < CH; ++t) w[t] = r.load(t * NT + tid);
    }
    const int single = r.single(tid);
    const float x1 = single >= 0 ? r.at(single) : -__builtin_inff();
    Teacher te;
    bool close = false;
    if (leader) te.init<TYPE>(p, r, entries, row, lane, eT);
    if (WAVES > 1 && wave == 0) __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): what was read of Z is here before it may be written
    if (WAVES > 1 && threadIdx.x == 0) {
        s_row[0] = te.St;
        s_row[1] = __builtin_bit_cast(float, te.label);
    }
    Sums s = {x1, 0.0f, 0.0f};
    if constexpr (!LOSS) {
        s = {p.part[3 * row], p.part[3 * row + 1], p.part[3 * row + 2]};
    } else {
        if constexpr (CH > 0) {
#pragma unroll
            for (int t = 0; t < CH; ++t) {
                s.M = chunk_max<TYPE>(w[t], s.M);
                in_turn(s.M);
            }
            const float base = s.M == -__builtin_inff() ? 0.0f : s.M;  // (a thread whose classes are all masked out)
            add_chunks<TYPE>(s, w, base, two, eT, e1);
        } else {
            for (int c = tid; c < r.chunks; c += 4 * NT) {  // four chunks in flight
                u32x4 x[4];
                float top = s.M;
#pragma unroll
                for (int u = 0; u < 4; ++u) x[u] = r.load(c + u * NT);
#pragma unroll
                for (int u = 0; u < 4; ++u) top = chunk_max<TYPE>(x[u], top);
                const float base = top == -__builtin_inff() ? 0.0f : top;
                rebase(s, top, two, eT, e1);
                add_chunks<TYPE>(s, x, base, two, eT, e1);
            }
        }
        add_single(s, x1, two, eT, e1);
        s = join_sums<WAVES>(s, s_red, wave, two, eT, e1);
        if (!two) s.s1 = ce ? s.sT : 0.0f;
        if (!kLate && leader) {
            const float loss = te.loss(p, entries, lane, s, eT, close);
            if (lane == 0) {
                p.loss[row] = loss;
                if (p.stats) {
                    p.stats[3 * row] = s.M;
                    p.stats[3 * row + 1] = s.sT;
                    p.stats[3 * row + 2] = s.s1;
                }
            }
        }
    }
    if constexpr (kLate) {
        if (leader && lane == 0) {
            entries.row[0] = s.M;
            entries.row[1] = s.sT;
            entries.row[2] = s.s1;
            te.keep(entries.row + 3);
        }
    }
    if constexpr (GRAD) {
        const int label = WAVES > 1 ? __builtin_bit_cast(int, s_row[1]) : te.label;
        Dense d;
        d.init(p, row, WAVES > 1 ? s_row[0] : te.St, label, s, eT, e1);
        char* const out = (char*)p.dZ + row * p.lddz * Row<TYPE>::kBytes;
        char* const first = out + r.head * Row<TYPE>::kBytes;
        if constexpr (CH > 0) {
            d.chunks<TYPE, (WAVES > 1)>(first, tid, NT, r.chunks, w);
        } else {
            for (int c = tid; c < r.chunks; c += 4 * NT) {
                u32x4 x[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) x[u] = r.load(c + u * NT);
                d.chunks<TYPE, (WAVES > 1)>(first, c, NT, r.chunks, x);
            }
        }
        if (single >= 0) store_one<TYPE>(out, single, d.of(x1));
        if (kLate && leader) {
            wave_fence();
            const Sums own = {entries.row[0], entries.row[1], entries.row[2]};
            te.take(entries.row + 3);
            const float loss = te.loss(p, entries, lane, own, eT, close);
            if (lane == 0) p.loss[row] = loss;
        }
        __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): the dense stores have ended
        if constexpr (WAVES > 1) __syncthreads();
        else wave_fence();
        if (!LOSS && p.T > kCloseFrom) te.divergence(p, entries, lane, s, eT, close);  // (one wave a row)
        if (leader) write_exceptions<TYPE>(p, entries, out, lane, label, te.zy, d, close, 0, p.v);
    }
}

// ---- rows in segments -------------------------------------------------------------------------------------
// The largest logit of a segment and its sums; the first segment also notes the logits that the loss needs.
template <int TYPE>
__global__ __launch_bounds__(256) void distill_part_kernel(const DistillParams p) {
    __shared__ float s_red[3][4];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row = blockIdx.x / (unsigned)p.workgroups;
    const int segment = (int)(blockIdx.x % (unsigned)p.workgroups);
    Row<TYPE> r;
    r.init(p, row);
    const int c_begin = min(segment * p.chunks_per_segment, r.chunks), c_end = min(c_begin + p.chunks_per_segment, r.chunks);
    const int single = segment == 0 ? r.single(threadIdx.x) : -1;  // (the first segment takes the single values)
    const float x1 = single >= 0 ? r.at(single) : -__builtin_inff();
    const bool two = p.alpha > 0.0f && p.T != 1.0f;
    const Exponential eT = {p.eT_hi, p.eT_lo}, e1 = {p.e1_hi, p.e1_lo};
    Sums s = {x1, 0.0f, 0.0f};
    for (int c = c_begin + threadIdx.x; c < c_end; c += 4 * 256) {  // four chunks in flight
        u32x4 x[4];
        float top = s.M;
#pragma unroll
        for (int u = 0; u < 4; ++u) x[u] = r.load(c + 256 * u < c_end ? c + 256 * u : r.chunks);
#pragma unroll
        for (int u = 0; u < 4; ++u) top = chunk_max<TYPE>(x[u], top);
        const float base = top == -__builtin_inff() ? 0.0f : top;
        rebase(s, top, two, eT, e1);
        add_chunks<TYPE>(s, x, base, two, eT, e1);
    }
    add_single(s, x1, two, eT, e1);
    s = join_sums<4>(s, s_red, wave, two, eT, e1);
    if (threadIdx.x == 0) {
        float* o = p.part + 3 * (row * p.segments + segment);
        o[0] = s.M;
        o[1] = s.sT;
        o[2] = s.s1;
    }
    if (segment == 0) {
        for (int j = threadIdx.x; j <= p.top; j += 256) {
            int64_t c = -1;
            if (j < p.top) c = load_index(p.top_idx, p.idx_bytes, row * p.top + j);
            else if (p.alpha > 0.0f) c = load_index(p.labels, p.label_bytes, row);
            p.at_top[row * (p.top + 1) + j] = c >= 0 && c < p.v ? r.at((int)c) : 0.0f;
        }
    }
}

// The segments' sums joined (every wave the same way), the loss by the first segment's workgroup, and the gradient of
// this segment.  The logits at the teacher's classes come from at_top, where the loss was asked for, or from Z: of
// classes in other segments they are not used then (dZ may be Z).
template <int TYPE>
__global__ __launch_bounds__(256) void distill_segment_kernel(const DistillParams p) {
    constexpr int N = Row<TYPE>::N;
    __shared__ float s_row[2];
    __shared__ TopEntries entries;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row = blockIdx.x / (unsigned)p.workgroups;
    const int segment = (int)(blockIdx.x % (unsigned)p.workgroups);
    Row<TYPE> r;
    r.init(p, row);
    const int c_begin = min(segment * p.chunks_per_segment, r.chunks), c_end = min(c_begin + p.chunks_per_segment, r.chunks);
    const int single = segment == 0 ? r.single(threadIdx.x) : -1;  // (the first segment takes the single values)
    const float x1 = single >= 0 ? r.at(single) : -__builtin_inff();
    const bool ce = p.alpha > 0.0f, two = ce && p.T != 1.0f;
    const Exponential eT = {p.eT_hi, p.eT_lo}, e1 = {p.e1_hi, p.e1_lo};
    u32x4 w[4];  // (on their way while the first wave looks at the teacher's entries)
    auto load_chunks = [&](int c) {
#pragma unroll
        for (int u = 0; u < 4; ++u) w[u] = r.load(c + 256 * u < c_end ? c + 256 * u : r.chunks);
    };
    if (p.dZ) load_chunks(c_begin + threadIdx.x);
    Teacher te;
    if (wave == 0) {
        te.init<TYPE>(p, r, entries, row, lane, eT);
        if (p.loss) {
            const float* at = p.at_top + row * (p.top + 1);
            for (int j = lane; j < p.top; j += 64) entries.z[j] = at[j];
            te.zy = at[p.top];
            wave_fence();
        }
        if (lane == 0) {
            s_row[0] = te.St;
            s_row[1] = __builtin_bit_cast(float, te.label);
        }
        __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): what was read of Z is here before it may be written
    }
    Sums s = {-__builtin_inff(), 0.0f, 0.0f};
    const float* part = p.part + 3 * row * p.segments;
    if (p.segments == 1) {  // (the row's own, as they are)
        s = {part[0], part[1], part[2]};
    } else {
        for (int i = lane; i < p.segments; i += 64) s.M = __builtin_fmaxf(s.M, part[3 * i]);
        s.M = wave_max(s.M);
        for (int i = lane; i < p.segments; i += 64) {
            Sums o = {part[3 * i], part[3 * i + 1], part[3 * i + 2]};
            rebase(o, s.M, two, eT, e1);
            s.sT += o.sT;
            s.s1 += o.s1;
        }
        s.sT = wave_sum(s.sT);
        s.s1 = two ? wave_sum(s.s1) : ce ? s.sT : 0.0f;
    }
    // (Of the gradient alone the logits of classes in other segments may be gone: no row is close there.)
    bool close = false;
    if (p.loss && wave == 0 && (segment == 0 || p.T > kCloseFrom)) {
        const float loss = te.loss(p, entries, lane, s, eT, close);
        if (segment == 0 && lane == 0) {
            p.loss[row] = loss;
            if (p.stats) {
                p.stats[3 * row] = s.M;
                p.stats[3 * row + 1] = s.sT;
                p.stats[3 * row + 2] = s.s1;
            }
        }
    }
    if (!p.dZ) return;
    __syncthreads();
    Dense d;
    d.init(p, row, s_row[0], __builtin_bit_cast(int, s_row[1]), s, eT, e1);
    char* const out = (char*)p.dZ + row * p.lddz * Row<TYPE>::kBytes;
    char* const first = out + r.head * Row<TYPE>::kBytes;
    for (int c = c_begin + threadIdx.x; c < c_end;) {
        d.chunks<TYPE, true>(first, c, 256, c_end, w);
        c += 4 * 256;
        if (c < c_end) load_chunks(c);
    }
    if (single >= 0) store_one<TYPE>(out, single, d.of(x1));
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): the dense stores have ended
    __syncthreads();
    if (wave == 0) {
        // (the first segment's single values: before its chunks and behind the last)
#pragma unroll 1
        for (int i = 0; i < (segment == 0 ? 3 : 1); ++i) {
            const int from = i == 0 ? r.head + c_begin * N : i == 1 ? 0 : r.head + r.chunks * N;
            write_exceptions<TYPE>(p, entries, out, lane, te.label, te.zy, d, close, from, i == 0 ? r.head + c_end * N : i == 1 ? r.head : p.v);
        }
    }
}

// ---- which kernels a call takes -------------------------------------------------------------------------------------
// Rows are cut where they are few and long, since that takes a second launch: loss and gradient in segments and by a workgroup a
// row, bf16 16 x 32000 11.1 and 10.8 us, 16 x 65536 11.0 and 16.9, 64 x 131072 17.6 and 31.7, 150 x 65536 21.2 and 19.4; fp32 16
// x 16384 10.3 and 7.8, 16 x 32000 10.4 and 10.7, 150 x 131072 46.7 and 43.2.  Into about 512 segments in all, each at least 512
// chunks (16 x 131071 fp32 17.8 us; 256 segments 18.4, 2048 22.1).  The gradient alone takes 1024 chunks a workgroup, four a
// thread (4096 x 50001 bf16 with ordinary stores: 162 us; 512 chunks 187, 2048 183).
constexpr int kFewRows = 128, kLongRow = 4096, kLongRowF32 = 7500;  // rows; chunks
constexpr int kGradSegment = 1024;
struct DistillPlan {
    int segments, chunks_per_segment;
    size_t part_bytes, ws_bytes;
};
static DistillPlan distill_plan(int64_t m, int64_t v, int top, int chunk) {
    DistillPlan d = {};
    const int64_t chunks = ceil_div64(v, chunk);
    d.segments = 1;
    d.chunks_per_segment = (int)chunks;
    if (m < kFewRows && chunks > (chunk == 4 ? kLongRowF32 : kLongRow)) {
        const int64_t want = ceil_div64(512, m), most = ceil_div64(chunks, 512);
        const int64_t s = want < most ? want : most;
        if (s > 1) {
            d.chunks_per_segment = (int)ceil_div64(chunks, s);
            d.segments = (int)ceil_div64(chunks, d.chunks_per_segment);
        }
    }
    if (d.segments > 1) {
        d.part_bytes = ((size_t)m * d.segments * 12 + 255) & ~size_t(255);
        d.ws_bytes = d.part_bytes + (((size_t)m * (top + 1) * 4 + 255) & ~size_t(255));
    }
    return d;
}
static int chunk_of(int type) { return type == KQ_T_F32 ? 4 : 8; }

template <int TYPE, bool LOSS, bool GRAD>
static void launch_rows(const DistillParams& p, hipStream_t s) {
    const int chunks = p.v / Row<TYPE>::N;
    const dim3 four((unsigned)ceil_div64(p.m, 4)), one((unsigned)p.m);
    // (16 chunks a thread leave a CU one row, whose loads, sums and stores then come after each other: 1024 x 65536 fp32 103 us
    // and 126 read twice, 1024 x 50000 85 and 94; 2048 x 128256 bf16 212 and 238, but 100001 200 and 197, and with two
    // exponentials 253 and 211)
    const bool two = p.alpha > 0.0f && p.T != 1.0f;
    const bool hold = GRAD && chunks <= 16384 && (TYPE == KQ_T_F32 || (chunks > 13000 && !two));
    if (chunks <= 128) distill_row_kernel<TYPE, 2, 1, LOSS, GRAD><<<four, 256, 0, s>>>(p);
    else if (chunks <= 512) distill_row_kernel<TYPE, 8, 1, LOSS, GRAD><<<four, 256, 0, s>>>(p);
    if constexpr (LOSS) {
        if (chunks <= 512) return;
        if (chunks <= 2048) distill_row_kernel<TYPE, 8, 4, LOSS, GRAD><<<one, 256, 0, s>>>(p);
        else if (chunks <= 4096) distill_row_kernel<TYPE, 4, 16, LOSS, GRAD><<<one, 1024, 0, s>>>(p);
        else if (chunks <= 8192) distill_row_kernel<TYPE, 8, 16, LOSS, GRAD><<<one, 1024, 0, s>>>(p);
        else if (hold) distill_row_kernel<TYPE, GRAD ? 16 : 0, 16, LOSS, GRAD><<<one, 1024, 0, s>>>(p);
        else distill_row_kernel<TYPE, 0, 16, LOSS, GRAD><<<one, 1024, 0, s>>>(p);
    }
}
template <int TYPE>
static hipError_t launch_type(DistillParams p, hipStream_t s) {
    if (p.loss && p.segments == 1) {
        if (p.dZ) launch_rows<TYPE, true, true>(p, s);
        else launch_rows<TYPE, true, false>(p, s);
        return hipGetLastError();
    }
    if (!p.loss && p.v / Row<TYPE>::N <= 512) {
        launch_rows<TYPE, false, true>(p, s);
        return hipGetLastError();
    }
    if (p.loss) {
        p.workgroups = p.segments;
        distill_part_kernel<TYPE><<<dim3((unsigned)(p.m * p.segments)), 256, 0, s>>>(p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    // (the loss alone: a row's first segment has it)
    p.workgroups = p.dZ ? (int)ceil_div64(ceil_div64(p.v, Row<TYPE>::N), p.chunks_per_segment) : 1;
    distill_segment_kernel<TYPE><<<dim3((unsigned)(p.m * p.workgroups)), 256, 0, s>>>(p);
    return hipGetLastError();
}
static hipError_t launch_distill(const DistillParams& p, hipStream_t s) {
    return p.type == KQ_T_F32 ? launch_type<KQ_T_F32>(p, s) : p.type == KQ_T_BF16 ? launch_type<KQ_T_BF16>(p, s) : launch_type<KQ_T_F16>(p, s);
}

}  // namespace kq

using namespace kq;

namespace {
bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
bool plain_type(int32_t t) { return t == KQ_T_F32 || t == KQ_T_BF16 || t == KQ_T_F16; }
bool valid_tensor(const void* p, int32_t type) { return p != nullptr && aligned(p, type == KQ_T_F32 ? 4 : 2); }

kq_status make_params(DistillParams& p, const kq_distill_args* a) {
    if (a == nullptr || a->m < 0 || a->v < 1 || a->top < 1) return KQ_ERR_ARG;
    if (a->m > KQ_GROUP_MAX_ROWS || a->v > KQ_DISTILL_MAX_CLASSES || a->m * a->v > KQ_DISTILL_MAX_LOGITS || a->top > KQ_DISTILL_MAX_TOP)
        return KQ_ERR_UNSUPPORTED;
    if (!plain_type(a->type) || !plain_type(a->top_type) || (a->idx_bytes != 4 && a->idx_bytes != 8)) return KQ_ERR_UNSUPPORTED;
    if (!(a->temperature >= 0x1p-10f && a->temperature <= 0x1p20f)) return KQ_ERR_UNSUPPORTED;
    if (!(a->alpha >= 0.0f && a->alpha <= 1.0f)) return KQ_ERR_ARG;
    if (a->alpha > 0.0f && a->label_bytes != 4 && a->label_bytes != 8) return KQ_ERR_UNSUPPORTED;
    if (a->m > 0) {
        if (!valid_tensor(a->Z, a->type) || a->ldz < a->v || a->ldz > (int64_t(1) << 40)) return KQ_ERR_ARG;
        if (!valid_tensor(a->top_values, a->top_type) || !a->top_idx || !aligned(a->top_idx, a->idx_bytes)) return KQ_ERR_ARG;
        if (a->alpha > 0.0f && (!a->labels || !aligned(a->labels, a->label_bytes))) return KQ_ERR_ARG;
    }
    p = {};
    p.Z = a->Z;
    p.type = a->type;
    p.ldz = a->ldz;
    p.m = a->m;
    p.v = (int)a->v;
    p.top_values = a->top_values;
    p.top_type = a->top_type;
    p.top_idx = a->top_idx;
    p.idx_bytes = a->idx_bytes;
    p.top = a->top;
    p.labels = a->alpha > 0.0f ? a->labels : nullptr;
    p.label_bytes = a->label_bytes;
    p.T = a->temperature;
    p.alpha = a->alpha;
    const Exponential eT = Exponential::of(p.T), e1 = Exponential::of(1.0f);
    p.eT_hi = eT.hi;
    p.eT_lo = eT.lo;
    p.e1_hi = e1.hi;
    p.e1_lo = e1.lo;
    return KQ_OK;
}
kq_status add_gradient(DistillParams& p, const float* dloss, float scale, void* dZ, int64_t lddz) {
    if (!aligned(dloss, 4)) return KQ_ERR_ARG;
    if (p.m > 0 && (!valid_tensor(dZ, p.type) || lddz < p.v || lddz > (int64_t(1) << 40))) return KQ_ERR_ARG;
    p.dloss = dloss;
    p.scale = scale;
    p.dZ = dZ;
    p.lddz = lddz;
    return KQ_OK;
}
kq_status add_segments(DistillParams& p, void* ws, size_t ws_bytes) {
    const DistillPlan d = distill_plan(p.m, p.v, p.top, chunk_of(p.type));
    p.segments = d.segments;
    p.chunks_per_segment = d.chunks_per_segment;
    if (d.ws_bytes == 0) return KQ_OK;
    if (ws == nullptr || !aligned(ws, 256) || ws_bytes < d.ws_bytes) return KQ_ERR_WORKSPACE;
    p.part = (float*)ws;
    p.at_top = (float*)((char*)ws + d.part_bytes);
    return KQ_OK;
}
kq_status hip_status(hipError_t e) { return e == hipSuccess ? KQ_OK : KQ_ERR_HIP; }
}  // namespace

extern "C" {

size_t kq_distill_workspace_bytes(int32_t type, int64_t m, int64_t v, int32_t top) {
    if (!plain_type(type) || m < 1 || v < 1 || top < 1 || m > KQ_GROUP_MAX_ROWS || v > KQ_DISTILL_MAX_CLASSES ||
        m * v > KQ_DISTILL_MAX_LOGITS || top > KQ_DISTILL_MAX_TOP) return 0;
    return distill_plan(m, v, top, chunk_of(type)).ws_bytes;
}

kq_status kq_distill(const kq_distill_args* args, const float* dloss, float scale, float* loss, void* dZ, int64_t lddz,
                     void* ws, size_t ws_bytes, void* stream) {
    DistillParams p;
    kq_status st = make_params(p, args);
    if (st != KQ_OK || (st = add_gradient(p, dloss, scale, dZ, lddz)) != KQ_OK) return st;
    if (p.m == 0) return KQ_OK;
    if (!loss || !aligned(loss, 4)) return KQ_ERR_ARG;
    p.loss = loss;
    if ((st = add_segments(p, ws, ws_bytes)) != KQ_OK) return st;
    return hip_status(launch_distill(p, (hipStream_t)stream));
}

kq_status kq_distill_loss(const kq_distill_args* args, float* loss, float* stats, void* ws, size_t ws_bytes, void* stream) {
    DistillParams p;
    kq_status st = make_params(p, args);
    if (st != KQ_OK) return st;
    if (p.m == 0) return KQ_OK;
    if (!loss || !aligned(loss, 4) || !stats || !aligned(stats, 4)) return KQ_ERR_ARG;
    p.loss = loss;
    p.stats = stats;
    if ((st = add_segments(p, ws, ws_bytes)) != KQ_OK) return st;
    return hip_status(launch_distill(p, (hipStream_t)stream));
}

kq_status kq_distill_grad(const kq_distill_args* args, const float* stats, const float* dloss, float scale, void* dZ,
                          int64_t lddz, void* stream) {
    DistillParams p;
    kq_status st = make_params(p, args);
    if (st != KQ_OK || (st = add_gradient(p, dloss, scale, dZ, lddz)) != KQ_OK) return st;
    if (p.m == 0) return KQ_OK;
    if (!stats || !aligned(stats, 4)) return KQ_ERR_ARG;
    p.part = const_cast<float*>(stats);
    p.segments = 1;
    p.chunks_per_segment = kGradSegment;
    return hip_status(launch_distill(p, (hipStream_t)stream));
}

}  // extern "C"
