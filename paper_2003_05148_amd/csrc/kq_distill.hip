// Distillation from a teacher's top logits: the loss of every row and the gradient of its logits.
//
//   p = softmax of the row's present teacher logits / T;  q = softmax of z / T;  s = softmax of z
//   loss = (1 - alpha) T^2 sum_j p_j (log p_j - log q_idx[j]) + alpha (-log s_label)
//   dz_c = d [ (1 - alpha) T (q_c - p_c) + alpha (s_c - [c = label]) ]
// With M the row's largest logit everything is taken from differences to it: q_c = exp((z_c - M) / T) / S_T.
// The gradient is dense in q and s and differs from that at the teacher's classes and the label: the dense part is
// written first, and once those stores have ended the few others are written over it.
#include "kq_values.h"

namespace kq {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

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
    float* loss;
    float* stats;
    const float* in_stats;
    void* dZ;
    int64_t lddz;
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
__device__ __forceinline__ void store_one(void* base, int64_t at, float v) {
    if constexpr (TYPE == KQ_T_F32) ((float*)base)[at] = v;
    else ((uint16_t*)base)[at] = Act<TYPE == KQ_T_BF16>::one(v);
}

struct Max {
    static __device__ __forceinline__ float of(float a, float b) { return __builtin_fmaxf(a, b); }
};
struct Sum {
    static __device__ __forceinline__ float of(float a, float b) { return a + b; }
};
// over the workgroup, the same value in every thread
template <class OP, int WAVES>
__device__ __forceinline__ float reduce(float v, float* s_red) {
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) v = OP::of(v, __shfl_xor(v, off));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s_red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = s_red[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v = OP::of(v, s_red[w]);
    return v;
}

// A workgroup a row.  LOSS: the loss and (stats given) what the gradient needs; GRAD: the gradient, from in_stats
// where LOSS is not asked for.
template <int TYPE, bool LOSS, bool GRAD>
__global__ __launch_bounds__(256) void distill_row_kernel(const DistillParams p) {
    constexpr int kWaves = 4;
    __shared__ float s_red[kWaves];
    __shared__ int s_idx[KQ_DISTILL_MAX_TOP];
    __shared__ float s_p[KQ_DISTILL_MAX_TOP];
    __shared__ int s_label_hit;
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x, z_at = row * p.ldz;
    const float cT = kLog2e / p.T;
    const bool kl = p.alpha < 1.0f, ce = p.alpha > 0.0f, two = ce && p.T != 1.0f;

    float M, ST, S1;
    if constexpr (LOSS) {
        float a = -__builtin_inff();
        for (int c = tid; c < p.v; c += 256) a = __builtin_fmaxf(a, load_value_as<TYPE>(p.Z, z_at + c));
        M = reduce<Max, kWaves>(a, s_red);
        float sT = 0.0f, s1 = 0.0f;
        for (int c = tid; c < p.v; c += 256) {
            const float d = load_value_as<TYPE>(p.Z, z_at + c) - M;
            sT += __builtin_amdgcn_exp2f(d * cT);
            if (two) s1 += __builtin_amdgcn_exp2f(d * kLog2e);
        }
        ST = reduce<Sum, kWaves>(sT, s_red);
        S1 = two ? reduce<Sum, kWaves>(s1, s_red) : ce ? ST : 0.0f;
        if (p.stats && tid == 0) {
            p.stats[3 * row] = M;
            p.stats[3 * row + 1] = ST;
            p.stats[3 * row + 2] = S1;
        }
    } else {
        M = p.in_stats[3 * row];
        ST = p.in_stats[3 * row + 1];
        S1 = p.in_stats[3 * row + 2];
    }

    // the teacher's entries, one a thread
    int idx = -1;
    float t = -__builtin_inff(), zt = 0.0f;
    if (kl && tid < p.top) {
        const int64_t i = load_index(p.top_idx, p.idx_bytes, row * p.top + tid);
        t = load_any(p.top_values, p.top_type, row * p.top + tid);
        if (i >= 0 && i < p.v && t != -__builtin_inff()) {
            idx = (int)i;
            zt = load_value_as<TYPE>(p.Z, z_at + idx) - M;
        } else {
            t = -__builtin_inff();
        }
    }
    float pj = 0.0f, loss = 0.0f, any = 0.0f, St = 0.0f;
    if (kl) {
        any = reduce<Max, kWaves>(idx >= 0 ? 1.0f : 0.0f, s_red);
        const float tM = reduce<Max, kWaves>(t, s_red);
        const float e = idx >= 0 ? __builtin_amdgcn_exp2f((t - tM) * cT) : 0.0f;
        St = reduce<Sum, kWaves>(e, s_red);
        pj = idx >= 0 ? e / St : 0.0f;
        if constexpr (LOSS) {
            const float term = ((t - tM) - zt) * (1.0f / p.T) + kLn2 * (__builtin_amdgcn_logf(ST) - __builtin_amdgcn_logf(St));
            loss = reduce<Sum, kWaves>(idx >= 0 && pj != 0.0f ? pj * term : 0.0f, s_red) * ((1.0f - p.alpha) * p.T * p.T);
        }
    }
    int64_t label = -1;
    if (ce) label = load_index(p.labels, p.label_bytes, row);
    const bool has = ce && label >= 0 && label < p.v;
    float zy = 0.0f;
    if (has) zy = load_value_as<TYPE>(p.Z, z_at + label) - M;
    if constexpr (LOSS) {
        if (has) loss += p.alpha * (kLn2 * __builtin_amdgcn_logf(S1) - zy);
        if (tid == 0) p.loss[row] = loss;
    }

    if constexpr (GRAD) {
        const float d = p.dloss ? p.dloss[row] : p.scale;
        const float wT = kl ? d * (1.0f - p.alpha) * p.T : 0.0f, w1 = has ? d * p.alpha : 0.0f;
        // (0 times St: a NaN of the teacher's is one of the whole row's)
        const float fT = any > 0.0f ? wT / ST + 0.0f * St : 0.0f, f1 = has ? w1 / S1 : 0.0f;
        auto dense = [&](float dz) {
            const float a = fT * __builtin_amdgcn_exp2f(dz * cT);
            return has ? a + f1 * __builtin_amdgcn_exp2f(dz * kLog2e) : a;
        };
        s_idx[tid] = idx;
        s_p[tid] = pj;
        if (tid == 0) s_label_hit = 0;
        __syncthreads();
        const int64_t o_at = row * p.lddz;
        for (int c = tid; c < p.v; c += 256) store_one<TYPE>(p.dZ, o_at + c, dense(load_value_as<TYPE>(p.Z, z_at + c) - M));
        // an index that stands more than once is written by its first place
        bool first = idx >= 0;
        float pc = 0.0f;
        if (first) {
            for (int j = 0; j < p.top; ++j) {
                if (s_idx[j] != idx) continue;
                if (j < tid) first = false;
                pc += s_p[j];
            }
        }
        if (first && has && idx == label) s_label_hit = 1;
        __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): the dense stores have ended
        __syncthreads();
        if (first) store_one<TYPE>(p.dZ, o_at + idx, dense(zt) - wT * pc - (has && idx == label ? w1 : 0.0f));
        if (tid == 0 && has && !s_label_hit) store_one<TYPE>(p.dZ, o_at + label, dense(zy) - w1);
    }
}

template <bool LOSS, bool GRAD>
static hipError_t launch_distill(const DistillParams& p, hipStream_t s) {
    const dim3 grid((unsigned)p.m), block(256);
    if (p.type == KQ_T_F32) distill_row_kernel<KQ_T_F32, LOSS, GRAD><<<grid, block, 0, s>>>(p);
    else if (p.type == KQ_T_BF16) distill_row_kernel<KQ_T_BF16, LOSS, GRAD><<<grid, block, 0, s>>>(p);
    else distill_row_kernel<KQ_T_F16, LOSS, GRAD><<<grid, block, 0, s>>>(p);
    return hipGetLastError();
}

}  // namespace kq

using namespace kq;

namespace {
bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
bool plain_type(int32_t t) { return t == KQ_T_F32 || t == KQ_T_BF16 || t == KQ_T_F16; }
bool valid_tensor(const void* p, int32_t type) { return p != nullptr && aligned(p, type == KQ_T_F32 ? 4 : 2); }

kq_status make_params(DistillParams& p, const kq_distill_args* a) {
    if (a == nullptr || a->m < 0 || a->v < 1 || a->top < 1) return KQ_ERR_ARG;
    if (a->m > KQ_GROUP_MAX_ROWS || a->v > KQ_DISTILL_MAX_CLASSES || a->top > KQ_DISTILL_MAX_TOP) return KQ_ERR_UNSUPPORTED;
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
kq_status hip_status(hipError_t e) { return e == hipSuccess ? KQ_OK : KQ_ERR_HIP; }
}  // namespace

extern "C" {

size_t kq_distill_workspace_bytes(int64_t m, int64_t v, int32_t top) {
    (void)m, (void)v, (void)top;
    return 0;
}

kq_status kq_distill(const kq_distill_args* args, const float* dloss, float scale, float* loss, void* dZ, int64_t lddz,
                     void* ws, size_t ws_bytes, void* stream) {
    (void)ws, (void)ws_bytes;
    DistillParams p;
    kq_status st = make_params(p, args);
    if (st != KQ_OK || (st = add_gradient(p, dloss, scale, dZ, lddz)) != KQ_OK) return st;
    if (p.m == 0) return KQ_OK;
    if (!loss || !aligned(loss, 4)) return KQ_ERR_ARG;
    p.loss = loss;
    return hip_status(launch_distill<true, true>(p, (hipStream_t)stream));
}

kq_status kq_distill_loss(const kq_distill_args* args, float* loss, float* stats, void* ws, size_t ws_bytes, void* stream) {
    (void)ws, (void)ws_bytes;
    DistillParams p;
    const kq_status st = make_params(p, args);
    if (st != KQ_OK) return st;
    if (p.m == 0) return KQ_OK;
    if (!loss || !aligned(loss, 4) || !stats || !aligned(stats, 4)) return KQ_ERR_ARG;
    p.loss = loss;
    p.stats = stats;
    return hip_status(launch_distill<true, false>(p, (hipStream_t)stream));
}

kq_status kq_distill_grad(const kq_distill_args* args, const float* stats, const float* dloss, float scale, void* dZ,
                          int64_t lddz, void* stream) {
    DistillParams p;
    kq_status st = make_params(p, args);
    if (st != KQ_OK || (st = add_gradient(p, dloss, scale, dZ, lddz)) != KQ_OK) return st;
    if (p.m == 0) return KQ_OK;
    if (!stats || !aligned(stats, 4)) return KQ_ERR_ARG;
    p.in_stats = stats;
    return hip_status(launch_distill<false, true>(p, (hipStream_t)stream));
}

}  // extern "C"
